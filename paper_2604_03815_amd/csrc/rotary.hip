// Rotary positions (gfx950): each pair (a, b) of a row's first `rot` dimensions
// is turned by t = position * frequency and scaled by m,
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t);
// a pair is two neighbours (interleaved) or dimensions i and i + rot / 2.
// The gradient of a turn is the turn back, so one kernel serves both.
//
// Angles: the frequency in turns a position is held as a 64-bit fraction, so
// position * frequency modulo one turn is one wrapping integer product: far
// positions lose nothing.  The fraction is cut off at 2^-63 turns, times a position
// of at most 2^31, and the product's top 32 bits are used: off by less than 2^-32
// turns twice, 2^-28 radians.  Its top two bits (rounded) pick the quadrant; the rest, at most
// pi/4, goes through the Taylor sums of sine and cosine (to x^9 and x^10:
// remainders below 2e-9).  All in float32 (the rest's conversion, its factor and
// their product, 2.5 2^-24 of it, and the last sum's half step, 2^-25: below 2^-22 in
// all); the row's values are rounded once.
//
// A thread takes P pairs of one token for up to four heads, so that an angle is
// formed once for them; the threads of a token's heads are neighbours, so that
// a wave reads and writes whole tokens' rows.  Bound by memory: a row is read
// once and written once, 16 bytes a lane where the sizes allow.  Cold data, us:
// 16,383 tokens of 40 heads, d = 128, rot = 64, fp16 70 (4.8 TB/s; 84 where
// neighbours took other tokens, 92 with a thread for each head, 77 with eight
// heads a thread), 100,000 of 8 heads, d = 32, float32 to bf16 and back 72 (4.2
// TB/s; 76, 75 and 89).
#include <cmath>
#include <cstring>

#include "kmip_device.h"
#include "kmip_internal.h"

namespace kmip {
namespace {

constexpr int kMostPairs = 128;

struct Side {
    const char* x;
    char* y;
    int64_t x_row, x_head, y_row, y_head;   // bytes
};

struct RotaryArgs {
    Side s[2];
    const int32_t* positions;
    uint32_t threads;                 // N * group * units
    int32_t units, rot_units;         // threads a row, those with pairs
    int32_t heads, first_heads, group;   // heads of both, of the first, threads that share them
    int32_t rot;
    float cos_scale, sin_scale;
    uint64_t turns[kMostPairs];
};

struct Half16 {   // float16
    typedef uint16_t word;
    static __device__ __forceinline__ float widen(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
struct Brain16 {   // bfloat16
    typedef uint16_t word;
    static __device__ __forceinline__ float widen(uint16_t x) { return bf16_bits_to_f32(x); }
    static __device__ __forceinline__ uint16_t round(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
struct Single {
    typedef float word;
    static __device__ __forceinline__ float widen(float x) { return x; }
    static __device__ __forceinline__ float round(float x) { return x; }
};

// P values of type T, aligned to their size (at most 16 bytes).
template <typename T, int P>
struct alignas(sizeof(typename T::word) * P) Pack {
    typename T::word v[P];
};

// PAST: past the caches, for results that do not fit them.
template <bool PAST, typename T, int P>
__device__ __forceinline__ void put(char* p, const Pack<T, P>& w) {
    if constexpr (PAST) {
        typedef uint32_t words __attribute__((ext_vector_type(sizeof(w) / 4)));
        __builtin_nontemporal_store(__builtin_bit_cast(words, w), reinterpret_cast<words*>(p));
    } else {
        *reinterpret_cast<Pack<T, P>*>(p) = w;
    }
}

// sin and cos of phase / 2^32 turns.
__device__ __forceinline__ void sin_cos(uint32_t phase, float* s, float* c) {
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float z = x * x;
    // (fused steps written out, here and in turn(): every form rounds alike)
    const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const float u = (quarter & 1) ? cs : sn, w = (quarter & 1) ? sn : cs;
    *s = (quarter & 2) ? -u : u;
    *c = ((quarter + 1) & 2) ? -w : w;
}

// (u, v) of a thread turned: INTER with P > 1: P / 2 pairs in each, else pairs (u[e], v[e]).
template <int P, bool INTER>
__device__ __forceinline__ void turn(float (&u)[P], float (&v)[P], const float (&c)[P], const float (&s)[P]) {
    auto pair = [](float& a, float& b, float cs, float sn) {
        const float bs = b * sn, as = a * sn;
        a = fmaf(a, cs, -bs);
        b = fmaf(b, cs, as);
    };
#pragma unroll
    for (int e = 0; e < P; ++e) {
        if constexpr (INTER && P > 1) {
            if (e < P / 2)
                pair(u[2 * e], u[2 * e + 1], c[e], s[e]);
            else
                pair(v[2 * e - P], v[2 * e - P + 1], c[e], s[e]);
        } else {
            pair(u[e], v[e], c[e], s[e]);
        }
    }
}

// Rows of a thread, whose loads go out before the first store (which may write
// the same memory, so that the compiler cannot move a load across it).
constexpr int kRows = 4;

template <typename TI, typename TO, int P, bool INTER, bool PAST>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
    constexpr int kIn = sizeof(typename TI::word), kOut = sizeof(typename TO::word);
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    if (id >= a.threads) return;
    const uint32_t place = id / (uint32_t)a.units;
    const int unit = (int)(id - place * (uint32_t)a.units);
    const uint32_t token = place / (uint32_t)a.group;
    const int h0 = (int)(place - token * (uint32_t)a.group);
    const bool turned = unit < a.rot_units;
    // A thread's two runs of P values lie half of the turned (or of the passed
    // on) dimensions apart: neighbouring threads touch neighbouring runs.
    int one, two;
    if (turned) {
        one = P * unit, two = one + a.rot / 2;
        if (INTER && P == 1) one = 2 * unit, two = one + 1;
    } else {
        one = a.rot + P * (unit - a.rot_units), two = one + P * (a.units - a.rot_units);
    }
    float c[P], s[P];
    if (turned) {
        const uint64_t pos = (uint64_t)(int64_t)(a.positions != nullptr ? a.positions[token] : (int32_t)token);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            int i = P * unit + e;
            if (INTER && P > 1) i = e < P / 2 ? one / 2 + e : two / 2 + e - P / 2;
            sin_cos((uint32_t)((pos * a.turns[i]) >> 32), &s[e], &c[e]);
            c[e] *= a.cos_scale;
            s[e] *= a.sin_scale;
        }
    }
    for (int h = h0; h < a.heads; h += kRows * a.group) {
        Pack<TI, P> x[kRows][2];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int hr = h + r * a.group;
            if (hr >= a.heads) break;
            const bool second = hr >= a.first_heads;
            const Side& t = a.s[second];
            const char* p = t.x + (int64_t)token * t.x_row + (second ? hr - a.first_heads : hr) * t.x_head;
            x[r][0] = *reinterpret_cast<const Pack<TI, P>*>(p + one * kIn);
            x[r][1] = *reinterpret_cast<const Pack<TI, P>*>(p + two * kIn);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int hr = h + r * a.group;
            if (hr >= a.heads) break;
            const bool second = hr >= a.first_heads;
            const Side& t = a.s[second];
            char* y = t.y + (int64_t)token * t.y_row + (second ? hr - a.first_heads : hr) * t.y_head;
            float u[P], v[P];
#pragma unroll
            for (int e = 0; e < P; ++e) u[e] = TI::widen(x[r][0].v[e]), v[e] = TI::widen(x[r][1].v[e]);
            if (turned) turn<P, INTER>(u, v, c, s);
            Pack<TO, P> w[2];
#pragma unroll
            for (int e = 0; e < P; ++e) w[0].v[e] = TO::round(u[e]), w[1].v[e] = TO::round(v[e]);
            put<PAST>(y + one * kOut, w[0]);
            put<PAST>(y + two * kOut, w[1]);
        }
    }
}

int32_t size_of(int32_t dtype) { return dtype == KMIP_FP32 ? 4 : 2; }

kmip_status_t ok() { return record_error(KMIP_OK, "%s", ""); }

template <typename TI, typename TO, int P, bool PAST>
void launch(const RotaryArgs& a, bool inter, dim3 grid, hipStream_t stream) {
    if (inter)
        hipLaunchKernelGGL((rotary_kernel<TI, TO, P, true, PAST>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((rotary_kernel<TI, TO, P, false, PAST>), grid, dim3(256), 0, stream, a);
}

template <typename TI, typename TO>
void launch_types(const RotaryArgs& a, int pairs, bool inter, bool past, dim3 grid, hipStream_t stream) {
    if constexpr (sizeof(typename TI::word) == 2 && sizeof(typename TO::word) == 2) {
        if (pairs == 8) return past ? launch<TI, TO, 8, true>(a, inter, grid, stream) : launch<TI, TO, 8, false>(a, inter, grid, stream);
    }
    if (pairs == 4) return past ? launch<TI, TO, 4, true>(a, inter, grid, stream) : launch<TI, TO, 4, false>(a, inter, grid, stream);
    launch<TI, TO, 1, false>(a, inter, grid, stream);
}

template <typename TI>
void launch_out(const RotaryArgs& a, int32_t out, int pairs, bool inter, bool past, dim3 grid, hipStream_t stream) {
    if (out == KMIP_BF16) launch_types<TI, Brain16>(a, pairs, inter, past, grid, stream);
    if (out == KMIP_FP16) launch_types<TI, Half16>(a, pairs, inter, past, grid, stream);
    if (out == KMIP_FP32) launch_types<TI, Single>(a, pairs, inter, past, grid, stream);
}

}  // namespace
}  // namespace kmip

extern "C" kmip_status_t kmip_rotary(const void* X, void* Y, int32_t H, const void* X2, void* Y2, int32_t H2,
                                     int32_t dtype_in, int32_t dtype_out, const int64_t* strides, const int32_t* positions,
                                     const double* freqs, int64_t N, int32_t d, int32_t rot, int32_t interleaved,
                                     float magnitude, int32_t inverse, void* stream) {
    using namespace kmip;
    if (N < 0 || N >= (int64_t(1) << 31)) return record_error(KMIP_ERR_INVALID_ARG, "N=%lld out of range", (long long)N);
    if (H < 1 || H2 < 0 || (int64_t)H + H2 >= (1 << 20)) return record_error(KMIP_ERR_INVALID_ARG, "H=%d, H2=%d", H, H2);
    if (d < 2 || d > 2 * kMostPairs || d % 2 != 0) return record_error(KMIP_ERR_UNSUPPORTED, "d=%d must be even, 2 .. %d", d, 2 * kMostPairs);
    if (rot < 2 || rot > d || rot % 2 != 0) return record_error(KMIP_ERR_INVALID_ARG, "rot=%d must be even, 2 .. d", rot);
    if (dtype_in < KMIP_BF16 || dtype_in > KMIP_FP32 || dtype_out < KMIP_BF16 || dtype_out > KMIP_FP32)
        return record_error(KMIP_ERR_UNSUPPORTED, "dtypes %d, %d", dtype_in, dtype_out);
    if (freqs == nullptr) return record_error(KMIP_ERR_INVALID_ARG, "null freqs");
    uint32_t bits;
    std::memcpy(&bits, &magnitude, sizeof(bits));
    if ((bits & 0x7F800000u) == 0x7F800000u) return record_error(KMIP_ERR_INVALID_ARG, "magnitude must be finite");
    RotaryArgs a{};
    for (int32_t i = 0; i < rot / 2; ++i) {
        uint64_t fb;
        std::memcpy(&fb, &freqs[i], sizeof(fb));
        if (((fb >> 52) & 0x7FF) == 0x7FF) return record_error(KMIP_ERR_INVALID_ARG, "freqs[%d] is not finite", i);
        // the fraction of a turn, to 2^-63 (signed, so that it wraps)
        const long double turns = (long double)freqs[i] * 0.15915494309189533576888376337251436L;
        const long double part = turns < 0x1p62L && turns > -0x1p62L ? turns - (long double)(int64_t)turns : turns - floorl(turns);
        a.turns[i] = (uint64_t)(int64_t)(part * 0x1p63L) << 1;
    }
    if (N == 0) return ok();
    if (!X || !Y || (H2 > 0 && (!X2 || !Y2))) return record_error(KMIP_ERR_INVALID_ARG, "null buffer passed to kmip_rotary");
    const int32_t si = size_of(dtype_in), so = size_of(dtype_out);
    const int64_t packed[8] = {(int64_t)H * d, d, (int64_t)H * d, d, (int64_t)H2 * d, d, (int64_t)H2 * d, d};
    const int64_t* st = strides != nullptr ? strides : packed;
    // the longest runs, up to 16 bytes, that sizes, strides and pointers allow
    auto fits = [&](int p) {
        if (rot / 2 % p != 0 || (d - rot) % (2 * p) != 0 || p * si > 16 || p * so > 16) return false;
        for (int t = 0; t < (H2 > 0 ? 2 : 1); ++t) {
            const void *x = t ? X2 : X, *y = t ? Y2 : Y;
            if (reinterpret_cast<uintptr_t>(x) % (p * si) != 0 || reinterpret_cast<uintptr_t>(y) % (p * so) != 0) return false;
            for (int i = 0; i < 4; ++i)
                if (st[4 * t + i] % p != 0) return false;
        }
        return true;
    };
    const int pairs = fits(8) ? 8 : fits(4) ? 4 : 1;
    for (int t = 0; t < (H2 > 0 ? 2 : 1); ++t) {
        const void *x = t ? X2 : X, *y = t ? Y2 : Y;
        if (reinterpret_cast<uintptr_t>(x) % si != 0 || reinterpret_cast<uintptr_t>(y) % so != 0)
            return record_error(KMIP_ERR_INVALID_ARG, "buffers must be aligned to their type");
        for (int i = 0; i < 4; ++i)
            if (st[4 * t + i] < 0) return record_error(KMIP_ERR_INVALID_ARG, "negative stride");
        if (x == y && (si != so || st[4 * t] != st[4 * t + 2] || st[4 * t + 1] != st[4 * t + 3]))
            return record_error(KMIP_ERR_INVALID_ARG, "in place needs one type and the same strides");
        a.s[t] = Side{static_cast<const char*>(t ? X2 : X), static_cast<char*>(t ? Y2 : Y), st[4 * t] * si,
                      st[4 * t + 1] * si, st[4 * t + 2] * so, st[4 * t + 3] * so};
    }
    a.positions = positions;
    a.units = d / (2 * pairs);
    a.rot_units = rot / 2 / pairs;
    a.heads = H + H2;
    a.first_heads = H;
    // Threads a token and unit: each takes up to kRows heads, one where that leaves
    // the chip's SIMDs less than two waves (or all, where ids would pass 32 bits)
    const int64_t runs = N * a.units;
    a.group = runs * a.heads < (int64_t(1) << 17) ? a.heads : (a.heads + kRows - 1) / kRows;
    if (runs * a.group >= (int64_t(1) << 32) - 256) a.group = 1;
    const int64_t threads = runs * a.group;
    if (threads >= (int64_t(1) << 32) - 256) return record_error(KMIP_ERR_INVALID_ARG, "N * d / %d >= 2^32", 2 * pairs);
    a.threads = (uint32_t)threads;
    // Results larger than the chip's 32 MB of L2 are stored past it (100,000 tokens
    // of 8 heads, d = 32, float32 to bf16 and back 75 us without, 63 with)
    const bool past = pairs > 1 && N * a.heads * d * so > (int64_t(32) << 20);
    a.rot = rot;
    a.cos_scale = magnitude;
    a.sin_scale = inverse ? -magnitude : magnitude;
    const dim3 grid((unsigned)((threads + 255) / 256));
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool inter = interleaved != 0;
    if (dtype_in == KMIP_BF16) launch_out<Brain16>(a, dtype_out, pairs, inter, past, grid, s);
    if (dtype_in == KMIP_FP16) launch_out<Half16>(a, dtype_out, pairs, inter, past, grid, s);
    if (dtype_in == KMIP_FP32) launch_out<Single>(a, dtype_out, pairs, inter, past, grid, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return record_error(KMIP_ERR_HIP, "rotary launch: %s", hipGetErrorString(e));
    return ok();
}
