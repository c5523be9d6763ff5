// Full softmax attention over packed sequences: forward (gfx950).
//
// For query row i (a token and head) of a sequence with keys j:
//   s_ij = q_i . k_j,  out_i = sum_j p_ij v_j,  p_ij = exp(scale s_ij - lse_i),
//   lse_i = log sum_j exp(scale s_ij),
// in one pass over the keys with a running maximum m and sum l: a tile's
// weights are 2^(c (s - m)), c = scale log2 e, and what was summed before a
// new maximum is multiplied by 2^(c (m_old - m_new)).  The score matrix is
// never stored.
//
// Rows: the query heads that share a key head and the tokens of a sequence
// form one list, row = token * rep + head in the group, so that a tile of 32
// rows reads the keys once for all its heads (a single token of 8 grouped heads
// fills 8 columns of one product instead of one of 8).
//
// Two forms:
//   ROWS = 128: four waves of 32 rows share each tile of keys (two buffers,
//     one barrier a tile); with HALVES = 2 two such groups, each on half of
//     the tiles, whose sums are added at the end;
//   ROWS = 32: the four waves hold the same rows and take every fourth block of
//     32 keys, each with LDS of its own and no barrier, and are joined at the
//     end.  For few rows.
// With `split` keys per job, jobs of a row tile take runs of its keys and write
// partial sums, which full_join_kernel joins in the order of the runs.
//
// Measured (MI355X) and what bounds it:
//   - d = 128: matrix and vector instructions, which overlap in part, and power
//     (2.0 to 2.2 GHz).  A prompt of 16,384 tokens, 8 heads on 2 key heads, causal: 540
//     us, 1.02 PFLOP/s (a library product of 8192^3: 1.2); the matrix units are busy 58% of the
//     time, the vector units issue 48% of it.  Interleaving the scores of a
//     tile, the weights of the one before and the product of the one before that
//     in one block of code gave nothing (580 us for 584 then).
//   - d <= 64: vector issue.  64 keys of 32 rows at d = 64 are 98 vector
//     instructions, 32 exponentials and 16 products: 1014 clocks if nothing
//     waits, 1219 measured (17 prompts of up to 4000 tokens, 16 heads on 4, 220 us).
//   - few rows: the cache's bytes.  One token over each of 64 caches of up to 32,767,
//     32 heads on 8, d = 128: 203 us, 5.5 TB/s (a large copy moves 4.9, reads alone
//     5.3 to 6.5), and 6 us for the join.
#include <type_traits>

#include "full_common.h"

namespace kmip {
namespace {

struct FwdArgs {
    const char *q, *k, *v;
    uint16_t* out;
    float* lse;
    float *part_o, *part_ml;    // split: [job][ROWS][dv] sums, [job][ROWS][2] maximum (times c) and sum
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;   // bytes between tokens, heads
    int32_t H, Hk, rep, dv, split;
    bool causal, fold;
    float scale;
    int32_t first_job;          // of the launch, among the call's
    FullSeqs s;
};

// The reference of a row that has seen no key: below every score, and finite, so that no
// difference of two infinities is formed (these sources are built for code without NaN).
constexpr float kNoKey = -3.402823466e38f;

// A wave's running state: 32 columns of rows, two lanes a column.
template <typename T, int DK, int DV>
struct FwdWave {
    static constexpr int kT = kPieces<DV>;
    s16x8 q[DK / 16];
    f32x16 o[kT];
    float m, l;     // reference of the weights, sum of this lane's
    int32_t lim;    // keys this row sees

    // NB blocks of 32 keys from key0 on; keys and values at distance `at` from the operands' addresses.
    template <int NB, typename In, typename At>
    __device__ __forceinline__ void step(const In& in, At at, int32_t key0, int32_t lim_first, float c, int lane) {
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            clear(s[b]);
#pragma unroll
            for (int t = 0; t < DK / 16; ++t) s[b] = T::mfma(in.x_rows(t, at + b * 64 * DK), q[t], s[b]);
        }
        // the wave in its exponentials goes first, the other's products run beside them (16 heads, 8192
        // tokens, d = 64, causal 170 -> 163 us; at wider heads the products are the longer part)
        constexpr bool kFirst = DK + DV <= 128;
        if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
        if (key0 + 32 * NB > lim_first) {
            const int32_t left = lim - key0 - 4 * (lane >> 5);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * b + (r & 3) + 8 * (r >> 2) >= left) s[b][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
        const float2 tops = both_halves(top);
        top = fmaxf(tops.x, tops.y);
        // The reference follows the maximum only where a weight would pass 2^8: bfloat16
        // weights keep their relative precision at any reference; float16 ones are 2^6
        // times as large (T::kUp), so that small ones have their bits too.
        // (2^-120: a first key is always that far above kNoKey)
        if (__any((top - m) * fmaxf(c, 0x1p-120f) > 8.0f)) {
            const float to = fmaxf(top, m);
            // (no key seen yet: the factor is that of a sum of nothing)
            const float f = m == kNoKey ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            l *= f;
#pragma unroll
            for (int t = 0; t < kT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= f;
        }
        const float mc = m == kNoKey ? 0.0f : m * c - T::kUp;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -mc));
                sum += s[b][r];
            }
            l += sum;
            if (kFirst && b == NB - 1) __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // rounded to the inputs' type, the operand of the product: half a step of each weight
                const s16x8 p = round8<T>(s[b], i);
#pragma unroll
                for (int t = 0; t < kT; ++t) o[t] = T::mfma(in.y_columns(t, at + (32 * b + 16 * i) * 2 * DV), p, o[t]);
            }
        }
    }
};

template <typename T, int DK, int DV, int ROWS, int HALVES>
__global__ __launch_bounds__(256 * HALVES, ROWS == 128 ? 2 : 1) void full_fwd_kernel(const FwdArgs a) {
    using B = Buffers<DK, DV, ROWS == 128 ? (DK + DV == 32 ? 128 : 64) : 32>;   // [buffer][K, V]
    constexpr int kTile = B::kTile, kWaves = 4, kOwn = ROWS == 128 ? HALVES : kWaves;   // buffer sets
    constexpr int kBufs = 2, kT = kPieces<DV>;
    __shared__ __attribute__((aligned(1024))) char sh[kOwn * kBufs * B::kBytes];
    static_assert(ROWS == 128 || sizeof(sh) >= 32 * DV * 4 * kWaves, "room for the join");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3);
    const int half = HALVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
    const RowJob j = row_job<ROWS>(a.s, a.Hk, a.rep, a.causal, a.fold, a.split, blockIdx.x, lane);
    const int32_t nrows = j.q_len * a.rep;
    const int32_t row0 = j.tile * ROWS + (ROWS == 128 ? 32 * wave : 0);
    const int32_t off = j.k_len - j.q_len;
    auto sees = [&](int32_t row) {   // keys row sees (ascending in row)
        if (!a.causal) return j.k_len;
        return max(0, min(row, nrows - 1) / a.rep + off + 1);
    };
    const int32_t row = row0 + (lane & 31);
    const bool live = row < nrows;
    const int32_t token = min(row, nrows - 1) / a.rep, head = j.kv_head * a.rep + min(row, nrows - 1) % a.rep;

    FwdWave<T, DK, DV> w;
    load_columns<DK>(w.q, a.q + (j.q_lo + (int64_t)token) * a.q_row + head * a.q_head, lane);
#pragma unroll
    for (int t = 0; t < kT; ++t) clear(w.o[t]);
    w.m = kNoKey;
    w.l = 0.0f;
    w.lim = sees(row);

    const int32_t lo = a.split > 0 ? j.run * a.split : 0;
    int32_t hi = sees(j.tile * ROWS + ROWS - 1);
    if (a.split > 0) hi = full_run_end(lo, hi, a.split);
    const int32_t lim_first = sees(row0), lim_last = row0 < nrows ? sees(row0 + 31) : 0;
    const float c = a.scale * kLog2e;
    const char* kp = a.k + (int64_t)j.k_lo * a.k_row + j.kv_head * a.k_head;
    const char* vp = a.v + (int64_t)j.k_lo * a.v_row + j.kv_head * a.v_head;
    const uint32_t base = lds_addr(sh) + (ROWS == 128 ? half : wave) * kBufs * B::kBytes;
    PairLoad<B, DK, DV, ROWS == 128> load;
    load.init(lane, wave, a.k_row, a.v_row);
    auto fetch = [&](int32_t key, int buf) {
        load.issue(base + buf * B::kBytes, kp + (int64_t)key * a.k_row, vp + (int64_t)key * a.v_row, j.k_len - key);
    };
    PairOperands<B, DK, DV> in;
    in.init(base, lane);
    if constexpr (ROWS == 128) {
        // each half takes its part of the tiles; the first one's is as long or one longer
        const int32_t n = lo < hi ? (hi - lo - 1) / kTile + 1 : 0, most = (n + HALVES - 1) / HALVES;
        const int32_t first = lo + half * most * kTile, mine = half == 0 ? most : n - most;
        stream_tiles(
            most, mine, [&](int32_t i, int buf) { fetch(first + i * kTile, buf); },
            [&](int32_t i, auto buf) {
                const int32_t key = first + i * kTile;
                if (key < lim_last)
                    w.template step<kTile / 32>(in, Constant<decltype(buf)::value * B::kBytes>(), key, lim_first, c, lane);
            });
    } else {
        // blocks lo + 32 (wave + 4 i)
        const int32_t mine = lo + 32 * wave, n = mine < hi ? (hi - mine + 32 * kWaves - 1) / (32 * kWaves) : 0;
        stream_blocks<kBufs, B::kOwnLoads>(
            n, [&](int32_t i, int stage) { fetch(mine + 32 * kWaves * i, stage); },
            [&](int32_t i, int stage) {
                w.template step<1>(in, (uint32_t)stage * B::kBytes, mine + 32 * kWaves * i, lim_first, c, lane);
            });
    }

    const float2 ls = both_halves(w.l);
    float l = ls.x + ls.y, mc = w.m == kNoKey ? -INFINITY : w.m * c - T::kUp;
    const int h = lane >> 5;
    if constexpr (HALVES > 1) {
        // the second half's sums to LDS, a piece of 32 columns at a time [wave][piece][4 registers][lane], then added
        __shared__ float sm[kWaves][64], sl[kWaves][64];
        static_assert(sizeof(sh) >= kWaves * kT * 4096, "room for the sums");
        f32x4* const so = reinterpret_cast<f32x4*>(sh) + wave * kT * 256 + lane;
        wait_and_sync();
        if (half == 1) {
            sm[wave][lane] = mc;
            sl[wave][lane] = l;
#pragma unroll
            for (int t = 0; t < kT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    so[t * 256 + r * 64] = f32x4{w.o[t][4 * r], w.o[t][4 * r + 1], w.o[t][4 * r + 2], w.o[t][4 * r + 3]};
        }
        wait_and_sync();
        if (half == 1) return;
        const float mo = sm[wave][lane], top = fmaxf(mc, mo);
        const float f = mc == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mc - top);
        const float g = mo == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mo - top);
        l = l * f + sl[wave][lane] * g;
        mc = top;
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 x = so[t * 256 + r * 16];
#pragma unroll
                for (int e = 0; e < 4; ++e) w.o[t][r + e] = w.o[t][r + e] * f + x[e] * g;
            }
    }
    const int64_t job = (int64_t)a.first_job + blockIdx.x;
    if constexpr (ROWS == 128) {
        if (!live) return;
        if (j.runs > 1) {
            float* po = a.part_o + (job * ROWS + (row - j.tile * ROWS)) * DV;
#pragma unroll
            for (int t = 0; t < kT; ++t) store_sums<DV>(po, w.o[t], t, lane);
            if (h == 0) {
                float* ml = a.part_ml + (job * ROWS + (row - j.tile * ROWS)) * 2;
                ml[0] = mc;
                ml[1] = l;
            }
            return;
        }
        const int64_t at = (j.q_lo + (int64_t)token) * a.H + head;
        const float f = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int t = 0; t < kT; ++t) store_piece<T, DV>(a.out + at * DV, w.o[t], t, f, lane);
        if (h == 0) a.lse[at] = l > 0.0f ? (mc + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    } else {
        // The four waves' sums of the same rows: to a common reference, added in
        // LDS [wave][row][DV], stored by columns.
        float* const so = reinterpret_cast<float*>(sh);
        __shared__ float sm[kWaves][32], sl[kWaves][32];
        if (h == 0) {
            sm[wave][lane] = mc;
            sl[wave][lane] = l;
        }
        wait_and_sync();
        const int rw = lane & 31;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) top = fmaxf(top, sm[i][rw]);
        const float f = mc == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mc - top);
#pragma unroll
        for (int t = 0; t < kT; ++t) put_piece<DV>(so + wave * 32 * DV, w.o[t], t, f, lane);
        wait_and_sync();
        for (int i = threadIdx.x; i < 32 * (DV / 4); i += 256) {
            const int rr = i / (DV / 4), g = i % (DV / 4);
            const int32_t rowi = j.tile * ROWS + rr;
            if (rowi >= nrows) continue;
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
            float mm = -INFINITY, ll = 0.0f;
#pragma unroll
            for (int u = 0; u < kWaves; ++u) {
                x += get_piece<DV>(so + u * 32 * DV, rr, g);
                mm = fmaxf(mm, sm[u][rr]);
            }
#pragma unroll
            for (int u = 0; u < kWaves; ++u)
                if (sl[u][rr] > 0.0f) ll += sl[u][rr] * __builtin_amdgcn_exp2f(sm[u][rr] - mm);
            if (j.runs > 1) {
                *reinterpret_cast<f32x4*>(a.part_o + (job * ROWS + rr) * DV + 4 * g) = x;
                if (g == 0) {
                    float* ml = a.part_ml + (job * ROWS + rr) * 2;
                    ml[0] = mm;
                    ml[1] = ll;
                }
                continue;
            }
            const int64_t at = (j.q_lo + (int64_t)(rowi / a.rep)) * a.H + j.kv_head * a.rep + rowi % a.rep;
            const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
            *reinterpret_cast<s16x4*>(a.out + at * DV + 4 * g) = round4<T>(x, inv);
            if (g == 0) a.lse[at] = ll > 0.0f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
        }
    }
}

struct JoinArgs {
    FwdArgs f;                  // f.s: the sequences with several runs, a job for each tile and key head
    int32_t part0[kFullSeqs];   // their first jobs' places among the sums
    int32_t rows;               // of a tile
    int32_t lanes;              // threads that share a row's four columns, a power of two
};

// Joins the runs of row tiles (5 to 6 us, latency).  A thread takes four columns of a row and every
// lanes-th run in one pass (reference, sum of weights, sums), then the threads
// of a row are joined in their order.
template <typename T>
__global__ __launch_bounds__(256) void full_join_kernel(const JoinArgs b) {
    const FwdArgs& a = b.f;
    __shared__ f32x4 part[256];
    __shared__ float sm[256], sl[256];
    const JobSeq s = seq_of_job(a.s, blockIdx.x, threadIdx.x & 63);
    const int32_t q_lo = s.q_lo, nrows = s.q_len * a.rep, runs = full_runs(s.k_len, a.split);
    const int32_t tiles = (nrows - 1) / b.rows + 1;
    const int32_t kv_head = (blockIdx.x - s.job0) % a.Hk, place = (blockIdx.x - s.job0) / a.Hk;
    const int32_t tile = full_tile(place, tiles, a.causal, false, a.fold);
    const int groups = a.dv / 4, at_once = 256 / groups / b.lanes;
    const int g = threadIdx.x % groups, t = threadIdx.x / groups % b.lanes;
    // run 0; run r is r * Hk jobs on
    const int64_t job = (int64_t)a.first_job + b.part0[s.index] + (int64_t)place * runs * a.Hk + kv_head;
    const int64_t step = (int64_t)a.Hk * b.rows;
    const int32_t left = min(b.rows, nrows - tile * b.rows);
    for (int32_t r0 = blockIdx.y * at_once; r0 < left; r0 += gridDim.y * at_once) {
        const int32_t rr = r0 + threadIdx.x / groups / b.lanes, row = tile * b.rows + rr;
        const bool live = rr < left;
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + job * b.rows + rr;
        const float* po = a.part_o + (job * b.rows + rr) * a.dv + 4 * g;
        float top = -INFINITY, sum = 0.0f;
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        auto add = [&](float m, float l, const f32x4& y) {   // m: -inf for a run without a key that the row sees
            const float to = fmaxf(fmaxf(top, m), -1e30f);
            const float f = __builtin_amdgcn_exp2f(top - to), h = __builtin_amdgcn_exp2f(m - to);
            top = fmaxf(top, m);
            sum = sum * f + l * h;
            x = x * f + y * h;
        };
        auto stream = [&](auto ahead) {   // that many runs' loads go out together
            constexpr int kAhead = decltype(ahead)::value;
            for (int32_t r0 = t; r0 < runs; r0 += kAhead * b.lanes) {
                float2 m[kAhead];
                f32x4 y[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int64_t r = min(r0 + u * b.lanes, runs - 1);
                    m[u] = ml[r * step];
                    y[u] = *reinterpret_cast<const f32x4*>(po + r * step * a.dv);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) add(r0 + u * b.lanes < runs ? m[u].x : -INFINITY, m[u].y, y[u]);
            }
        };
        if (live) {
            if (runs > 2 * b.lanes)
                stream(std::integral_constant<int, 8>());
            else
                stream(std::integral_constant<int, 1>());
        }
        part[threadIdx.x] = x;
        sm[threadIdx.x] = top;
        sl[threadIdx.x] = sum;
        __syncthreads();
        if (live && t == 0) {
            for (int u = 1; u < b.lanes; ++u) {
                const int i = threadIdx.x + u * groups;
                add(sm[i], sl[i], part[i]);
            }
            const int64_t at = (q_lo + (int64_t)(row / a.rep)) * a.H + kv_head * a.rep + row % a.rep;
            *reinterpret_cast<s16x4*>(a.out + at * a.dv + 4 * g) = round4<T>(x, sum > 0.0f ? 1.0f / sum : 0.0f);
            if (g == 0) a.lse[at] = sum > 0.0f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
        }
        __syncthreads();
    }
}

template <typename T, int DK, int DV>
hipError_t launch_fwd(const FullCall& f, const FullPlan& p, float* part_o, float* part_ml, hipStream_t stream) {
    FwdArgs a{};
    a.q = reinterpret_cast<const char*>(f.q);
    a.k = reinterpret_cast<const char*>(f.k);
    a.v = reinterpret_cast<const char*>(f.v);
    a.out = reinterpret_cast<uint16_t*>(f.out);
    a.lse = f.lse;
    a.part_o = part_o;
    a.part_ml = part_ml;
    a.q_row = 2 * f.q_row, a.q_head = 2 * f.q_head;
    a.k_row = 2 * f.k_row, a.k_head = 2 * f.k_head;
    a.v_row = 2 * f.v_row, a.v_head = 2 * f.v_head;
    a.H = f.H, a.Hk = f.Hk, a.rep = f.H / f.Hk, a.dv = f.dv, a.causal = f.causal != 0;
    a.split = p.split;
    a.scale = f.scale;
    for (const FullLaunch& l : p.launches) {
        a.s = l.seqs;
        a.first_job = l.first_job;
        a.fold = l.fold;
        if (p.rows == 128 && p.halves == 2)
            hipLaunchKernelGGL((full_fwd_kernel<T, DK, DV, 128, 2>), dim3(l.jobs), dim3(512), 0, stream, a);
        else if (p.rows == 128)
            hipLaunchKernelGGL((full_fwd_kernel<T, DK, DV, 128, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((full_fwd_kernel<T, DK, DV, 32, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (l.tile_jobs > 0) {
            JoinArgs b{};
            b.f = a;
            b.f.s = l.tiles;
            for (int i = 0; i < kFullSeqs; ++i) b.part0[i] = l.part0[i];
            const int groups = f.dv / 4;
            b.rows = p.rows;
            b.lanes = 1;
            while (2 * b.lanes <= l.runs && 2 * b.lanes * groups <= 256) b.lanes *= 2;
            // a workgroup takes this many rows at a time; more than eight workgroups a CU do several rounds
            const int at_once = 256 / groups / b.lanes, rounds = (l.tile_rows + at_once - 1) / at_once;
            const int ny = rounds < 2048 / l.tile_jobs + 1 ? rounds : 2048 / l.tile_jobs + 1;
            hipLaunchKernelGGL((full_join_kernel<T>), dim3(l.tile_jobs, ny), dim3(256), 0, stream, b);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_full_fwd(const FullCall& f, const FullPlan& p, float* part_o, float* part_ml, hipStream_t stream) {
#define KMIP_FULL_CASE(DK, DV) \
    if (f.d == DK && f.dv == DV) \
        return f.fp16 ? launch_fwd<Fp16, DK, DV>(f, p, part_o, part_ml, stream) : launch_fwd<Bf16, DK, DV>(f, p, part_o, part_ml, stream);
#define KMIP_FULL_FWD(DK) KMIP_FULL_CASE(DK, 16) KMIP_FULL_CASE(DK, 32) KMIP_FULL_CASE(DK, 64) KMIP_FULL_CASE(DK, 128)
    KMIP_FULL_FWD(16)
    KMIP_FULL_FWD(32)
    KMIP_FULL_FWD(64)
    KMIP_FULL_FWD(128)
#undef KMIP_FULL_FWD
#undef KMIP_FULL_CASE
    return hipErrorInvalidValue;
}

}  // namespace kmip
