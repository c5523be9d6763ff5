// Shared by the kernels of full softmax attention (full_fwd.hip, full_bwd.hip).
//
// All products run as 32 x 32 x 16 matrix instructions on 16-bit operands
// with float32 sums.  The side a wave keeps (32 rows, "columns" below) is the
// right operand, held in registers; the other side streams through LDS in
// tiles of rows and is the left operand, so that a score tile comes out
// transposed: lane l holds column l % 32 and, in register r, the streamed row
// (r & 3) + 8 (r >> 2) + 4 (l / 32).  Two properties carry the kernels:
//   - statistics of a column (maximum, sum, log-sum) are the lane's own and
//     its partner's (l ^ 32);
//   - eight consecutive registers, rounded to 16 bits, are the right operand
//     of the next product over the streamed rows, with the contraction in
//     the order {0-3, 8-11} (lanes 0-31), {4-7, 12-15} (lanes 32-63) of each 16
//     rows; the left operand is read from LDS transposed (ds_read_b64_tr_b16:
//     four rows of one column a lane) in the same order.  No value changes
//     lanes between the two products.
//
// LDS tiles are rows of D 16-bit values; the 16-byte chunk c of row r lies at
// place c ^ swz(r), which spreads both kinds of reads over the 64 banks
// (measured: 205 bytes a clock and CU for the plain reads, 256 for the
// transposed ones, of 256; 16 without the permutation).  Tiles are written by
// loads that go from memory to LDS directly, 1 KB an instruction; the
// permutation is applied to the address each lane reads from.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kmip_device.h"
#include "full_plan.h"

namespace kmip {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
#define KMIP_LDS __attribute__((address_space(3)))
#define KMIP_GLOBAL __attribute__((address_space(1)))

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The two types.  kUp: the forward's weights are 2^kUp times as large (2^14 at
// most in float16, twice that where scores reach 2^24 and the reference is rounded; its values below 2^-14 lose bits).
// kUpBack: the backward's for the product with dout, as a factor.  They are at most 1, or 2^5 where scores reach
// 2^24 and lse is off by that: 2^9 keeps the bits of weights from 2^-23 on (without it from 2^-14 on, which 16,384 alike
// keys have), for a multiplication a weight: training in float16, 24 texts 135 -> 136 us, 16 heads of 4096 tokens
// at d = 64 211 -> 215.
struct Bf16 {
    static constexpr float kUp = 0.0f, kUpBack = 1.0f;
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                       0, 0);
    }
    static __device__ __forceinline__ short round(float x) { return __builtin_bit_cast(short, (__bf16)x); }
    static __device__ __forceinline__ float widen(short x) { return __uint_as_float((uint32_t)(uint16_t)x << 16); }
};

struct Fp16 {
    static constexpr float kUp = 6.0f, kUpBack = 512.0f;
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                      0);
    }
    static __device__ __forceinline__ short round(float x) { return __builtin_bit_cast(short, (_Float16)x); }
    static __device__ __forceinline__ float widen(short x) { return (float)__builtin_bit_cast(_Float16, x); }
};

// Place permutation of a row's 16-byte chunks.  Transposed reads touch 64
// bytes of eight rows, plain ones 16 bytes of 32: the chunk's bits above 2
// (64-byte places) follow the row's lowest bits, as far as the row length
// leaves rows in the same 256 bytes, its low two bits the next ones.
template <int D>
__device__ __forceinline__ int swz(int r) {
    if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    if constexpr (D == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    if constexpr (D == 32) return (r >> 2) & 3;
    return (r >> 3) & 1;
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
    return (uint32_t)(uintptr_t)(const KMIP_LDS char*)p;
}

// This lane's LDS addresses of the left operands in a tile at `tile`; a tile
// elsewhere is at a distance, which becomes the instructions' offset where it is
// known when compiling.
//   row[t]: rows 0 .. 31, dimensions 16 t .. 16 t + 15; rows R .. R + 31 (R a multiple of 32) at + R * 2D;
//   tr[i][t]: transposed, the tile's columns 32 t .. 32 t + 31 as operand rows and tile rows 0 .. 15
//   as contraction, first and second half; rows R .. R + 15 (R a multiple of 16) at + R * 2D.
template <int D>
struct Operands {
    static constexpr int kT = D < 32 ? 1 : D / 32;
    uint32_t row[D / 16], tr[2][kT];

    __device__ __forceinline__ void init(uint32_t tile, int lane) {
        {
            const int r = lane & 31, c = lane >> 5;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) row[t] = tile + r * 2 * D + (((c + 2 * t) ^ swz<D>(r)) << 4);
        }
        const int l = lane & 15, g = (lane >> 4) & 1, h = lane >> 5;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 8 * i + 4 * h + (l >> 2);
#pragma unroll
            for (int t = 0; t < kT; ++t) {
                const int c = 4 * t + (D >= 32 ? 2 * g : 0) + ((l >> 1) & 1);
                tr[i][t] = tile + r * 2 * D + ((c ^ swz<D>(r)) << 4) + (l & 1) * 8;
            }
        }
    }
    __device__ __forceinline__ s16x8 rows(int t, uint32_t at) const {
        return *(const KMIP_LDS s16x8*)(uintptr_t)(row[t] + at);
    }
    __device__ __forceinline__ s16x8 columns(int t, uint32_t at) const {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KMIP_LDS s16x4*)(uintptr_t)(tr[0][t] + at));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KMIP_LDS s16x4*)(uintptr_t)(tr[1][t] + at));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// A number known when compiling, for the buffers that alternate.
template <uint32_t N>
struct Constant {
    __device__ constexpr operator uint32_t() const { return N; }
};

// x of this lane and of its partner lane ^ 32, as (lower lane's, upper lane's).
__device__ __forceinline__ float2 both_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// x, uniform over the wave, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}

// Memory to LDS, 16 bytes a lane: lane l's 16 bytes at base + off go to
// lds + 16 l (base and lds uniform; the LDS address travels in m0, which is left
// as it was).  No register is written, and the kernels wait by count (wait_loads
// and what follows): with the compiler's own form of these loads, it waits for
// all of them before any transposed read of LDS, which holds up every tile's
// second product until the next tile has arrived.  (Waits of the instructions:
// one between m0 and the load, five between a vector instruction that wrote base
// and the load.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char* base, uint32_t off) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "s"(uniform(lds)), "v"(off), "s"(uniform((uint64_t)base))
                 : "memory");
}

// The same with 4 bytes a lane, each from an address of its own.
__device__ __forceinline__ void load_word_to_lds(uint32_t lds, const float* p) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "s"(uniform(lds)), "v"(p)
                 : "memory");
}

// All but the last n loads of this wave have ended.
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// All loads of this wave have ended, those to registers among them, in a form
// that the compiler knows (it would wait for them where they are used, in the
// loop, and there for all loads to LDS too).
__device__ __forceinline__ void wait_all_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// All LDS accesses of this wave have ended.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Every load to LDS and LDS access of this wave has ended, and then of the
// workgroup's other waves.
__device__ __forceinline__ void wait_and_sync() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Loads tiles of rows of a strided tensor into LDS.  A round of PARTS
// instructions (one from each of PARTS waves) writes PARTS * 512 / D rows.
template <int D, int PARTS>
struct TileLoad {
    static constexpr int kPer = 512 / D * PARTS;            // rows of a round
    static constexpr int kVar = kPer < 16 ? 16 / kPer : 1;  // rounds after which the permutation repeats
    uint32_t off[kVar];   // this lane's bytes in a round's rows
    uint32_t row;         // its row among them
    uint32_t stride;      // bytes between rows

    __device__ __forceinline__ void init(int lane, int part, uint32_t row_stride) {
        row = part * (512 / D) + lane / (D / 8);
        stride = row_stride;
#pragma unroll
        for (int v = 0; v < kVar; ++v) {
            const uint32_t c = (uint32_t)(lane & (D / 8 - 1)) ^ (uint32_t)swz<D>((int)row + v * kPer);
            off[v] = row * stride + 16 * c;
        }
    }
    // ROWS rows from the one at `base` on; those from `left` on are replaced by
    // row left - 1 (left >= 1), so that no address lies behind the last row.
    template <int ROWS>
    __device__ __forceinline__ void issue(uint32_t lds, const char* base, int part, int32_t left) const {
        static_assert(ROWS % kPer == 0, "whole rounds");
        constexpr int kRounds = ROWS / kPer;
        lds += part * 1024;
        if (left >= ROWS) {
#pragma unroll
            for (int i = 0; i < kRounds; ++i)
                load_to_lds(lds + i * PARTS * 1024, base + (uint64_t)(uint32_t)(i * kPer) * stride, off[i % kVar]);
        } else {
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                const uint32_t back = row - (uint32_t)min((int32_t)row + i * kPer, left - 1);
                load_to_lds(lds + i * PARTS * 1024, base, off[i % kVar] - back * stride);
            }
        }
    }
};

// ---- jobs (full_plan.h) ----

// The sequence a job belongs to (uniform over the workgroup).
struct JobSeq {
    int32_t index, q_lo, q_len, job0, k_lo, k_len, k_slot;
};

// Lanes take entries; what they hold of the found one is read from its lane, so
// that the search and the entry cost one trip to the arguments and not two.
__device__ __forceinline__ JobSeq seq_of_job(const FullSeqs& s, int32_t job, int lane) {
    if (s.count == 1) return JobSeq{0, s.q_lo(0), s.q_len(0), s.job0(0), s.k_lo(0), s.k_len(0), s.k_slot(0)};
    JobSeq j{};
    int n = 0;
    for (int i = 0; i < s.count; i += 64) {
        const int e = i + lane < s.count ? i + lane : s.count - 1;
        const int32_t q_lo = s.q_lo(e), q_len = s.q_len(e), job0 = s.job0(e);
        const int32_t k_lo = s.k_lo(e), k_len = s.k_len(e), k_slot = s.k_slot(e);
        const int here = __popcll(__ballot(i + lane < s.count && job0 <= job));
        if (here == 0) break;
        n = i + here;
        const int l = here - 1;
        j = JobSeq{n - 1,
                   __builtin_amdgcn_readlane(q_lo, l),
                   __builtin_amdgcn_readlane(q_len, l),
                   __builtin_amdgcn_readlane(job0, l),
                   __builtin_amdgcn_readlane(k_lo, l),
                   __builtin_amdgcn_readlane(k_len, l),
                   __builtin_amdgcn_readlane(k_slot, l)};
        if (here < 64) break;
    }
    return j;
}

// A job of a row tile: ROWS rows of one key head's list, and the run of keys
// it takes (all of them where split is 0).
struct RowJob {
    int32_t q_lo, q_len, k_lo, k_len, kv_head, tile, run, runs;
};

template <int ROWS>
__device__ __forceinline__ RowJob row_job(const FullSeqs& seqs, int32_t Hk, int32_t rep, bool causal, bool fold,
                                          int32_t split, int32_t job, int lane) {
    const JobSeq s = seq_of_job(seqs, job, lane);
    RowJob j;
    j.q_lo = s.q_lo, j.q_len = s.q_len, j.k_lo = s.k_lo, j.k_len = s.k_len;
    j.runs = full_runs(j.k_len, split);
    const int32_t tiles = (int32_t)(((int64_t)j.q_len * rep + ROWS - 1) / ROWS);
    // key heads first: with 8 of them (or a divisor) workgroups of one XCD,
    // which come round robin, share a head's keys in its L2
    int32_t rest = job - s.job0;
    j.kv_head = rest % Hk;
    rest /= Hk;
    j.run = 0;
    if (j.runs > 1) {
        j.run = rest % j.runs;
        rest /= j.runs;
    }
    j.tile = full_tile(rest, tiles, causal, false, fold);
    return j;
}

// The right operand of 32 columns from a strided tensor: this lane's row
// (16-byte aligned).
template <int D>
__device__ __forceinline__ void load_columns(s16x8 (&x)[D / 16], const char* row, int lane) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t) x[t] = *reinterpret_cast<const s16x8*>(row + 2 * (16 * t + 8 * (lane >> 5)));
}

__device__ __forceinline__ void clear(f32x16& x) {
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.0f;
}

// Registers 8 i .. 8 i + 7, rounded: the right operand for 16 streamed rows.
template <typename T>
__device__ __forceinline__ s16x8 round8(const f32x16& x, int i) {
    s16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = T::round(x[8 * i + e]);
    return p;
}

// Stores column tile t of a transposed result (this lane's row at `row`),
// times f.
template <typename T, int D>
__device__ __forceinline__ void store_piece(uint16_t* row, const f32x16& x, int t, float f, int lane) {
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        const int col = 32 * t + 2 * r + 4 * (lane >> 5);
        if (col < D) {
            s16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = T::round(x[r + e] * f);
            *reinterpret_cast<s16x4*>(row + col) = y;
        }
    }
}

// The same in float32, unrounded (a run's sums).
template <int D>
__device__ __forceinline__ void store_sums(float* row, const f32x16& x, int t, int lane) {
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        const int col = 32 * t + 2 * r + 4 * (lane >> 5);
        if (col < D) *reinterpret_cast<f32x4*>(row + col) = f32x4{x[r], x[r + 1], x[r + 2], x[r + 3]};
    }
}

template <typename T>
__device__ __forceinline__ s16x4 round4(const f32x4& x, float f) {
    s16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = T::round(x[e] * f);
    return y;
}

// Widths a kernel is built for: DK of queries and keys, DV of values.  How
// the streamed rows lie in LDS: buffers of kTile rows of both tensors.
template <int DK, int DV, int TILE>
struct Buffers {
    // the first tensor's, both tensors' bytes
    static constexpr int kTile = TILE, kFirst = TILE * 2 * DK, kBytes = kFirst + TILE * 2 * DV;
    // waves that load a tensor: all four, or two where its tile has only two loads
    static constexpr int kPartsK = kFirst >= 4096 ? 4 : 2, kPartsV = TILE * 2 * DV >= 4096 ? 4 : 2;
    // the same for a wave with buffers of its own: its loads
    static constexpr int kOwnLoads = TILE / TileLoad<DK, 1>::kPer + TILE / TileLoad<DV, 1>::kPer;
};

// 32-wide pieces of a width.
template <int D>
constexpr int kPieces = D < 32 ? 1 : D / 32;

// The left operands of both tensors of a buffer; tensors of one width share
// their addresses, a constant distance apart.
template <typename B, int DK, int DV>
struct PairOperands {
    Operands<DK> x;
    Operands<DV> y;

    __device__ __forceinline__ void init(uint32_t buffer, int lane) {
        x.init(buffer, lane);
        if constexpr (DK != DV) y.init(buffer + B::kFirst, lane);
    }
    __device__ __forceinline__ s16x8 x_rows(int t, uint32_t at) const { return x.rows(t, at); }
    __device__ __forceinline__ s16x8 x_columns(int t, uint32_t at) const { return x.columns(t, at); }
    __device__ __forceinline__ s16x8 y_rows(int t, uint32_t at) const {
        if constexpr (DK == DV) return x.rows(t, at + B::kFirst);
        return y.rows(t, at);
    }
    __device__ __forceinline__ s16x8 y_columns(int t, uint32_t at) const {
        if constexpr (DK == DV) return x.columns(t, at + B::kFirst);
        return y.columns(t, at);
    }
};

// Loads a tile of both tensors: `shared`, each of four waves a part of it; else one wave all of it.
template <typename B, int DK, int DV, bool SHARED>
struct PairLoad {
    TileLoad<DK, SHARED ? B::kPartsK : 1> x;
    TileLoad<DV, SHARED ? B::kPartsV : 1> y;
    int px, py;   // this wave's parts, negative: none

    __device__ __forceinline__ void init(int lane, int wave, int64_t x_row, int64_t y_row) {
        px = SHARED ? (wave < B::kPartsK ? wave : -1) : 0;
        py = SHARED ? wave - (4 - B::kPartsV) : 0;
        x.init(lane, px < 0 ? 0 : px, (uint32_t)x_row);
        y.init(lane, py < 0 ? 0 : py, (uint32_t)y_row);
    }
    __device__ __forceinline__ void issue(uint32_t lds, const char* xp, const char* yp, int32_t left) const {
        if (!SHARED || B::kPartsK == 4 || px >= 0) x.template issue<B::kTile>(lds, xp, px, left);
        if (!SHARED || B::kPartsV == 4 || py >= 0) y.template issue<B::kTile>(lds + B::kFirst, yp, py, left);
    }
};

// A group of waves' stream of `mine` tiles through two buffers, in step with another group's of at most `most`:
// `fetch(i, buf)` issues this wave's loads of tile i, `use(i, buf)` computes on it.  One barrier a tile.  (A third
// buffer and loads two tiles ahead changed nothing: 64 texts of up to 1000 tokens, d = 64 197 and 199 us.)
template <typename Fetch, typename Use>
__device__ __forceinline__ void stream_tiles(int32_t most, int32_t mine, const Fetch& fetch, const Use& use) {
    auto stage = [&](int32_t i, auto buf) {
        wait_and_sync();
        if (i + 1 < mine) fetch(i + 1, buf ^ 1);
        if (i < mine) use(i, buf);
    };
    if (mine > 0) fetch(0, 0);
    wait_all_loads();
    for (int32_t i = 0; i < most; i += 2) {
        stage(i, std::integral_constant<int, 0>());
        if (i + 1 < most) stage(i + 1, std::integral_constant<int, 1>());
    }
}

// A wave's own stream: `fetch(i, stage)` issues block i's loads (LOADS
// instructions), `use(i, stage)` computes on it, for i < n.  Two stages: more
// take the LDS of other workgroups (one token over 8 caches of 8000, d = 64 31 us
// with two, 37 with three, 39 with four; d = 16 30, 30 and 31).
template <int STAGES, int LOADS, typename Fetch, typename Use>
__device__ __forceinline__ void stream_blocks(int32_t n, const Fetch& fetch, const Use& use) {
    static_assert((STAGES - 1) * LOADS < 64, "counted by vmcnt");
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < n) fetch(i, i);
    wait_all_loads();
    for (int32_t i = 0, stage = 0; i < n; ++i, stage = stage + 1 == STAGES ? 0 : stage + 1) {
        if (i + STAGES - 1 < n) {
            wait_lds();   // the reads of the stage that is filled again
            fetch(i + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
            wait_loads<(STAGES - 1) * LOADS>();
        } else {
            wait_loads<0>();
        }
        use(i, stage);
    }
}

// A wave's transposed result of 32 rows to LDS at so, rows of D floats, their
// groups of four turned by the row (so that the rows meet different banks).
template <int D>
__device__ __forceinline__ void put_piece(float* so, const f32x16& x, int t, float f, int lane) {
    const int rw = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        const int g = 8 * t + (r >> 1) + (lane >> 5);
        if (4 * g < D)
            *reinterpret_cast<f32x4*>(so + rw * D + 4 * ((g ^ rw) & (D / 4 - 1))) =
                f32x4{x[r] * f, x[r + 1] * f, x[r + 2] * f, x[r + 3] * f};
    }
}

template <int D>
__device__ __forceinline__ f32x4 get_piece(const float* so, int row, int g) {
    return *reinterpret_cast<const f32x4*>(so + row * D + 4 * ((g ^ row) & (D / 4 - 1)));
}

// Adds the second half's sums of a tile to the first's through LDS (`sh`: 16 KB
// per piece of 32 columns), for the first half; false for the second.  All
// waves of the workgroup call it, when they are done with what sh holds.
template <int KT>
__device__ __forceinline__ bool add_half(f32x16 (&x)[KT], char* sh, int wave, int half, int lane) {
    f32x4* const so = reinterpret_cast<f32x4*>(sh) + wave * KT * 256 + lane;
    wait_and_sync();
    if (half == 1) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) so[t * 256 + r * 16] = f32x4{x[t][r], x[t][r + 1], x[t][r + 2], x[t][r + 3]};
    }
    wait_and_sync();
    if (half == 1) return false;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 y = so[t * 256 + r * 16];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][r + e] += y[e];
        }
    return true;
}

}  // namespace kmip
