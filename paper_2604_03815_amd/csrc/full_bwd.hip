// Full softmax attention over packed sequences: backward (gfx950).
//
// With p_ij = exp(scale s_ij - lse_i) recomputed from the forward's lse:
//   D_i = dout_i . out_i,  dp_ij = dout_i . v_j,  g_ij = p_ij (dp_ij - D_i),
//   dq_i = scale sum_j g_ij k_j,  dk_j = scale sum_i g_ij q_i,  dv_j = sum_i p_ij dout_i.
// Two kernels, so that every sum has one owner and no atomics are needed
// (results are the same from call to call):
//   full_dq_kernel   keeps rows (as the forward does: tokens and the heads that
//                    share a key head) and streams keys: s, dp, then dq; it also
//                    forms D of its rows and leaves it for the other kernel;
//   full_dkv_kernel  keeps keys and streams the tokens of one head after the
//                    other of its group: s, dp, then dv and dk.
// They form s and dp twice, seven products where one pass with atomics would
// need five; its sums would change from call to call.  Forms for many and for few
// kept rows as in the forward.
//
// p and g are rounded to the inputs' type for the products, half a step of each:
// gradients are then off by 0.0025 of their size (bf16, against 64 bits) instead
// of 0.0017, the rounding of the result itself.  A second product for what is
// rounded off would cost a third of the matrix instructions more.  In float16 p is
// 2^9 times as large (kUpBack) and dv divided by it at the end; g, whose size is
// the caller's choice of dout's, is not.
//
// Measured (MI355X): 8192 tokens, 8 heads on 2 key heads, d = 128, causal: dq 200 us,
// dk and dv 280, their runs' sums 14.  Bound as the forward is: matrix units
// busy 51% (dq) and 48% of the time, vector issue 33 and 27%, no LDS bank conflicts.
// 128 graphs of 100 to 450 nodes, 3 heads, d = 32: 25 us each, the chain of a job's tiles.
#include <type_traits>

#include "full_common.h"

namespace kmip {
namespace {

struct BwdArgs {
    const char *q, *k, *v, *dout;
    const uint16_t* out;
    const float* lse;
    float *lse2, *D;                          // [Nq, H]: lse log2 e (+inf for a row that sees no key), -D
    uint16_t *dq, *dk, *dv_out;
    float *part_dq, *part_dk, *part_dv;       // runs: [job][rows][width] sums
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, do_row, do_head;   // bytes between tokens, heads
    int32_t H, Hk, rep, split;
    bool causal, fold;
    float scale;
    int32_t first_job;
    FullSeqs s;
};

template <typename T, int DK, int DV, int ROWS, int HALVES>
__global__ __launch_bounds__(256 * HALVES, ROWS == 128 ? 2 : 1) void full_dq_kernel(const BwdArgs a) {
    using B = Buffers<DK, DV, ROWS == 128 ? (DK + DV == 32 ? 128 : 64) : 32>;   // [buffer][K, V]
    constexpr int kTile = B::kTile, kWaves = 4, kOwn = ROWS == 128 ? HALVES : kWaves;
    constexpr int kBufs = 2, kT = kPieces<DK>;
    __shared__ __attribute__((aligned(1024))) char sh[kOwn * kBufs * B::kBytes];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3);
    const int half = HALVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
    const RowJob j = row_job<ROWS>(a.s, a.Hk, a.rep, a.causal, a.fold, a.split, blockIdx.x, lane);
    const int32_t nrows = j.q_len * a.rep;
    const int32_t row0 = j.tile * ROWS + (ROWS == 128 ? 32 * wave : 0);
    const int32_t off = j.k_len - j.q_len;
    auto sees = [&](int32_t row) {
        if (!a.causal) return j.k_len;
        return max(0, min(row, nrows - 1) / a.rep + off + 1);
    };
    const int32_t row = row0 + (lane & 31);
    const bool live = row < nrows;
    const int32_t token = min(row, nrows - 1) / a.rep, head = j.kv_head * a.rep + min(row, nrows - 1) % a.rep;
    const int64_t at = (j.q_lo + (int64_t)token) * a.H + head;

    s16x8 q[DK / 16], g[DV / 16];
    load_columns<DK>(q, a.q + (j.q_lo + (int64_t)token) * a.q_row + head * a.q_head, lane);
    load_columns<DV>(g, a.dout + (j.q_lo + (int64_t)token) * a.do_row + head * a.do_head, lane);
    float di = 0.0f;
    {
        s16x8 o[DV / 16];
        load_columns<DV>(o, reinterpret_cast<const char*>(a.out + at * DV), lane);
#pragma unroll
        for (int t = 0; t < DV / 16; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) di = fmaf(T::widen(g[t][e]), T::widen(o[t][e]), di);
        const float2 ds = both_halves(di);
        di = ds.x + ds.y;
    }
    const float lse = a.lse[at];
    // a row that sees no key: every weight 0
    const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
    if (live && lane < 32 && (ROWS == 128 ? half == 0 : wave == 0) && j.run == 0) {
        a.lse2[at] = lse2;
        a.D[at] = -di;
    }
    const float c = a.scale * kLog2e;
    const int32_t lim = sees(row), lim_first = sees(row0), lim_last = row0 < nrows ? sees(row0 + 31) : 0;
    const int32_t lo = a.split > 0 ? j.run * a.split : 0;
    int32_t hi = sees(j.tile * ROWS + ROWS - 1);
    if (j.runs > 1) hi = full_run_end(lo, hi, a.split);

    const char* kp = a.k + (int64_t)j.k_lo * a.k_row + j.kv_head * a.k_head;
    const char* vp = a.v + (int64_t)j.k_lo * a.v_row + j.kv_head * a.v_head;
    const uint32_t base = lds_addr(sh) + (ROWS == 128 ? half : wave) * kBufs * B::kBytes;
    PairLoad<B, DK, DV, ROWS == 128> load;
    load.init(lane, wave, a.k_row, a.v_row);
    auto fetch = [&](int32_t key, int buf) {
        load.issue(base + buf * B::kBytes, kp + (int64_t)key * a.k_row, vp + (int64_t)key * a.v_row, j.k_len - key);
    };
    f32x16 acc[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) clear(acc[t]);
    PairOperands<B, DK, DV> in;
    in.init(base, lane);
    // dp - D comes out of the product, which starts at -D (where there are registers for it)
    constexpr bool kStart = DK + DV < 192;
    f32x16 start;
#pragma unroll
    for (int r = 0; r < 16; ++r) start[r] = kStart ? -di : 0.0f;
    auto compute = [&](int32_t key0, auto at) {
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            f32x16 s, dp;
            clear(s);
#pragma unroll
            for (int t = 0; t < DK / 16; ++t) s = T::mfma(in.x_rows(t, at + b * 64 * DK), q[t], s);
#pragma unroll
            for (int t = 0; t < DV / 16; ++t) dp = T::mfma(in.y_rows(t, at + b * 64 * DV), g[t], t == 0 ? start : dp);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * (kStart ? dp[r] : dp[r] - di);
            if (key0 + 32 * b + 32 > lim_first) {
                const int32_t left = lim - key0 - 32 * b - 4 * (lane >> 5);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((r & 3) + 8 * (r >> 2) >= left) s[r] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const s16x8 p = round8<T>(s, i);   // rounded to the inputs' type, the operand of the product
#pragma unroll
                for (int t = 0; t < kT; ++t) acc[t] = T::mfma(in.x_columns(t, at + (32 * b + 16 * i) * 2 * DK), p, acc[t]);
            }
        }
    };
    if constexpr (ROWS == 128) {
        const int32_t n = lo < hi ? (hi - lo - 1) / kTile + 1 : 0, most = (n + HALVES - 1) / HALVES;
        const int32_t first = lo + half * most * kTile, mine = half == 0 ? most : n - most;
        stream_tiles(
            most, mine, [&](int32_t i, int buf) { fetch(first + i * kTile, buf); },
            [&](int32_t i, auto buf) {
                const int32_t key = first + i * kTile;
                if (key < lim_last) compute(key, Constant<decltype(buf)::value * B::kBytes>());
            });
        static_assert(HALVES == 1 || sizeof(sh) >= kWaves * kT * 4096, "room for the sums");
        if constexpr (HALVES > 1)
            if (!add_half<kT>(acc, sh, wave, half, lane)) return;
        if (!live) return;
        const int64_t job = (int64_t)a.first_job + blockIdx.x;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            if (j.runs > 1)
                store_sums<DK>(a.part_dq + (job * ROWS + (row - j.tile * ROWS)) * DK, acc[t], t, lane);
            else
                store_piece<T, DK>(a.dq + at * DK, acc[t], t, a.scale, lane);
        }
    } else {
        // blocks lo + 32 (wave + 4 i)
        const int32_t mine = lo + 32 * wave, n = mine < hi ? (hi - mine + 32 * kWaves - 1) / (32 * kWaves) : 0;
        stream_blocks<kBufs, B::kOwnLoads>(
            n, [&](int32_t i, int stage) { fetch(mine + 32 * kWaves * i, stage); },
            [&](int32_t i, int stage) { compute(mine + 32 * kWaves * i, (uint32_t)stage * B::kBytes); });
        // the four waves' sums, in their order
        wait_and_sync();
        float* const so = reinterpret_cast<float*>(sh);
#pragma unroll
        for (int t = 0; t < kT; ++t) put_piece<DK>(so + wave * 32 * DK, acc[t], t, 1.0f, lane);
        wait_and_sync();
        for (int i = threadIdx.x; i < 32 * (DK / 4); i += 256) {
            const int rr = i / (DK / 4), gg = i % (DK / 4);
            const int32_t rowi = j.tile * ROWS + rr;
            if (rowi >= nrows) continue;
            f32x4 x = get_piece<DK>(so, rr, gg);
#pragma unroll
            for (int u = 1; u < kWaves; ++u) x += get_piece<DK>(so + u * 32 * DK, rr, gg);
            const int64_t to = (j.q_lo + (int64_t)(rowi / a.rep)) * a.H + j.kv_head * a.rep + rowi % a.rep;
            if (j.runs > 1)
                *reinterpret_cast<f32x4*>(a.part_dq + (((int64_t)a.first_job + blockIdx.x) * ROWS + rr) * DK + 4 * gg) = x;
            else
                *reinterpret_cast<s16x4*>(a.dq + to * DK + 4 * gg) = round4<T>(x, a.scale);
        }
    }
}

template <typename T, int DK, int DV, int KEYS, int HALVES>
__global__ __launch_bounds__(256 * HALVES, KEYS == 128 ? 2 : 1) void full_dkv_kernel(const BwdArgs a) {
    // tokens a buffer holds: fewer where the kept K and V are in LDS too, which they
    // are where registers would spill
    constexpr bool kHeld = KEYS == 32 || DK + DV < 256;
    using B = Buffers<DK, DV, KEYS == 128 ? (DK + DV == 32 ? 128 : kHeld ? 64 : 32) : 32>;   // [buffer][Q, dout]
    constexpr int kTile = B::kTile, kWaves = 4, kOwn = KEYS == 128 ? HALVES : kWaves;
    constexpr int kBufs = 2, kTK = kPieces<DK>, kTV = kPieces<DV>, kK = DK / 16, kV = DV / 16;
    __shared__ __attribute__((aligned(1024))) char sh[kOwn * kBufs * B::kBytes];
    __shared__ __attribute__((aligned(1024))) s16x8 kept[kHeld ? 1 : kWaves * (kK + kV) * 64];   // [wave][K's, V's][lane]
    __shared__ __attribute__((aligned(16))) float st[kOwn][kBufs][2][kTile];   // [buffer][lse log2 e, -D]

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3);
    const int half = HALVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
    const JobSeq sq = seq_of_job(a.s, blockIdx.x, lane);
    const int32_t q_lo = sq.q_lo, q_len = sq.q_len, k_lo = sq.k_lo, k_len = sq.k_len, slot = sq.k_slot;
    const int32_t runs = full_runs((int64_t)q_len * a.rep, a.split), kv_head = (blockIdx.x - sq.job0) % a.Hk;
    const int32_t rest = (blockIdx.x - sq.job0) / a.Hk, run = runs > 1 ? rest % runs : 0;
    const int32_t tile = full_tile(runs > 1 ? rest / runs : rest, (slot - 1) / KEYS + 1, a.causal, true, a.fold);
    const int32_t off = k_len - q_len;
    const int32_t tile_lo = tile * KEYS;                       // keys from here on
    const int32_t key0 = tile_lo + (KEYS == 128 ? 32 * wave : 0), key = key0 + (lane & 31);
    const int64_t key_at = min(key, max(k_len, 1) - 1);
    s16x8 k[kK], v[kV];
    if (k_len > 0) {
        load_columns<DK>(k, a.k + (k_lo + key_at) * a.k_row + kv_head * a.k_head, lane);
        load_columns<DV>(v, a.v + (k_lo + key_at) * a.v_row + kv_head * a.v_head, lane);
    } else {
#pragma unroll
        for (int t = 0; t < kK; ++t) k[t] = s16x8{};
#pragma unroll
        for (int t = 0; t < kV; ++t) v[t] = s16x8{};
    }
    s16x8* const own = kept + (kHeld ? 0 : wave * (kK + kV) * 64 + lane);   // (both halves')
    if (!kHeld && half == 0) {
#pragma unroll
        for (int t = 0; t < kK; ++t) own[t * 64] = k[t];
#pragma unroll
        for (int t = 0; t < kV; ++t) own[(kK + t) * 64] = v[t];
    }
    // the first token that sees the tile, and its first and last key of this wave
    const int32_t t_lo = tile_lo >= k_len ? q_len : a.causal ? max(0, tile_lo - off) : 0;
    const int32_t t_wave = a.causal ? key0 - off : 0, t_all = a.causal ? key0 + 31 - off : 0;
    const float c = a.scale * kLog2e;

    f32x16 dk[kTK], dv[kTV];
#pragma unroll
    for (int t = 0; t < kTK; ++t) clear(dk[t]);
#pragma unroll
    for (int t = 0; t < kTV; ++t) clear(dv[t]);
    const uint32_t base = lds_addr(sh) + (KEYS == 128 ? half : wave) * kBufs * B::kBytes;
    float(*const stats)[2][kTile] = st[KEYS == 128 ? half : wave];
    const int part = KEYS == 128 ? wave : 0;
    PairLoad<B, DK, DV, KEYS == 128> load;
    load.init(lane, wave, a.q_row, a.do_row);
    const uint32_t st_base = lds_addr(stats);
    const int64_t to_D = a.D - a.lse2;   // (both lie in the workspace)
    auto fetch = [&](int32_t hr, int32_t tok, int buf) {
        const int32_t head = kv_head * a.rep + hr;
        load.issue(base + buf * B::kBytes, a.q + (q_lo + (int64_t)tok) * a.q_row + head * a.q_head,
                   a.dout + (q_lo + (int64_t)tok) * a.do_row + head * a.do_head, q_len - tok);
        // the tokens' statistics, 64 values a wave
        if (part < kTile / 32) {
            const int i = 64 * part + lane;
            const int64_t at = (q_lo + (int64_t)min(tok + i % kTile, q_len - 1)) * a.H + head;
            load_word_to_lds(st_base + buf * kTile * 8 + 256 * part, a.lse2 + at + (i < kTile ? 0 : to_D));
        }
    };
    PairOperands<B, DK, DV> in;
    in.init(base, lane);
    auto compute = [&](int32_t tok, auto at, int buf) {
#pragma unroll
        for (int b = 0; b < kTile / 32; ++b) {
            f32x16 s, dp;
            const float* sb = &stats[buf][0][32 * b + 4 * (lane >> 5)];
            clear(s);
            // dp - D comes out of the product, which starts at -D (where there are registers for it)
            constexpr bool kStart = DK + DV < 192;
            clear(dp);
            if constexpr (kStart) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 di = *reinterpret_cast<const f32x4*>(sb + kTile + 2 * r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dp[r + e] = di[e];
                }
            }
#pragma unroll
            for (int t = 0; t < kK; ++t) s = T::mfma(in.x_rows(t, at + b * 64 * DK), kHeld ? k[t] : own[t * 64], s);
#pragma unroll
            for (int t = 0; t < kV; ++t) dp = T::mfma(in.y_rows(t, at + b * 64 * DV), kHeld ? v[t] : own[(kK + t) * 64], dp);
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 l = *reinterpret_cast<const f32x4*>(sb + 2 * r);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r + e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], c, -l[e]));
            }
            // rows of the block that do not see the key, or lie behind the last token
            if (tok + 32 * b < t_all || tok + 32 * b + 32 > q_len) {
                const int32_t at0 = tok + 32 * b + 4 * (lane >> 5);
                const int32_t from = a.causal ? key - off - at0 : 0, upto = q_len - at0;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = (r & 3) + 8 * (r >> 2);
                    if (i < from || i >= upto) s[r] = 0.0f;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                f32x4 di = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (!kStart) di = *reinterpret_cast<const f32x4*>(sb + kTile + 2 * r);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dp[r + e] = s[r + e] * (dp[r + e] + di[e]);
                    s[r + e] *= T::kUpBack;   // (1 in bfloat16)
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const s16x8 p = round8<T>(s, i), x = round8<T>(dp, i);   // rounded, the operands of the products
#pragma unroll
                for (int t = 0; t < (kTK > kTV ? kTK : kTV); ++t) {
                    const int tv = t < kTV ? t : 0, tk = t < kTK ? t : 0;
                    if (t < kTV) dv[tv] = T::mfma(in.y_columns(tv, at + (32 * b + 16 * i) * 2 * DV), p, dv[tv]);
                    if (t < kTK) dk[tk] = T::mfma(in.x_columns(tk, at + (32 * b + 16 * i) * 2 * DK), x, dk[tk]);
                }
            }
        }
    };

    // streamed tiles: rep heads of `per` each; this run's part of them
    const int32_t per = (q_len - t_lo + kTile - 1) / kTile;
    const int64_t all = t_lo < q_len ? (int64_t)per * a.rep : 0;
    const int32_t first = (int32_t)(all * run / runs), n = (int32_t)(all * (run + 1) / runs) - first;
    const int64_t job = (int64_t)a.first_job + blockIdx.x;
    if constexpr (KEYS == 128) {
        const int32_t most = (n + HALVES - 1) / HALVES, mine = half == 0 ? most : n - most, begin = first + half * most;
        const int32_t tok0 = mine > 0 ? t_lo + begin % per * kTile : 0;
        // of the tile that is fetched next, of the one in use
        int32_t hr = mine > 0 ? begin / per : 0, tok = tok0, now = tok0;
        auto next = [&](int32_t t) { return t + kTile < q_len ? t + kTile : t_lo; };
        stream_tiles(
            most, mine,
            [&](int32_t, int buf) {
                fetch(hr, tok, buf);
                tok = next(tok);
                hr += tok == t_lo;
            },
            [&](int32_t, auto buf) {
                if (now + kTile > t_wave) compute(now, Constant<decltype(buf)::value * B::kBytes>(), decltype(buf)::value);
                now = next(now);
            });
        static_assert(HALVES == 1 || sizeof(sh) >= kWaves * (kTK > kTV ? kTK : kTV) * 4096, "room for the sums");
        if constexpr (HALVES > 1) {
            add_half<kTK>(dk, sh, wave, half, lane);
            if (!add_half<kTV>(dv, sh, wave, half, lane)) return;
        }
        if (key >= slot) return;
        const int64_t at = (k_lo + (int64_t)key) * a.Hk + kv_head;
        // rows behind the keys in use have no gradient
        const bool used = key < k_len;
#pragma unroll
        for (int t = 0; t < kTK; ++t) {
            if (!used) clear(dk[t]);
            if (runs > 1)
                store_sums<DK>(a.part_dk + (job * KEYS + (key - tile_lo)) * DK, dk[t], t, lane);
            else
                store_piece<T, DK>(a.dk + at * DK, dk[t], t, a.scale, lane);
        }
#pragma unroll
        for (int t = 0; t < kTV; ++t) {
            if (!used) clear(dv[t]);
            if (runs > 1)
                store_sums<DV>(a.part_dv + (job * KEYS + (key - tile_lo)) * DV, dv[t], t, lane);
            else
                store_piece<T, DV>(a.dv_out + at * DV, dv[t], t, 1.0f / T::kUpBack, lane);
        }
    } else {
        // tiles first + wave + 4 i
        const int32_t mine = n > wave ? (n - wave + kWaves - 1) / kWaves : 0;
        auto tok_of = [&](int32_t i) { return t_lo + (first + wave + kWaves * i) % per * kTile; };
        stream_blocks<kBufs, B::kOwnLoads + 1>(
            mine, [&](int32_t i, int stage) { fetch((first + wave + kWaves * i) / per, tok_of(i), stage); },
            [&](int32_t i, int stage) { compute(tok_of(i), (uint32_t)stage * B::kBytes, stage); });
        // the four waves' sums, in their order: dK, then dV
        auto join = [&](auto& x, auto width, float* part, uint16_t* to, float f) {
            constexpr int W = decltype(width)::value;
            float* const so = reinterpret_cast<float*>(sh);
            wait_and_sync();
#pragma unroll
            for (int t = 0; t < kPieces<W>; ++t) put_piece<W>(so + wave * 32 * W, x[t], t, 1.0f, lane);
            wait_and_sync();
            for (int i = threadIdx.x; i < 32 * (W / 4); i += 256) {
                const int rr = i / (W / 4), gg = i % (W / 4);
                if (tile_lo + rr >= slot) continue;
                f32x4 y = get_piece<W>(so, rr, gg);
#pragma unroll
                for (int u = 1; u < kWaves; ++u) y += get_piece<W>(so + u * 32 * W, rr, gg);
                if (tile_lo + rr >= k_len) y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (runs > 1)
                    *reinterpret_cast<f32x4*>(part + (job * KEYS + rr) * W + 4 * gg) = y;
                else
                    *reinterpret_cast<s16x4*>(to + ((k_lo + (int64_t)(tile_lo + rr)) * a.Hk + kv_head) * W + 4 * gg) = round4<T>(y, f);
            }
        };
        join(dk, std::integral_constant<int, DK>(), a.part_dk, a.dk, a.scale);
        join(dv, std::integral_constant<int, DV>(), a.part_dv, a.dv_out, 1.0f / T::kUpBack);
    }
}

struct SumArgs {
    const float* part[2];       // [job][rows][width], one or (dK, dV) two of them
    uint16_t* to[2];
    int32_t width[2];
    float scale[2];
    FullSeqs s;                 // the sequences with several runs, a job for each tile and key head
    int32_t part0[kFullSeqs];
    int32_t first_job, rows, split, Hk, rep;
    bool causal, fold, keys;    // keys: rows are keys of the slot, else (token, head) pairs
};

// Adds the runs of a tile in their order.
template <typename T>
__global__ __launch_bounds__(256) void full_sum_kernel(const SumArgs a) {
    const JobSeq s = seq_of_job(a.s, blockIdx.x, threadIdx.x & 63);
    const int32_t nrows = a.keys ? s.k_slot : s.q_len * a.rep;
    const int32_t runs = full_runs(a.keys ? (int64_t)s.q_len * a.rep : s.k_len, a.split);
    const int32_t kv_head = (blockIdx.x - s.job0) % a.Hk, place = (blockIdx.x - s.job0) / a.Hk;
    const int32_t tile = full_tile(place, (nrows - 1) / a.rows + 1, a.causal, a.keys, a.fold);
    const int which = blockIdx.z, width = a.width[which], groups = width / 4;
    const int i = blockIdx.y * 256 + threadIdx.x, rr = i / groups, g = i % groups;
    const int32_t row = tile * a.rows + rr;
    if (rr >= a.rows || row >= nrows) return;
    const int64_t job = (int64_t)a.first_job + a.part0[s.index] + (int64_t)place * runs * a.Hk + kv_head;
    const float* p = a.part[which] + (job * a.rows + rr) * width + 4 * g;
    const int64_t step = (int64_t)a.Hk * a.rows * width;
    f32x4 x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
    for (int32_t r = 1; r < runs; ++r) x += *reinterpret_cast<const f32x4*>(p + r * step);
    const int64_t at = a.keys ? (s.k_lo + (int64_t)row) * a.Hk + kv_head
                              : (s.q_lo + (int64_t)(row / a.rep)) * (a.Hk * a.rep) + kv_head * a.rep + row % a.rep;
    *reinterpret_cast<s16x4*>(a.to[which] + at * width + 4 * g) = round4<T>(x, a.scale[which]);
}

template <typename T>
hipError_t launch_sum(SumArgs& b, const BwdArgs& a, const FullLaunch& l, const FullPlan& p, bool keys, hipStream_t stream) {
    b.s = l.tiles;
    for (int i = 0; i < kFullSeqs; ++i) b.part0[i] = l.part0[i];
    b.first_job = l.first_job, b.rows = p.rows, b.split = p.split, b.Hk = a.Hk, b.rep = a.rep;
    b.causal = a.causal, b.fold = l.fold, b.keys = keys;
    const int32_t widest = b.width[0] > b.width[1] ? b.width[0] : b.width[1];
    const dim3 grid(l.tile_jobs, (p.rows * (widest / 4) + 255) / 256, keys ? 2 : 1);
    hipLaunchKernelGGL((full_sum_kernel<T>), grid, dim3(256), 0, stream, b);
    return hipGetLastError();
}

template <typename T, int DK, int DV>
hipError_t launch_bwd(const FullCall& f, const FullPlan& dq, const FullPlan& dkv, const FullBwdSpace& ws,
                      hipStream_t stream) {
    BwdArgs a{};
    a.q = reinterpret_cast<const char*>(f.q);
    a.k = reinterpret_cast<const char*>(f.k);
    a.v = reinterpret_cast<const char*>(f.v);
    a.dout = reinterpret_cast<const char*>(f.dout);
    a.out = reinterpret_cast<const uint16_t*>(f.out_in);
    a.lse = f.lse_in;
    a.lse2 = ws.lse2, a.D = ws.D;
    a.part_dq = ws.dq, a.part_dk = ws.dk, a.part_dv = ws.dv;
    a.dq = reinterpret_cast<uint16_t*>(f.dq);
    a.dk = reinterpret_cast<uint16_t*>(f.dk);
    a.dv_out = reinterpret_cast<uint16_t*>(f.dv_out);
    a.q_row = 2 * f.q_row, a.q_head = 2 * f.q_head;
    a.k_row = 2 * f.k_row, a.k_head = 2 * f.k_head;
    a.v_row = 2 * f.v_row, a.v_head = 2 * f.v_head;
    a.do_row = 2 * f.do_row, a.do_head = 2 * f.do_head;
    a.H = f.H, a.Hk = f.Hk, a.rep = f.H / f.Hk, a.causal = f.causal != 0;
    a.scale = f.scale;
    for (const FullLaunch& l : dq.launches) {
        a.s = l.seqs, a.first_job = l.first_job, a.fold = l.fold, a.split = dq.split;
        if (dq.rows == 128 && dq.halves == 2)
            hipLaunchKernelGGL((full_dq_kernel<T, DK, DV, 128, 2>), dim3(l.jobs), dim3(512), 0, stream, a);
        else if (dq.rows == 128)
            hipLaunchKernelGGL((full_dq_kernel<T, DK, DV, 128, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((full_dq_kernel<T, DK, DV, 32, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && l.tile_jobs > 0) {
            SumArgs b{{ws.dq}, {a.dq}, {f.d}, {f.scale}};
            e = launch_sum<T>(b, a, l, dq, false, stream);
        }
        if (e != hipSuccess) return e;
    }
    for (const FullLaunch& l : dkv.launches) {
        a.s = l.seqs, a.first_job = l.first_job, a.fold = l.fold, a.split = dkv.split;
        // (at d = d_V = 128 registers for one group are missing, and the plan has two)
        if (dkv.rows == 128 && dkv.halves == 2)
            hipLaunchKernelGGL((full_dkv_kernel<T, DK, DV, 128, 2>), dim3(l.jobs), dim3(512), 0, stream, a);
        else if (dkv.rows == 32)
            hipLaunchKernelGGL((full_dkv_kernel<T, DK, DV, 32, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        else if constexpr (DK + DV == 256)
            return hipErrorInvalidValue;
        else
            hipLaunchKernelGGL((full_dkv_kernel<T, DK, DV, 128, 1>), dim3(l.jobs), dim3(256), 0, stream, a);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && l.tile_jobs > 0) {
            SumArgs b{{ws.dk, ws.dv}, {a.dk, a.dv_out}, {f.d, f.dv}, {f.scale, 1.0f / T::kUpBack}};
            e = launch_sum<T>(b, a, l, dkv, true, stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_full_bwd(const FullCall& f, const FullPlan& dq, const FullPlan& dkv, const FullBwdSpace& ws,
                           hipStream_t stream) {
#define KMIP_FULL_CASE(DK, DV) \
    if (f.d == DK && f.dv == DV) \
        return f.fp16 ? launch_bwd<Fp16, DK, DV>(f, dq, dkv, ws, stream) : launch_bwd<Bf16, DK, DV>(f, dq, dkv, ws, stream);
#define KMIP_FULL_BWD(DK) KMIP_FULL_CASE(DK, 16) KMIP_FULL_CASE(DK, 32) KMIP_FULL_CASE(DK, 64) KMIP_FULL_CASE(DK, 128)
    KMIP_FULL_BWD(16)
    KMIP_FULL_BWD(32)
    KMIP_FULL_BWD(64)
    KMIP_FULL_BWD(128)
#undef KMIP_FULL_BWD
#undef KMIP_FULL_CASE
    return hipErrorInvalidValue;
}

}  // namespace kmip
