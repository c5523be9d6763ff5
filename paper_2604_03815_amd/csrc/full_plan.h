// Host side of full softmax attention: what a call is, and how it is cut into
// jobs (full_api.hip), for its launchers (full_fwd.hip, full_bwd.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "kmip_internal.h"

namespace kmip {

// The sequences of one launch travel in the kernel's arguments: a launch needs
// no copy of them in device memory, and a captured one keeps them.  Jobs of
// entry s: job0(s) .. job0(s + 1) - 1; sequences without a job have no entry.
// Twice as many fit where queries and keys lie alike (same; 300 graphs of 20 to
// 100 nodes, 4 heads, d = 32, forward and backward 105 us in nine launches, 89 in six).
constexpr int kFullSeqs = 128;

struct FullSeqs {
    int32_t w[6 * kFullSeqs];   // q_lo, q_len, job0, then (not same) k_lo, k_len, k_slot
    int32_t count;
    bool same;

    __host__ __device__ int32_t most() const { return same ? 2 * kFullSeqs : kFullSeqs; }
    __host__ __device__ int32_t q_lo(int32_t s) const { return w[s]; }
    __host__ __device__ int32_t q_len(int32_t s) const { return w[most() + s]; }
    __host__ __device__ int32_t job0(int32_t s) const { return w[2 * most() + s]; }
    __host__ __device__ int32_t k_lo(int32_t s) const { return w[same ? s : 3 * kFullSeqs + s]; }
    __host__ __device__ int32_t k_len(int32_t s) const { return w[same ? most() + s : 4 * kFullSeqs + s]; }
    __host__ __device__ int32_t k_slot(int32_t s) const { return w[same ? most() + s : 5 * kFullSeqs + s]; }
};

// Runs that the streamed rows of a tile are cut into.
__host__ __device__ inline int32_t full_runs(int64_t streamed, int32_t split) {
    return split > 0 && streamed > split ? (int32_t)((streamed - 1) / split + 1) : 1;
}

// End of a tile's run from lo on, of streamed rows that end at hi (both below 2^31, while lo + split may pass it).
__host__ __device__ inline int32_t full_run_end(int32_t lo, int32_t hi, int32_t split) {
    return hi - lo > split ? lo + split : hi;
}

// Tile of place i of n.  Causal tiles differ in work; `falling`: tile 0 has the
// most.  Most first while workgroups queue for the CUs.  Where all of them are
// resident at once, the second half in the opposite order (fold), so that the
// second workgroup of a CU is the shorter the longer its first one is.
__host__ __device__ inline int32_t full_tile(int32_t i, int32_t n, bool causal, bool falling, bool fold) {
    if (!causal) return i;
    if (fold && i >= n / 2) i = n - 1 - (i - n / 2);
    return falling ? i : n - 1 - i;
}

struct FullCall {
    const void *q, *k, *v, *dout, *out_in;
    void* out;
    float* lse;
    const float* lse_in;
    void *dq, *dk, *dv_out;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, do_row, do_head;   // values between tokens, heads
    int64_t Nq, Nk;
    int32_t H, Hk, d, dv, causal;
    bool fp16;
    float scale;
};

struct FullLaunch {
    FullSeqs seqs;
    int32_t jobs, first_job;
    bool fold;              // tiles in the order of full_tile()'s fold
    // the launch that joins runs: the sequences that have several, with a job for
    // each tile and key head; most rows of a tile and most runs among them
    FullSeqs tiles;
    int32_t part0[kFullSeqs];   // their first jobs in the launch above
    int32_t tile_jobs, tile_rows, runs;
};

struct FullPlan {
    int32_t rows = 0;    // rows (or keys) of a tile, 128 or 32
    int32_t halves = 1;  // groups of four waves that share a tile's streamed rows, 2 or 1
    int32_t split = 0;   // streamed rows of a run, 0: not split
    int64_t jobs = 0;
    std::vector<FullLaunch> launches;
};

// Workspace of the backward.
struct FullBwdSpace {
    float *lse2, *D;               // [Nq, H] each
    float *dq, *dk, *dv;           // [job][rows][width] sums of runs
};
// dQ first (plan dq; it also writes lse2 and D), then dK and dV (plan dkv).
hipError_t launch_full_bwd(const FullCall& f, const FullPlan& dq, const FullPlan& dkv, const FullBwdSpace& ws,
                           hipStream_t stream);
hipError_t launch_full_fwd(const FullCall& f, const FullPlan& p, float* part_o, float* part_ml, hipStream_t stream);

}  // namespace kmip
