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
// entry s: job0[s] .. job0[s + 1] - 1; sequences without a job have no entry.
constexpr int kFullSeqs = 128;

struct FullSeqs {
    int32_t q_lo[kFullSeqs], q_len[kFullSeqs], k_lo[kFullSeqs], k_len[kFullSeqs], k_slot[kFullSeqs], job0[kFullSeqs];
    int32_t count;
};

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
    int32_t split_rows;     // rows of the largest row tile whose keys are split, 0 if none is
};

struct FullPlan {
    int32_t rows = 0;    // rows of a row tile, 128 or 32
    int32_t split = 0;   // keys of a run, 0: not split
    int64_t jobs = 0;
    std::vector<FullLaunch> launches;
};

// dQ first (plan dq; it also writes D [Nq, H]), then dK and dV (plan dkv, rows: keys
// of a job).
hipError_t launch_full_bwd(const FullCall& f, const FullPlan& dq, const FullPlan& dkv, float* D, hipStream_t stream);
hipError_t launch_full_fwd(const FullCall& f, const FullPlan& p, float* part_o, float* part_ml, hipStream_t stream);

}  // namespace kmip
