// Host side of full softmax attention (include/kmip.h): argument checks, the
// cut into jobs, workspace layout and launches.
#include <algorithm>
#include <cstring>
#include <new>

#include "full_plan.h"
#include "kmip.h"

namespace {

using kmip::FullCall;
using kmip::FullLaunch;
using kmip::FullPlan;
using kmip::record_error;

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

kmip_status_t ok() { return record_error(KMIP_OK, "%s", ""); }

kmip_status_t hip_fail(hipError_t e, const char* what) {
    return record_error(KMIP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

struct Seq {
    int32_t q_lo, q_len, k_lo, k_len, k_slot;
};

// Where the sequences lie; NULL offsets: see include/kmip.h.
struct Sequences {
    const int32_t *q, *k, *len;
    int32_t count;
    int64_t Nq, Nk;

    Seq at(int32_t g) const {
        if (q == nullptr) return Seq{0, (int32_t)Nq, 0, len != nullptr ? len[0] : (int32_t)Nk, (int32_t)Nk};
        const int32_t* ko = k != nullptr ? k : q;
        const int32_t slot = ko[g + 1] - ko[g];
        return Seq{q[g], q[g + 1] - q[g], ko[g], len != nullptr ? len[g] : slot, slot};
    }
};

kmip_status_t check_offsets(const int32_t* off, int32_t G, int64_t N, const char* name) {
    if (off[0] != 0) return record_error(KMIP_ERR_INVALID_ARG, "%s[0]=%d must be 0", name, off[0]);
    for (int32_t g = 0; g < G; ++g)
        if (off[g + 1] < off[g]) return record_error(KMIP_ERR_INVALID_ARG, "%s decrease at %d", name, g);
    if (off[G] != N) return record_error(KMIP_ERR_INVALID_ARG, "%s[G]=%d != %lld", name, off[G], (long long)N);
    return KMIP_OK;
}

bool width_ok(int32_t d) { return d == 16 || d == 32 || d == 64 || d == 128; }

kmip_status_t check_call(const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths, int32_t G,
                         int64_t Nq, int64_t Nk, int32_t H, int32_t Hk, int32_t d, int32_t dv, Sequences* s) {
    constexpr int64_t kMost = (int64_t(1) << 31) - 4096;
    if (Nq < 0 || Nk < 0 || Nk >= kMost)
        return record_error(KMIP_ERR_INVALID_ARG, "Nq=%lld, Nk=%lld out of range", (long long)Nq, (long long)Nk);
    if (H < 1 || Hk < 1 || H % Hk != 0)
        return record_error(KMIP_ERR_INVALID_ARG, "H=%d must be a multiple of the %d key heads", H, Hk);
    if (!width_ok(d) || !width_ok(dv))
        return record_error(KMIP_ERR_UNSUPPORTED, "d=%d, d_V=%d not in {16, 32, 64, 128}", d, dv);
    if (Nq >= kMost || Nq * (int64_t)H >= kMost) return record_error(KMIP_ERR_INVALID_ARG, "Nq*H >= 2^31 - 4096");
    *s = Sequences{q_offsets, k_offsets, k_lengths, q_offsets != nullptr ? G : 1, Nq, Nk};
    if (q_offsets == nullptr) {
        if (k_offsets != nullptr) return record_error(KMIP_ERR_INVALID_ARG, "k_offsets without q_offsets");
    } else {
        if (G < 1) return record_error(KMIP_ERR_INVALID_ARG, "num_seqs=%d must be >= 1 with offsets", G);
        kmip_status_t e = check_offsets(q_offsets, G, Nq, "q_offsets");
        if (e == KMIP_OK) e = check_offsets(k_offsets != nullptr ? k_offsets : q_offsets, G, Nk, "k_offsets");
        if (e != KMIP_OK) return e;
    }
    if (k_lengths != nullptr)
        for (int32_t g = 0; g < s->count; ++g) {
            const int32_t* ko = k_offsets != nullptr ? k_offsets : q_offsets;
            const int64_t slot = ko == nullptr ? Nk : ko[g + 1] - ko[g];
            if (k_lengths[g] < 0 || k_lengths[g] > slot)
                return record_error(KMIP_ERR_INVALID_ARG, "k_lengths[%d]=%d outside [0, %lld]", g, k_lengths[g],
                                    (long long)slot);
        }
    return KMIP_OK;
}

bool finite_bits(float x) {   // (the sources are built without NaN tests)
    uint32_t b;
    std::memcpy(&b, &x, sizeof(b));
    return (b & 0x7F800000u) != 0x7F800000u;
}

// Cuts the list of sequences, with tiles_of(seq) tiles (of all key heads) of
// streamed_of(seq) streamed rows each, into launches, the costliest sequences
// first (ties in their order), so that the last jobs are short ones.
template <typename Tiles, typename Kept, typename Streamed>
kmip_status_t cut(std::vector<Seq>& seqs, bool causal, const Tiles& tiles_of, const Kept& kept_of,
                  const Streamed& streamed_of, FullPlan* p) {
    auto cost = [](const Seq& s) { return (int64_t)std::max(s.q_len, 1) * std::max(s.k_len, 1); };
    std::stable_sort(seqs.begin(), seqs.end(), [&](const Seq& x, const Seq& y) { return cost(x) > cost(y); });
    p->jobs = 0;
    // (a call with runs keeps the long form, whose launches list the cut sequences a second time)
    bool same = p->split == 0;
    for (const Seq& s : seqs) same = same && s.q_lo == s.k_lo && s.q_len == s.k_len && s.k_len == s.k_slot;
    const size_t most = same ? 2 * kmip::kFullSeqs : kmip::kFullSeqs;
    for (size_t first = 0; first < seqs.size(); first += most) {
        p->launches.emplace_back();
        FullLaunch& l = p->launches.back();
        std::memset(static_cast<void*>(&l), 0, sizeof(l));
        const size_t n = std::min(seqs.size() - first, most);
        l.seqs.same = same;
        int64_t jobs = 0, tile_jobs = 0;
        auto put = [&](kmip::FullSeqs& q, const Seq& s, int64_t job0) {
            const int32_t i = q.count++;
            int32_t* const w = q.w + i;
            w[0] = s.q_lo, w[most] = s.q_len, w[2 * most] = (int32_t)job0;
            if (!same) w[3 * most] = s.k_lo, w[4 * most] = s.k_len, w[5 * most] = s.k_slot;
            return i;
        };
        for (size_t i = 0; i < n; ++i) {
            const Seq& s = seqs[first + i];
            const int64_t tiles = tiles_of(s);
            const int32_t runs = kmip::full_runs(streamed_of(s), p->split);
            put(l.seqs, s, jobs);
            if (runs > 1) {
                l.part0[put(l.tiles, s, tile_jobs)] = (int32_t)jobs;
                tile_jobs += tiles;
                l.runs = std::max(l.runs, runs);
                l.tile_rows = (int32_t)std::max<int64_t>(l.tile_rows, std::min<int64_t>(p->rows, kept_of(s)));
            }
            jobs += tiles * runs;
            if (p->jobs + jobs >= (int64_t(1) << 31) - 1)
                return record_error(KMIP_ERR_INVALID_ARG, "too many rows and key runs for one call");
        }
        l.jobs = (int32_t)jobs;
        l.tile_jobs = (int32_t)tile_jobs;
        l.first_job = (int32_t)p->jobs;
        // two workgroups a CU are resident at once, or more (see full_tile)
        l.fold = p->halves == 1 && causal && jobs <= 512;
        p->jobs += jobs;
    }
    return KMIP_OK;
}

// Workgroups that are resident at once whatever the widths, two on each of 256 CUs (at d, d_V <= 64 a CU holds up to four of the
// one-group kernels: the plan has one number for all of them).
constexpr int64_t kSlots = 512;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// How `seqs` become tiles of kept rows, kept_of(s) of them for each key head, that
// stream streamed_of(s) rows each; width: d + d_V.
//   128 rows: waves share the streamed tiles, a quarter of the traffic; for
//     tiles that are at least half full and fill the chip, by themselves or in runs
//     of at least 512 streamed rows.
//   32 rows otherwise, in runs of at least 512 where that makes more jobs (one text
//     of 1000 tokens, 8 heads, d = 64, forward and backward 40 us; 64 such texts of up to 1000
//     329 with this form, 196 with the other).
// Runs cost the sums' way through memory, so that there are as few as fill the chip
// (32 rows: 1024 jobs; one token over each of 64 caches of up to 32,767, d = 128 212 us with 1024 jobs aimed
// at, 234 with 512, 222 with 2048; over 8 of 8000 54, 50, 54).
//
// Two groups of waves on a 128-row tile (halves; only_halves: the kernel has no
// other form): a CU works on one tile at a time and the last ones take half as
// long, but the groups' sums have to be added and fewer workgroups share a CU.
// So at narrow widths, whose sums are small, where there are few jobs and they are long.
// us with one group and with two:
//   d = 32, causal, forward and backward: 16 heads, 3000 tokens 119, 103; 4 texts of 2048, 8 heads 115, 105
//   d = 64, the same: 8 heads, 4 texts of up to 2000 (208 jobs) 104, 77; 16 heads, 3000 tokens (376) 173, 159,
//     4096 tokens (512) 238, 206; 8 heads, 8 texts of up to 2000 (800 jobs of 1500 rows) 156, 169;
//     all pairs, 8 graphs of 1024 (512 jobs) 99, 108
// At d = d_V = 128 one workgroup of two groups or two of one fill a CU.  Two groups win where causal jobs, of unequal
// length, make one to two rounds of CUs, and where jobs make a whole round; with fewer, one group has runs, with more, jobs
// that wait fill the gaps.  us of the forward with one group and with two (a head's tokens x heads: jobs):
//   causal: 8192 x 3: 192 96, 98; 4096 x 8: 256 82, 64; 8192 x 5: 320 157, 123; 16,384 x 3: 384 306, 245;
//     8192 x 8: 512 169, 145; 2048 x 32: 512 50, 49; 6144 x 12: 576 142, 138; 2304 x 32: 576 59, 64;
//     8192 x 10: 640 194, 196; 8192 x 12: 768 207, 230; 16,384 x 8: 1024 542, 541; 8192 x 32: 2048 517, 556
//   all pairs: 3900 x 8: 243 93, 120; 4096 x 8: 256 92, 78; 2048 x 16: 256 62, 45; 4200 x 8: 262 115, 135;
//     6144 x 8: 384 173, 190; 8192 x 8: 512 260, 271; 8192 x 16: 1024 506, 535
template <typename Kept, typename Streamed>
kmip_status_t plan(std::vector<Seq>& seqs, int32_t Hk, bool causal, const Kept& kept_of, const Streamed& streamed_of,
                   int32_t width, bool only_halves, FullPlan* p) {
    auto tiles = [&](const Seq& s, int64_t rows) { return (kept_of(s) + rows - 1) / rows * Hk; };
    int64_t kept = 0, jobs = 0, work = 0, work32 = 0, longest = 0;
    for (const Seq& s : seqs) {
        kept += kept_of(s) * Hk;
        jobs += tiles(s, 128);
        work += tiles(s, 128) * streamed_of(s);
        work32 += tiles(s, 32) * streamed_of(s);
        longest = std::max<int64_t>(longest, streamed_of(s));
    }
    const bool full = 2 * kept >= 128 * jobs;
    p->rows = full && (jobs >= kSlots || work >= kSlots * 512) ? 128 : 32;
    const int64_t half_slots = kSlots / 2;
    const int64_t least = width <= 64 || jobs <= half_slots ? 1024 : 2048;
    const bool halves = width <= 192 ? jobs <= 2 * kSlots && work >= jobs * least
                                     : (jobs == half_slots || (causal && jobs > half_slots && jobs <= kSlots)) && work >= jobs * 2048;
    p->halves = p->rows == 128 && (only_halves || halves) ? 2 : 1;
    int64_t run = 0;
    if (p->rows == 32)
        run = std::max<int64_t>(round_up(work32 / (2 * kSlots), 128), 512);
    else if (jobs < (p->halves == 2 ? half_slots : kSlots))
        run = std::max<int64_t>(round_up(work / kSlots, 128), 512);
    static_assert(2 * 512 >= KMIP_FULL_LONG, "streams below are not cut");
    p->split = run > 0 && longest >= 2 * run ? (int32_t)std::min<int64_t>(run, INT32_MAX) : 0;
    return cut(seqs, causal, [&](const Seq& s) { return tiles(s, p->rows); }, kept_of, streamed_of, p);
}

kmip_status_t plan_rows(const Sequences& sq, int32_t H, int32_t Hk, bool causal, int32_t width, FullPlan* p) {
    const int64_t rep = H / Hk;
    std::vector<Seq> seqs;
    for (int32_t g = 0; g < sq.count; ++g)
        if (sq.at(g).q_len > 0) seqs.push_back(sq.at(g));
    return plan(
        seqs, Hk, causal, [=](const Seq& s) { return s.q_len * rep; }, [](const Seq& s) { return (int64_t)s.k_len; }, width,
        false, p);
}

// Key tiles cover every slot, since rows without a gradient are written too.
kmip_status_t plan_keys(const Sequences& sq, int32_t H, int32_t Hk, bool causal, int32_t width, FullPlan* p) {
    const int64_t rep = H / Hk;
    std::vector<Seq> seqs;
    for (int32_t g = 0; g < sq.count; ++g)
        if (sq.at(g).k_slot > 0) seqs.push_back(sq.at(g));
    return plan(
        seqs, Hk, causal, [](const Seq& s) { return (int64_t)s.k_slot; }, [=](const Seq& s) { return s.q_len * rep; }, width,
        width == 256, p);
}

// (The workspace queries plan without a mask: a causal plan never has more runs, since a mask only makes two groups, and so
// none or longer ones, more likely.)

// Workspace of the forward: the runs' sums, then their maxima and sums of weights.
struct FwdLayout {
    size_t ml, total;
};
FwdLayout fwd_layout(const FullPlan& p, int32_t dv) {
    if (p.split == 0) return FwdLayout{0, 0};
    const size_t rows = (size_t)p.jobs * p.rows;
    const size_t ml = align_up(rows * dv * sizeof(float));
    return FwdLayout{ml, ml + align_up(rows * 2 * sizeof(float))};
}

// Workspace of the backward: lse2 and D, then the runs' sums of dQ, dK and dV.
struct BwdLayout {
    size_t D, dq, dk, dv, total;
};
BwdLayout bwd_layout(const FullPlan& dq, const FullPlan& dkv, int64_t Nq, int32_t H, int32_t d, int32_t dv) {
    BwdLayout L;
    auto sums = [](const FullPlan& p, int32_t width) {
        return p.split == 0 ? (size_t)0 : align_up((size_t)p.jobs * p.rows * width * sizeof(float));
    };
    L.D = align_up((size_t)Nq * H * sizeof(float));
    L.dq = 2 * L.D;
    L.dk = L.dq + sums(dq, d);
    L.dv = L.dk + sums(dkv, d);
    L.total = L.dv + sums(dkv, dv);
    return L;
}

// A stride in values between rows of a 16-bit tensor that the kernels read 16
// bytes at a time.
kmip_status_t check_strides(const char* name, const void* p, int64_t row, int64_t head) {
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0)
        return record_error(KMIP_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0)
        return record_error(KMIP_ERR_INVALID_ARG, "%s: strides %lld, %lld must be multiples of 8 values", name, (long long)row,
                            (long long)head);
    if (row >= (int64_t(1) << 23))
        return record_error(KMIP_ERR_UNSUPPORTED, "%s: %lld values between rows", name, (long long)row);
    return KMIP_OK;
}

kmip_status_t fill_call(const void* Q, const void* K, const void* V, int32_t dtype, const int64_t* strides, int64_t Nq,
                        int64_t Nk, int32_t H, int32_t Hk, int32_t d, int32_t dv, float scale, int32_t causal, FullCall* f) {
    if (dtype != KMIP_BF16 && dtype != KMIP_FP16) return record_error(KMIP_ERR_UNSUPPORTED, "dtype %d", dtype);
    if (!finite_bits(scale) || !(scale > 0.0f)) return record_error(KMIP_ERR_INVALID_ARG, "scale must be finite and > 0");
    *f = FullCall{};
    f->q = Q, f->k = K, f->v = V;
    f->Nq = Nq, f->Nk = Nk, f->H = H, f->Hk = Hk, f->d = d, f->dv = dv, f->causal = causal != 0;
    f->fp16 = dtype == KMIP_FP16;
    f->scale = scale;
    const int64_t packed[6] = {(int64_t)H * d, d, (int64_t)Hk * d, d, (int64_t)Hk * dv, dv};
    const int64_t* s = strides != nullptr ? strides : packed;
    f->q_row = s[0], f->q_head = s[1], f->k_row = s[2], f->k_head = s[3], f->v_row = s[4], f->v_head = s[5];
    f->do_row = strides != nullptr ? 0 : (int64_t)H * dv, f->do_head = strides != nullptr ? 0 : dv;
    kmip_status_t e = KMIP_OK;
    if (Nq > 0) e = check_strides("Q", Q, f->q_row, f->q_head);
    if (e == KMIP_OK && Nk > 0) e = check_strides("K", K, f->k_row, f->k_head);
    if (e == KMIP_OK && Nk > 0) e = check_strides("V", V, f->v_row, f->v_head);
    return e;
}

kmip_status_t check_workspace(const void* ws, size_t bytes, size_t need) {
    if (need == 0) return KMIP_OK;
    if (ws == nullptr || bytes < need)
        return record_error(KMIP_ERR_WORKSPACE, "workspace of %zu bytes < %zu required", bytes, need);
    if ((reinterpret_cast<uintptr_t>(ws) & (kAlign - 1)) != 0)
        return record_error(KMIP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    return KMIP_OK;
}

// No exception crosses the ABI (the lists of jobs are the only allocations).
template <typename F>
kmip_status_t guarded(const F& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return record_error(KMIP_ERR_INVALID_ARG, "out of host memory for the list of sequences");
    }
}

}  // namespace

extern "C" {

size_t kmip_full_fwd_workspace_size(const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths,
                                    int32_t num_seqs, int64_t Nq, int64_t Nk, int32_t H, int32_t Hk, int32_t d, int32_t dv) {
    size_t bytes = 0;
    guarded([&]() {
        Sequences sq;
        FullPlan p;
        kmip_status_t e = check_call(q_offsets, k_offsets, k_lengths, num_seqs, Nq, Nk, H, Hk, d, dv, &sq);
        if (e == KMIP_OK) e = plan_rows(sq, H, Hk, false, d + dv, &p);
        if (e == KMIP_OK) bytes = fwd_layout(p, dv).total;
        return e;
    });
    return bytes;
}

kmip_status_t kmip_full_fwd(const void* Q, const void* K, const void* V, int32_t dtype, const int64_t* strides,
                            const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths,
                            int32_t num_seqs, int64_t Nq, int64_t Nk, int32_t H, int32_t Hk, int32_t d, int32_t dv,
                            float scale, int32_t causal, void* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
    return guarded([&]() {
        Sequences sq;
        FullCall f;
        FullPlan p;
        kmip_status_t e = check_call(q_offsets, k_offsets, k_lengths, num_seqs, Nq, Nk, H, Hk, d, dv, &sq);
        if (e == KMIP_OK && Nq > 0 && (!Q || !out || !lse || (Nk > 0 && (!K || !V))))
            e = record_error(KMIP_ERR_INVALID_ARG, "null buffer passed to kmip_full_fwd");
        if (e == KMIP_OK) e = fill_call(Q, K, V, dtype, strides, Nq, Nk, H, Hk, d, dv, scale, causal, &f);
        if (e == KMIP_OK && Nq > 0 && (reinterpret_cast<uintptr_t>(out) & 15u) != 0)
            e = record_error(KMIP_ERR_INVALID_ARG, "out must be 16-byte aligned");
        if (e == KMIP_OK) e = plan_rows(sq, H, Hk, causal != 0, d + dv, &p);
        if (e != KMIP_OK) return e;
        const FwdLayout L = fwd_layout(p, dv);
        if ((e = check_workspace(workspace, workspace_bytes, L.total)) != KMIP_OK) return e;
        f.out = out;
        f.lse = lse;
        char* ws = reinterpret_cast<char*>(workspace);
        hipError_t h = kmip::launch_full_fwd(f, p, reinterpret_cast<float*>(ws),
                                             L.total > 0 ? reinterpret_cast<float*>(ws + L.ml) : nullptr,
                                             reinterpret_cast<hipStream_t>(stream));
        return h == hipSuccess ? ok() : hip_fail(h, "full attention launch");
    });
}

size_t kmip_full_bwd_workspace_size(const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths,
                                    int32_t num_seqs, int64_t Nq, int64_t Nk, int32_t H, int32_t Hk, int32_t d, int32_t dv) {
    size_t bytes = 0;
    guarded([&]() {
        Sequences sq;
        FullPlan dq, dkv;
        kmip_status_t e = check_call(q_offsets, k_offsets, k_lengths, num_seqs, Nq, Nk, H, Hk, d, dv, &sq);
        if (e == KMIP_OK) e = plan_rows(sq, H, Hk, false, d + dv, &dq);
        if (e == KMIP_OK) e = plan_keys(sq, H, Hk, false, d + dv, &dkv);
        if (e == KMIP_OK) bytes = bwd_layout(dq, dkv, Nq, H, d, dv).total;
        return e;
    });
    return bytes;
}

kmip_status_t kmip_full_bwd(const void* Q, const void* K, const void* V, const void* dOut, const void* out,
                            const float* lse, int32_t dtype, const int64_t* strides, const int32_t* q_offsets,
                            const int32_t* k_offsets, const int32_t* k_lengths, int32_t num_seqs, int64_t Nq, int64_t Nk,
                            int32_t H, int32_t Hk, int32_t d, int32_t dv, float scale, int32_t causal, void* dQ, void* dK,
                            void* dV, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() {
        Sequences sq;
        FullCall f;
        FullPlan dq, dkv;
        kmip_status_t e = check_call(q_offsets, k_offsets, k_lengths, num_seqs, Nq, Nk, H, Hk, d, dv, &sq);
        if (e == KMIP_OK && ((Nq > 0 && (!Q || !dOut || !out || !lse || !dQ)) || (Nk > 0 && (!K || !V || !dK || !dV))))
            e = record_error(KMIP_ERR_INVALID_ARG, "null buffer passed to kmip_full_bwd");
        if (e == KMIP_OK) e = fill_call(Q, K, V, dtype, strides, Nq, Nk, H, Hk, d, dv, scale, causal, &f);
        if (e != KMIP_OK) return e;
        if (strides != nullptr) f.do_row = strides[6], f.do_head = strides[7];
        if (Nq > 0) e = check_strides("dOut", dOut, f.do_row, f.do_head);
        for (const void* p : {out, static_cast<const void*>(dQ), static_cast<const void*>(dK), static_cast<const void*>(dV)})
            if (e == KMIP_OK && (reinterpret_cast<uintptr_t>(p) & 15u) != 0)
                e = record_error(KMIP_ERR_INVALID_ARG, "out, dQ, dK and dV must be 16-byte aligned");
        if (e == KMIP_OK) e = plan_rows(sq, H, Hk, causal != 0, d + dv, &dq);
        if (e == KMIP_OK) e = plan_keys(sq, H, Hk, causal != 0, d + dv, &dkv);
        if (e != KMIP_OK) return e;
        const BwdLayout L = bwd_layout(dq, dkv, Nq, H, d, dv);
        if ((e = check_workspace(workspace, workspace_bytes, L.total)) != KMIP_OK) return e;
        f.dout = dOut, f.out_in = out, f.lse_in = lse;
        f.dq = dQ, f.dk = dK, f.dv_out = dV;
        auto at = [&](size_t off) { return reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + off); };
        const kmip::FullBwdSpace ws{at(0), at(L.D), at(L.dq), at(L.dk), at(L.dv)};
        hipError_t h = kmip::launch_full_bwd(f, dq, dkv, ws, reinterpret_cast<hipStream_t>(stream));
        return h == hipSuccess ? ok() : hip_fail(h, "full attention backward launch");
    });
}

}  // extern "C"
