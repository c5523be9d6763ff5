// The plans of full attention's calls, without a GPU: the host side as it is, with launchers that print what they are given.
// Reads calls from the standard input, one a line:
//   bwd H Hk d dv causal Nq Nk G, then (G > 0) G + 1 offsets of queries, G + 1 of keys and G lengths
// and prints a line for each: for each plan "fwd|dq|dkv rows halves split jobs launches", then "keys N", the keys that the
// runs of forward's or dQ's longest sequence take, and "status S".
#include "full_api.hip"

#include <cstdarg>
#include <cstdio>
#include <iostream>

extern "C" const char* hipGetErrorString(hipError_t) { return ""; }

namespace kmip {

kmip_status_t record_error(kmip_status_t s, const char*, ...) { return s; }

static void show(const char* name, const FullPlan& p) {
    std::printf(" %s %d %d %d %lld %zu", name, p.rows, p.halves, p.split, (long long)p.jobs, p.launches.size());
}

// Keys that the runs of the longest sequence take one after the other, as the kernels form a run's bounds; -1 for a gap.
static void show_keys(const FullPlan& p) {
    int32_t k_len = 0;
    for (const FullLaunch& l : p.launches)
        for (int32_t i = 0; i < l.seqs.count; ++i) k_len = std::max(k_len, l.seqs.k_len(i));
    const int32_t runs = full_runs(k_len, p.split);
    int64_t end = 0;
    for (int32_t run = 0; run < runs && end >= 0; ++run) {
        const int32_t lo = p.split > 0 ? run * p.split : 0, hi = p.split > 0 ? full_run_end(lo, k_len, p.split) : k_len;
        end = lo == end ? hi : -1;
    }
    std::printf(" keys %lld", (long long)end);
}

hipError_t launch_full_fwd(const FullCall&, const FullPlan& p, float*, float*, hipStream_t) {
    show("fwd", p);
    show_keys(p);
    return hipSuccess;
}

hipError_t launch_full_bwd(const FullCall&, const FullPlan& dq, const FullPlan& dkv, const FullBwdSpace&, hipStream_t) {
    show("dq", dq);
    show("dkv", dkv);
    show_keys(dq);
    return hipSuccess;
}

}  // namespace kmip

int main() {
    int bwd, H, Hk, d, dv, causal, G;
    int64_t Nq, Nk;
    void* const some = reinterpret_cast<void*>(256);   // (never dereferenced: nothing is launched)
    const size_t room = size_t(1) << 50;
    while (std::cin >> bwd >> H >> Hk >> d >> dv >> causal >> Nq >> Nk >> G) {
        std::vector<int32_t> qo(G + 1), ko(G + 1), len(G);
        if (G > 0)
            for (auto* x : {&qo, &ko, &len})
                for (int32_t& v : *x) std::cin >> v;
        const int32_t *q = G > 0 ? qo.data() : nullptr, *k = G > 0 ? ko.data() : nullptr, *l = G > 0 ? len.data() : nullptr;
        int s;
        if (bwd)
            s = kmip_full_bwd(some, some, some, some, some, static_cast<float*>(some), KMIP_BF16, nullptr, q, k, l, G, Nq, Nk, H, Hk, d,
                              dv, 1.0f, causal, some, some, some, some, room, nullptr);
        else
            s = kmip_full_fwd(some, some, some, KMIP_BF16, nullptr, q, k, l, G, Nq, Nk, H, Hk, d, dv, 1.0f, causal, some,
                              static_cast<float*>(some), some, room, nullptr);
        std::printf(" status %d\n", s);
    }
}
