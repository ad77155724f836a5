// The launches that kvb_attend plans, on the host: the library's own checks and plans with launches that print
// what they are given.  Arguments: heads, kv_heads, d, entries of a block list (0: none), then n and T of each sequence.
// A line for each launch: tile, then of each sequence its position in the call's tokens, runs and their blocks.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "kvb_host.cpp"

namespace cap {
hipError_t launch_kvb_append(const KvbAppendParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_kvb_select(const KvbSelectParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_kvb_attend(const KvbAttendParams& p, hipStream_t) {
    if (p.wgs == 0) return hipSuccess;
    std::printf("%d", p.tile);
    for (int i = 0; i < p.n_seq; ++i) std::printf(" %lld,%d,%d", (long long)p.seq[i].t0, p.seq[i].nsplit, p.seq[i].per);
    std::printf("\n");
    return hipSuccess;
}
}  // namespace cap

int main(int argc, char** argv) {
    if (argc < 7 || argc % 2 == 0) return 2;
    auto at = [](uint64_t x) { return reinterpret_cast<void*>((uintptr_t)x << 40); };
    kvb_attend_args a{};
    a.heads = std::atoi(argv[1]), a.kv_heads = std::atoi(argv[2]), a.d = std::atoi(argv[3]), a.n_sel = std::atoi(argv[4]);
    std::vector<kvb_seq> seqs;
    for (int i = 5; i < argc; i += 2) {
        const int64_t n = std::atoll(argv[i]), T = std::atoll(argv[i + 1]);
        seqs.push_back({at(10 + 3 * seqs.size()), at(11 + 3 * seqs.size()), static_cast<float*>(at(12 + 3 * seqs.size())), nullptr, nullptr,
                        (n + 63) / 64 * 64, n, T});
        a.tokens += T;
    }
    a.seqs = seqs.data(), a.n_seq = (int32_t)seqs.size(), a.in_dtype = CAP_DTYPE_BF16, a.scale = 1.0f;
    a.q = at(1), a.o = at(2), a.idx = a.n_sel ? static_cast<int32_t*>(at(3)) : nullptr;
    a.workspace = at(4), a.workspace_bytes = kvb_attend_workspace_bytes(&a);
    const int rc = kvb_attend(&a, nullptr);
    if (rc != CAP_OK) std::printf("status %d\n", rc);
    return rc == CAP_OK ? 0 : 1;
}
