// Host-only check run under AddressSanitizer and UndefinedBehaviorSanitizer (tests/test_cache8_host.py builds and runs it; no GPU).  It links the
// argument checks and the planning of the cache's entry points against stub launchers, and walks extreme sizes: every call must either be
// refused or reach its launcher with numbers that fit.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "../../paper_2107_06419_amd/csrc/flat_cache8.hpp"

static int g_launches = 0, g_failed = 0;
#define EXPECT(cond)                                         \
    do {                                                     \
        if (!(cond)) {                                       \
            printf("FAILED line %d: %s\n", __LINE__, #cond); \
            ++g_failed;                                      \
        }                                                    \
    } while (0)

namespace flat {
hipError_t launch_rope(const RopeProblem& p, hipStream_t) {
    ++g_launches;
    return (long long)p.B * p.N * p.d <= 0x7fffffffLL ? hipSuccess : hipErrorInvalidValue;
}
hipError_t launch_cache8_write(const flat_cache8& c, const CacheWrite& w, hipStream_t) {
    ++g_launches;
    return (long long)w.B * cache8_write_blocks(w.N) * c.n_heads * 2 <= 0x7fffffffLL ? hipSuccess : hipErrorInvalidValue;
}
hipError_t launch_cache8_copy(const flat_cache8&, const int*, const int*, int, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_cache8_fork(const flat_cache8&, int*, int, int, int*, const int*, const int*, const int*, int, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_cache8_free(int*, int, int, int*, const int*, int, int, int*, int*, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_cache8_compact(const flat_cache8&, const int*, int*, int, int, int*, int*, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_cache8_fwd(const flat_cache8& c, const Cache8Attend& a, const Cache8Plan& p, hipStream_t) {
    ++g_launches;
    const long long rows = (long long)a.Nq * (a.H / c.n_heads);
    const bool fits = p.entries > 0 && (long long)a.B * p.row_blocks == p.entries && (long long)p.row_blocks * p.rows_per_block >= rows && (p.limit == 0 || (p.limit >= p.entries && p.limit >= p.aim)) &&
                      (long long)(p.limit ? p.limit : p.entries) * c.n_heads <= 0x7ffffff8LL && (long long)a.B * c.n_heads * rows <= 0x7fffffffLL &&
                      (long long)a.max_pages * c.page_tokens <= 0x7fffffffLL;
    return fits ? hipSuccess : hipErrorInvalidValue;
}
}  // namespace flat

int main() {
    const int sizes[] = {1, 2, 7, 16, 48, 64, 1000, 65536, 1 << 20, 0x7fffffff};
    int ok = 0, refused = 0;
    auto count = [&](int rc) {
        EXPECT(rc == FLAT_OK || rc == FLAT_ERR_SHAPE || rc == FLAT_ERR_WORKSPACE || rc == FLAT_ERR_ALIAS);
        rc == FLAT_OK ? ++ok : ++refused;
    };
    auto at = [](int i) { return (void*)(uintptr_t)(0x1000ull + ((unsigned long long)i << 56)); };
    for (int n_pages : sizes)
        for (int heads : sizes)
            for (int T : {16, 64, 65536})
                for (int d : {32, 256})
                    for (int B : sizes)
                        for (int N : sizes) {
                            const flat_cache8 c{at(1), at(2), (float*)at(3), (float*)at(4), n_pages, heads, T, d, 0};
                            const int max_pages = n_pages < 1 << 14 ? n_pages : 1 << 14;
                            count(flat_attn_cache8_write(&c, at(5), at(6), B, N, (int*)at(7), max_pages, (int*)at(8), nullptr, nullptr));
                            const int H = heads <= 0x7fffffff / 5 ? heads * 5 : heads;
                            const size_t need = flat_attn_fwd_cache8_workspace_bytes(B, H, heads, N, 64, d);
                            count(flat_attn_fwd_cache8(&c, at(5), at(6), B, H, N, (int*)at(7), max_pages, (int*)at(8), (int*)at(9), 1.f, 1, at(10), ~(size_t)0 >> 8, nullptr));
                            EXPECT(need < ((size_t)1 << 60));
                            count(flat_attn_rope(at(1), at(2), heads, at(3), at(4), 1, B, N, d, 1, d, 1, (double*)at(5), (int*)at(6), 1.f, 0, nullptr));
                            count(flat_attn_cache8_copy_pages(&c, (int*)at(5), (int*)at(6), N, nullptr));
                            count(flat_attn_cache8_fork(&c, (int*)at(5), max_pages, B, (int*)at(6), (int*)at(7), (int*)at(8), (int*)at(9), N, nullptr));
                            count(flat_attn_cache8_free((int*)at(5), max_pages, B, (int*)at(6), (int*)at(7), N, n_pages, (int*)at(8), (int*)at(9), nullptr));
                            count(flat_attn_cache8_compact(&c, (int*)at(5), (int*)at(6), max_pages, B, (int*)at(7), at(8), ~(size_t)0 >> 8, nullptr));
                        }
    EXPECT(ok == g_launches && ok > 1000 && refused > 1000);
    double f[128];
    for (int rot = 2; rot <= 256; rot += 2)
        for (int s = 0; s < 4; ++s) EXPECT(flat_attn_rope_freqs(f, rot, 1e4, s, 8.0, 4096.0, 1.0, 32.0) == FLAT_OK);
    printf(g_failed ? "%d checks failed\n" : "cache8 host checks passed\n", g_failed);
    return g_failed != 0;
}
