// Checks of the 8-bit products' host-side and index rules on the CPU, run by
// test_gemm_q8_host.py.  Prints each violation; exits with 1 if any.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "gemm_tile.h"
#include "q8.h"

using namespace clearmoe;

static int g_bad = 0;
static void expect(bool ok, const char* what, long a, long b) {
    if (!ok && ++g_bad <= 20) std::printf("%s: %ld %ld\n", what, a, b);
}

// A segment's row tiles, up to the most rows a product may have.
static void row_tiles() {
    const int64_t top = (int64_t{1} << 31) - 1;
    for (int bm : {16, 64, 128, 256, 320})
        for (int64_t base : {int64_t{0}, int64_t{4096}, top / 2, top - 700})
            for (int64_t rows = base; rows <= base + 700; ++rows)
                expect(gb_row_tiles(static_cast<int>(rows), bm) == (rows + bm - 1) / bm, "row tiles", rows, bm);
}

// No product is taken whose launch, by any of the kernels, passes 2^32 threads.
static void launch() {
    const int64_t top = (int64_t{1} << 31) - 1;
    expect(q8_launch_fits(top, 1, 64, kQ8OutBf16), "rows", top, kQ8OutBf16);
    expect(!q8_launch_fits(top, 1, 0, kQ8OutF32), "rows", top, kQ8OutF32);
    expect(q8_launch_fits(top - 256 * 8, 128, 0, kQ8OutF32), "rows", top - 256 * 8, kQ8OutF32);
    expect(!q8_launch_fits(top - 256 * 8, 128, 1, kQ8OutF32), "rows of a group", top - 256 * 8, kQ8OutF32);
    expect(!q8_launch_fits(top, 129, 0, kQ8OutBf16), "columns", 129, kQ8OutBf16);
    expect(!q8_launch_fits(int64_t{1} << 28, 65536, 0, kQ8OutE4M3), "columns", 65536, kQ8OutE4M3);
    for (int out : {kQ8OutF32, kQ8OutBf16, kQ8OutE4M3, kQ8OutE5M2})
        for (int groups : {0, 1, 64})
            for (int N : {1, 128, 129, 1000, 65536}) {
                // the most rows that are taken
                int64_t lo = 0, hi = top;
                while (lo < hi) {
                    const int64_t mid = lo + (hi - lo + 1) / 2;
                    if (q8_launch_fits(mid, N, groups, out)) lo = mid;
                    else hi = mid - 1;
                }
                const int64_t tiles = ((lo + 255) / 256 + groups) * ((N + 127) / 128);
                const int64_t threads = (tiles + 7) / 8 * 8 * (out == kQ8OutF32 ? 512 : 256);
                expect(threads < (int64_t{1} << 32), "threads of a launch", lo, N);
                expect(lo == top || threads > (int64_t{1} << 32) - (int64_t{1} << 20) * 512, "refused too early", lo, N);
            }
}

// The kernel of each product M N groups out (as q8.h numbers them).
static void kernels(int n, char** v) {
    static int32_t offsets[65];
    const char* names[] = {"rows", "small", "middle", "large"};
    for (int i = 0; i + 3 < n; i += 4) {
        Q8Desc g{};
        g.M = std::atol(v[i]);
        g.N = std::atoi(v[i + 1]);
        g.nseg = std::atoi(v[i + 2]);
        g.seg_offsets = g.nseg > 0 ? offsets : nullptr;
        g.out = std::atoi(v[i + 3]);
        std::printf("%s\n", names[q8_kernel(g)]);
    }
}

int main(int argc, char** argv) {
    if (argc < 2) return 2;
    if (std::strcmp(argv[1], "row_tiles") == 0) row_tiles();
    else if (std::strcmp(argv[1], "launch") == 0) launch();
    else if (std::strcmp(argv[1], "kernels") == 0) kernels(argc - 2, argv + 2);
    else return 2;
    return g_bad != 0;
}
