// Checks of the 4-bit products' host-side rules on the CPU, run by
// test_gemm_q4_host.py.  Prints each violation; exits with 1 if any.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "q8.h"

using namespace clearmoe;

static int g_bad = 0;
static void expect(bool ok, const char* what, long a, long b) {
    if (!ok && ++g_bad <= 20) std::printf("%s: %ld %ld\n", what, a, b);
}

static const char* const kNames[] = {"rows", "small", "split", "wide", "middle", "deep", "large"};

static Q8Desc desc(int64_t M, int N, int K, int groups, int fa, int out) {
    static int32_t offsets[65];
    Q8Desc g{};
    g.M = M; g.N = N; g.K = K; g.nseg = groups; g.fa = fa; g.out = out;
    g.seg_offsets = groups > 0 ? offsets : nullptr;
    return g;
}

// Threads of the launch of a product's kernel.
static int64_t threads(const Q8Desc& g) {
    int bm = 128, bn = 128, n = 256;
    switch (q4_kernel(g)) {
    case kQ4Rows: bm = bn = 16; n = 512; break;
    case kQ4Small: bm = bn = 64; n = 512; break;
    case kQ4Split: bm = 64; n = 512; break;
    case kQ4Wide: bm = 64; break;
    case kQ4Middle: case kQ4Deep: break;
    case kQ4Large:
        bn = 256;
        if (g.fa == kQ8E2M1 && g.out == kQ8OutBf16) { bm = 256; n = 512; }
    }
    const int64_t tiles = ((g.M + bm - 1) / bm + g.nseg) * ((g.N + bn - 1) / bn);
    return (tiles + 7) / 8 * 8 * n;
}

// No product is taken whose launch passes 2^32 threads.
static void launch() {
    const int64_t top = (int64_t{1} << 31) - 1;
    expect(q4_launch_fits(top - 128 * 40, 128, 0), "rows", top - 128 * 40, 128);
    expect(!q4_launch_fits(top, 1, 64), "rows", top, 64);
    expect(!q4_launch_fits(top, 129, 0), "columns", 129, 0);
    expect(!q4_launch_fits(int64_t{1} << 23, 65536, 0), "columns", 65536, 0);
    for (int fa : {kQ8E4M3, kQ8E2M1})
        for (int out : {kQ8OutF32, kQ8OutBf16, kQ8OutE4M3, kQ8OutE2M1})
            for (int K : {32, 512, 1024, 65536})
                for (int groups : {0, 1, 7, 64})
                    for (int N : {1, 16, 128, 129, 256, 384, 385, 1000, 65536}) {
                        int64_t lo = 0, hi = top;        // the most rows that are taken
                        while (lo < hi) {
                            const int64_t mid = lo + (hi - lo + 1) / 2;
                            if (q4_launch_fits(mid, N, groups)) lo = mid;
                            else hi = mid - 1;
                        }
                        for (int64_t M = lo; M > 0; M = M * 3 / 4) {
                            const int64_t n = threads(desc(M, N, K, groups, fa, out));
                            expect(n < (int64_t{1} << 32), "threads of a launch", M, N);
                        }
                    }
}

// Products in two launches: whole tiles of rows first, neither part cut again,
// and each row in one of them.
static void rounds() {
    int cut = 0;
    for (int fa : {kQ8E4M3, kQ8E2M1})
        for (int out : {kQ8OutF32, kQ8OutBf16, kQ8OutE4M3, kQ8OutE2M1})
            for (int K : {32, 544, 2048, 65536})
                for (int groups : {0, 3})
                    for (int N : {1, 256, 384, 1000, 4096, 65536})
                        for (int64_t M = 1; M < int64_t{1} << 31; M += M / 7 + 1) {
                            Q8Desc g = desc(M, N, K, groups, fa, out);
                            const int64_t rows = q4_whole_rows(g);
                            if (rows == M) continue;
                            ++cut;
                            expect(fa == kQ8E2M1 && out == kQ8OutBf16 && groups == 0, "cut", M, N);
                            expect(rows > 0 && rows < M && rows % 256 == 0, "rows", M, rows);
                            expect((M - rows + 255) / 256 * ((N + 255) / 256) <= 128, "the rest", M, rows);
                            g.M = rows;
                            expect(q4_whole_rows(g) == rows && q4_launch_fits(rows, N, 0) >= q4_launch_fits(M, N, 0),
                                   "first", M, rows);
                            g.M = M - rows;
                            expect(q4_whole_rows(g) == g.M, "rest", M, rows);
                        }
    expect(cut > 100, "cut products", cut, 0);
}

// The kernel of each product M N K groups fa out (as q8.h numbers them).
static void kernels(int n, char** v) {
    for (int i = 0; i + 5 < n; i += 6)
        std::printf("%s\n", kNames[q4_kernel(desc(std::atol(v[i]), std::atoi(v[i + 1]), std::atoi(v[i + 2]),
                                                  std::atoi(v[i + 3]), std::atoi(v[i + 4]), std::atoi(v[i + 5])))]);
}

int main(int argc, char** argv) {
    if (argc < 2) return 2;
    if (std::strcmp(argv[1], "launch") == 0) launch();
    else if (std::strcmp(argv[1], "rounds") == 0) rounds();
    else if (std::strcmp(argv[1], "whole") == 0)
        for (int i = 2; i + 2 < argc; i += 3)
            std::printf("%ld\n", static_cast<long>(q4_whole_rows(
                                     desc(std::atol(argv[i]), std::atoi(argv[i + 1]), std::atoi(argv[i + 2]), 0, kQ8E2M1,
                                          kQ8OutBf16))));
    else if (std::strcmp(argv[1], "kernels") == 0) kernels(argc - 2, argv + 2);
    else return 2;
    return g_bad != 0;
}
