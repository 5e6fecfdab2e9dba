// Checks of the 8-bit products' host-side and index rules on the CPU, run by
// test_gemm_q8_host.py.  Prints each violation; exits with 1 if any.
#include <cstdint>
#include <cstdio>
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

int main(int argc, char** argv) {
    if (argc < 2) return 2;
    if (std::strcmp(argv[1], "row_tiles") == 0) row_tiles();
    else return 2;
    return g_bad != 0;
}
