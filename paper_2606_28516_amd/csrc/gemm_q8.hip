// Products of 8-bit floating point matrices with a power-of-two scale for each
// block of 128 (q8.h), on CDNA4's scaled matrix instructions: the two scales
// of a block are operands of the instruction, so the sum stays in its float32
// accumulators from the first block to the last and no vector work is spent
// on them.
//
// What those instructions add up exactly (measured): eight products that
// follow each other along k are aligned to the largest of them and cut 14 bits
// below it, before the float32 sum; the rest of the sum keeps 24 bits.  A
// result is 1.5e-5 of its norm away from the exact one on normal data: far
// below the rounding of a bfloat16 (1.7e-3) or 8-bit result, but not what
// float32 promises.  Products with a float32 result therefore widen both
// operands to bfloat16 (exactly) and run on its instructions at half the rate,
// whose sums keep 24 bits, and apply the scales to each block's sum.
#include "q8_tile.h"

namespace clearmoe {

namespace {

// ---------------------------------------------------------------------------
// A few rows: 16 rows x 16 columns, operands straight from memory into
// registers.
// ---------------------------------------------------------------------------
// Bytes [k, k + 32) of a row (zeros from K on): lane group g of four takes
// k = 32 g of a 128-wide block, so four lanes read a whole line of a row.
__device__ __forceinline__ i32x8 q8_frag(const uint8_t* row, int k, int K, bool ok) {
    u32x4 a = {0u, 0u, 0u, 0u}, b = a;
    if (ok && k < K) a = *reinterpret_cast<const u32x4*>(row + k);
    if (ok && k + 16 < K) b = *reinterpret_cast<const u32x4*>(row + k + 16);
    i32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = static_cast<int>(a[i]);
        f[i + 4] = static_cast<int>(b[i]);
    }
    return f;
}

// Bytes 8 i .. 8 i + 7 of a fragment as bfloat16 (every 8-bit value is one).
template <int FMT>
__device__ __forceinline__ bf16x8 q8_widen(const i32x8& f, int i) {
    bf16x8 v;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t u = static_cast<uint32_t>(f[2 * i + w]);
        bf16x2_t lo, hi;
        if constexpr (FMT == kQ8E4M3) {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, true);
        } else {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, 1.0f, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(u, 1.0f, true);
        }
        v[4 * w] = lo[0];
        v[4 * w + 1] = lo[1];
        v[4 * w + 2] = hi[0];
        v[4 * w + 3] = hi[1];
    }
    return v;
}
// acc + c 2^(x - 127) 2^(y - 127): a block's sum c and the scale bytes of its
// operands.  The exponents are added before anything is multiplied: one scale
// may be so large or small that c times it alone leaves float32's range though
// the result is an ordinary number.  Where the two are no normal factor
// together, c's own exponent is moved.  What a result is depends on its own
// scales alone, not on the kernel or on the rows beside it.
__device__ __forceinline__ float q8_add_scaled(float acc, float c, uint32_t x, uint32_t y) {
    const int e = static_cast<int>(x + y) - kQ8One;
    const bool normal = e >= 1 && e <= 254;
    const float by_factor = __builtin_fmaf(c, __uint_as_float(static_cast<uint32_t>(normal ? e : 1) << 23), acc);
    const float r = normal ? by_factor : acc + __builtin_ldexpf(c, e - kQ8One);
    return x == 255u || y == 255u ? __builtin_nanf("") : r;
}

// Eight waves share the sum, since there are few tiles and each waits for its
// own operands (1 x 1536 x 384: 2.9 us).  WIDE: float32 results.
template <int FA, int FB, bool WIDE>
__global__ __launch_bounds__(512) void k_q8_rows(Q8Desc g, int mtiles, int ntiles) {
    constexpr int BM = 16, BN = 16, KW = 8;
    __shared__ float s_acc[KW][BM][BN + 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, 1, lane, t)) return;
    const int n0 = t.nt * BN, n = n0 + row;
    const bool mok = row < t.rows, nok = n < g.N;
    const uint8_t* ar = g.A + (t.m_lo + (mok ? row : 0)) * g.lda;
    const uint8_t* br = g.B + t.seg * g.b_seg_stride + static_cast<int64_t>(nok ? n : 0) * g.K;
    const uint8_t* sa = g.SA + (t.m_lo + (mok ? row : 0)) * g.sa_ld;
    const uint8_t* sb = g.SB + t.seg * g.sb_seg_stride + n0 / kQ8Block * g.sb_ld;     // 16 columns of one block
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int nk = static_cast<int>(q8_blocks(g.K));
    for (int kb = wave; kb < nk; kb += KW) {
        const i32x8 fa = q8_frag(ar, kb * kQ8Block + grp * 32, g.K, mok);
        const i32x8 fb = q8_frag(br, kb * kQ8Block + grp * 32, g.K, nok);
        if constexpr (WIDE) {
            f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_widen<FB>(fb, i), q8_widen<FA>(fa, i), c, 0, 0, 0);
            // (kept in front of what depends on a lane's scales: all lanes take
            // part in a matrix instruction)
            asm volatile("" : "+v"(c));
            // a lane's results are of the row that its A fragment has
            const uint32_t x = sa[kb], y = sb[kb];
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] = q8_add_scaled(acc[v], c[v], x, y);
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc, FB, FA, 0, sb[kb], 0, sa[kb]);
        }
    }
    // result v of a lane: column 4 grp + v of row `row`
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[wave][row][4 * grp + v] = acc[v];
    __syncthreads();
    const int m = tid / BN, c = tid % BN;
    if (m < t.rows && n0 + c < g.N) {
        float v = g.bias != nullptr ? g.bias[static_cast<int64_t>(t.seg) * g.N + n0 + c] : 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) v += s_acc[w][m][c];
        if (g.gelu) v = gelu_erf(v);
        const int64_t at = (t.m_lo + m) * g.ldc + n0 + c;
        if constexpr (WIDE) static_cast<float*>(g.C)[at] = v;
        else static_cast<bf16_bits*>(g.C)[at] = f32_to_bf16(v);
    }
}

template <int FA, int FB, bool WIDE>
hipError_t q8_rows(const Q8Desc& g, hipStream_t st) {
    const int64_t mt = (g.M + 15) / 16 + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + 15) / 16;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q8_rows<FA, FB, WIDE>, dim3(static_cast<unsigned>(grid)), dim3(512), 0, st, g,
                  static_cast<int>(mt), static_cast<int>(nt));
    return hipGetLastError();
}

// A few rows of float32 or bfloat16, quantised by every workgroup for itself
// into LDS (rows of `pitch` bytes, then rows of nk scale bytes), then as
// k_q8_rows.  The first blocks of B are on their way meanwhile, so a call is
// two trips to memory at most, which is what bounds it: 1 x 3072 x 768 takes
// 4.4 us under a profiler and 1 x 768 x 3072 5.1, where an empty kernel takes
// 2.3 to 2.8 and the weights' bytes 0.5.
template <typename TA, typename TC>
__global__ __launch_bounds__(512) void k_q8_few(Q8Desc g, const TA* A, int K0, int mtiles, int ntiles, int pitch) {
    constexpr int BM = 16, BN = 16, KW = 8, AHEAD = 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char s_a[];
    __shared__ float s_acc[KW][BM][BN + 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, 1, lane, t)) return;
    const int n0 = t.nt * BN, n = n0 + row, nk = static_cast<int>(q8_blocks(g.K));
    const bool nok = n < g.N, mok = row < t.rows;
    const uint8_t* br = g.B + t.seg * g.b_seg_stride + static_cast<int64_t>(nok ? n : 0) * g.K;
    const uint8_t* sb = g.SB + t.seg * g.sb_seg_stride + n0 / kQ8Block * g.sb_ld;
    i32x8 fb[AHEAD];
    int kb_scale[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int kb = wave + i * KW;
        fb[i] = q8_frag(br, kb * kQ8Block + grp * 32, g.K, nok);
        kb_scale[i] = sb[kb < nk ? kb : 0];
    }
    // 16 lanes a block of 128 columns
    unsigned char* s_sa = s_a + t.rows * pitch;
    for (int u = tid / kQ8Lanes; u < t.rows * nk; u += 512 / kQ8Lanes) {
        const int m = u / nk, blk = u - m * nk, sub = tid % kQ8Lanes;
        float f[8];
        q8_load8(A + (t.m_lo + m) * K0, blk * kQ8Block + sub * 8, K0, f);
        const float a = q8_max16(q8_mag8(f));
        const int e = q8_exponent(__float_as_uint(a), q8_top_exp(kQ8E4M3));
        *reinterpret_cast<uint2*>(s_a + m * pitch + blk * kQ8Block + sub * 8) = q8_pack8<kQ8E4M3>(f, q8_two_to(-e));
        if (sub == 0) s_sa[m * nk + blk] = static_cast<unsigned char>(e + kQ8One);
    }
    __syncthreads();
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto step = [&](int kb, const i32x8& b, int scale) {
        const unsigned char* p = s_a + (mok ? row : 0) * pitch + kb * kQ8Block + grp * 32;
        i32x8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = mok ? reinterpret_cast<const int*>(p)[i] : 0;
        const int sa = s_sa[(mok ? row : 0) * nk + kb];
        if constexpr (sizeof(TC) == 4) {
            // float32 results: as in k_q8_rows
            f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_widen<kQ8E4M3>(b, i), q8_widen<kQ8E4M3>(a, i), c, 0, 0, 0);
            asm volatile("" : "+v"(c));
#pragma unroll
            for (int v = 0; v < 4; ++v)
                acc[v] = q8_add_scaled(acc[v], c[v], static_cast<uint32_t>(sa), static_cast<uint32_t>(scale));
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, kQ8E4M3, kQ8E4M3, 0, scale, 0, sa);
        }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * KW < nk) step(wave + i * KW, fb[i], kb_scale[i]);
    for (int kb = wave + AHEAD * KW; kb < nk; kb += KW)
        step(kb, q8_frag(br, kb * kQ8Block + grp * 32, g.K, nok), sb[kb]);
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[wave][row][4 * grp + v] = acc[v];
    __syncthreads();
    const int m = tid / BN, c = tid % BN;
    if (m < t.rows && n0 + c < g.N) {
        float v = g.bias != nullptr ? g.bias[static_cast<int64_t>(t.seg) * g.N + n0 + c] : 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) v += s_acc[w][m][c];
        if (g.gelu) v = gelu_erf(v);
        static_cast<TC*>(g.C)[(t.m_lo + m) * g.ldc + n0 + c] = Elem<TC>::from_f32(v);
    }
}

template <typename TA, typename TC>
hipError_t q8_few(const Q8Desc& g, const void* A, int K0, hipStream_t st) {
    const int64_t mt = (g.M + 15) / 16 + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + 15) / 16;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    const int nk = static_cast<int>(q8_blocks(g.K)), pitch = nk * kQ8Block + 16;
    const int rows = g.M < 16 ? static_cast<int>(g.M) : 16;
    launch_kernel(k_q8_few<TA, TC>, dim3(static_cast<unsigned>(grid)), dim3(512),
                  static_cast<size_t>(rows) * (pitch + nk), st, g, static_cast<const TA*>(A), K0,
                  static_cast<int>(mt), static_cast<int>(nt), pitch);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Many rows: tiles through LDS.
// ---------------------------------------------------------------------------
// 32 bytes of a stage row in LDS: a stage is 128 bytes (one scale block) of k,
// so a stage row is a whole line and its scale one byte.
__device__ __forceinline__ i32x8 q8_lds_frag(const unsigned char* p, uint32_t off) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p + off), b = *reinterpret_cast<const u32x4*>(p + (off ^ 16u));
    i32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = static_cast<int>(a[i]);
        f[i + 4] = static_cast<int>(b[i]);
    }
    return f;
}

// 256 x 128 tile over four waves (64 x 128 each), two workgroups on a CU, so
// that one's epilogue runs beside the other's matrix instructions.  80 KB of
// LDS each: A has two stage buffers, B one, which is free as soon as its
// fragments are in registers.  Measured on an MI355X, calls in a row (and under
// a profiler, the first ones): 50432 x 768 x 3072 to bfloat16 118 us (142),
// 2020 TFLOP/s, 50432 x 3072 x 768 with GELU to e4m3 157 (198), 8192 x 8192 x
// 8192 440 (482), 2500 TFLOP/s; the library's large 8-bit product: 3065.  With
// few stages (k = 384, 768) the epilogue's vector work and stores bound it;
// over many, LDS does: 192 KB of fragments and 96 KB of new bytes a stage and
// CU take longer than its 2048 cycles of instructions.
// 256 x 256 tiles over eight waves, a grid that stays on the chip and takes
// tile after tile, and fetching B earlier were no faster.
template <int FA, int FB, int OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_q8_duo(Q8Desc g, int mtiles, int ntiles, int group) {
    constexpr int SB = kGbRow, BM = 256, BN = kQ8Block, CPR = 8, BK = kQ8Block, TM = 2, TN = 4, AL = 8, BL = 4;
    constexpr int ABUF = BM * SB, BOFF = 2 * ABUF;      // buffers A0 A1 B
    __shared__ __attribute__((aligned(1024))) unsigned char smem[BOFF + BN * SB];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lrow = lane & 31, lh = lane >> 5;

    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, group, lane, t)) return;
    const int n0 = t.nt * BN, K = g.K;
    const int lr = lane / CPR, cp = lane % CPR;
    // first k of the lane's chunk in an even load's 8 rows; odd: ^ 64
    const int kc0 = 16 * (cp ^ (lr >> 1));
    const gb_i32x4 da = gb_desc(g.A + t.m_lo * g.lda, (static_cast<int64_t>(t.rows) - 1) * g.lda + K);
    const int nrows = g.N - n0 < BN ? g.N - n0 : BN;
    const gb_i32x4 db = gb_desc(g.B + t.seg * g.b_seg_stride + static_cast<int64_t>(n0) * K,
                                static_cast<int64_t>(nrows) * K);
    // Load i brings the rows 8 i + lr of the wave.  Kept are the byte offsets
    // of the first even and odd one, to which i adds whole rows; rows past the
    // tile's lie past the descriptor's end and read zeros.  Of the last stage
    // of a k that ends inside it, chunks past the end get an offset past
    // everything.
    const uint32_t lda = static_cast<uint32_t>(g.lda);
    const int nk = static_cast<int>(q8_blocks(K)), left = K - (nk - 1) * BK;
    uint32_t va[2], vb[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        va[p] = static_cast<uint32_t>(wave * AL * 8 + lr) * lda + (kc0 ^ (64 * p));
        vb[p] = static_cast<uint32_t>((wave * BL * 8 + lr) * K + (kc0 ^ (64 * p)));
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((gb_lds_u32*)smem)));
    auto first = [&](const uint32_t (&v)[2], int kt, int p) {
        return kt == nk - 1 && (kc0 ^ (64 * p)) >= left ? kGbOob : v[p];
    };
    auto dma_a = [&](int kt, int b) {
        const uint32_t v[2] = {first(va, kt, 0), first(va, kt, 1)};
#pragma unroll
        for (int i = 0; i < AL; ++i)
            gb_dma16(da, v[i & 1] + static_cast<uint32_t>(8 * i) * lda, __builtin_amdgcn_readfirstlane(kt * BK),
                     __builtin_amdgcn_readfirstlane(lds0 + b * ABUF + (wave * AL + i) * 1024));
    };
    auto dma_b = [&](int kt) {
        const uint32_t v[2] = {first(vb, kt, 0), first(vb, kt, 1)};
#pragma unroll
        for (int i = 0; i < BL; ++i)
            gb_dma16(db, v[i & 1] + static_cast<uint32_t>(8 * i * K), __builtin_amdgcn_readfirstlane(kt * BK),
                     __builtin_amdgcn_readfirstlane(lds0 + BOFF + (wave * BL + i) * 1024));
    };
    // scales: a word holds those of four stages (rows past the tile's: 0)
    const __amdgpu_buffer_rsrc_t ra = raw_rsrc(g.SA + t.m_lo * g.sa_ld, static_cast<int64_t>(t.rows) * g.sa_ld);
    const uint32_t vs = static_cast<uint32_t>(wave * 64 + lrow) * static_cast<uint32_t>(g.sa_ld);
    const uint8_t* psb = g.SB + t.seg * g.sb_seg_stride + static_cast<int64_t>(t.nt) * g.sb_ld;
    uint32_t sa[TM], sb;
    auto scales = [&](int kt) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
            sa[i] = static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b32(
                ra, static_cast<int>(vs + static_cast<uint32_t>(i * 32) * static_cast<uint32_t>(g.sa_ld)), kt, 0));
        sb = *reinterpret_cast<const uint32_t*>(psb + kt);
    };
    scales(0);
    dma_a(0, 0);
    dma_b(0);
    f32x16 acc[TM][TN];
    // (through the second buffer of A, which is filled after the first wait)
    if (g.bias != nullptr) {
        q8_bias_load<TN>(g, t.seg, n0, lane, smem + ABUF + wave * 512);
        q8_start(lane, smem + ABUF + wave * 512, acc);
    } else {
        gb_zero(acc);
    }

    const int bcol = gb_col_of_slot(lrow);
    uint32_t oa[2], ob[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        oa[s] = static_cast<uint32_t>((wave * 64 + lrow) * SB + (((4 * s + 2 * lh) ^ gb_swz<SB>(lrow)) << 4));
        ob[s] = static_cast<uint32_t>(BOFF + bcol * SB + (((4 * s + 2 * lh) ^ gb_swz<SB>(bcol)) << 4));
    }
    i32x8 fa[2][TM], fb[2][TN];
    auto read_a = [&](int b, int s) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[s][i] = q8_lds_frag(smem + b * ABUF + i * 32 * SB, oa[s]);
    };
    auto read_b = [&](int s) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[s][j] = q8_lds_frag(smem + j * 32 * SB, ob[s]);
    };
    auto mm = [&](int s, int kt) {
        const int sh = 8 * (kt & 3);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                    fb[s][j], fa[s][i], acc[i][j], FB, FA, 0, static_cast<int>(sb >> sh), 0,
                    static_cast<int>(sa[i] >> sh));
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int k0 = 0; k0 < nk; k0 += 2) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int kt = k0 + b;
            if (kt >= nk) break;
            // stage kt has landed for every wave, and every wave is done
            // reading the other A buffer
            gb_wait_barrier<0>();
            if ((kt & 3) == 0) {
                // the words of these four stages have landed too: take them
                // before the next loads are issued, so that nothing waits
                // for those
#pragma unroll
                for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(sa[i]));
            }
            if (kt + 1 < nk) dma_a(kt + 1, b ^ 1);
            read_b(0);
            read_a(b, 0);
            read_b(1);
            mm(0, kt);
            if (kt + 1 < nk) {
                // every wave has read this stage's B
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                dma_b(kt + 1);
            }
            read_a(b, 1);
            mm(1, kt);
            if ((kt & 3) == 3 && kt + 1 < nk) scales(kt + 1);
        }
    }
    gb_wait_barrier<0>();                        // the stage buffers are free
    q8_epilogue<TM, TN, OUT, BM, false>(g, t, wave * 64, n0, 0, lane, smem + wave * (32 * 256), nullptr, acc);
}

// KG groups of WM x WN waves of TM x TN MFMA tiles (32 x 32), NS stages in LDS
// for each: of a stage the loads are issued NS - 1 stages ahead.  Every
// stage's loads end with the scale words of its rows and columns.  The groups
// take the stages in turn and their sums are added at the end: a workgroup
// that is alone on its CU waits for one stage after the other, with two groups
// for half as many (512 x 768 x 3072, 64 x 64 tiles: one group 10.3 us, two
// 8.6, four 8.8; float32 17.6, 13.1, 12.5; more stages ahead change nothing).
// WIDE: float32 results, on bfloat16 instructions (see above): eight a stage
// that wait for each other, their operands widened just before, which is what
// float32 takes longer here.
template <int KG, int WM, int WN, int TM, int TN, int NS, int FA, int FB, int OUT>
__global__ __launch_bounds__(64 * KG * WM * WN) void k_q8_tile(Q8Desc g, int mtiles, int ntiles, int group) {
    constexpr bool WIDE = OUT == kQ8OutF32;
    constexpr int NW = WM * WN, SB = kGbRow, BM = WM * TM * 32, BN = WN * TN * 32, CPR = 8, BK = kQ8Block;
    constexpr int AL = BM / (8 * NW), BL = BN / (8 * NW), LPS = AL + BL + 1;
    static_assert(AL >= 1 && BL >= 1 && BM % 64 == 0 && BN % 64 == 0 && BM + BN <= 64 * NW, "whole loads per wave");
    static_assert(NS % 2 == 0 && LPS * (NS - 1) < 64, "pipeline");
    static_assert(kQ8Block % (TN * 32) == 0 && (OUT == kQ8OutF32 || OUT == kQ8OutBf16 || BN % kQ8Block == 0),
                  "a wave's columns lie in one block, an 8-bit tile has whole blocks");
    static_assert(KG == 1 || OUT == kQ8OutF32 || OUT == kQ8OutBf16, "the 8-bit epilogue has a barrier for all waves");
    constexpr int STAGE_A = BM * SB, STAGE = (BM + BN) * SB, SOFF = NS * STAGE, SSTAGE = 256 * NW;
    constexpr int EPI = NW * 32 * TN * 32 * (OUT == kQ8OutF32 ? 4 : OUT == kQ8OutBf16 ? 2 : 1);
    constexpr int SSIZE = NS * SSTAGE > WN * BM * 4 ? NS * SSTAGE : WN * BM * 4;
    constexpr int GROUP = SOFF + SSIZE, SUMS = NW * 64 * TM * TN * 64;
    static_assert(SOFF >= EPI && (KG == 1 || SOFF >= SUMS), "the epilogue's rows and the sums fit the stages");
    __shared__ __attribute__((aligned(1024))) unsigned char smem_all[KG * GROUP + NW * 256];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave_all / NW, wave = wave_all % NW;
    unsigned char* smem = smem_all + kg * GROUP;
    const int wm = wave / WN, wn = wave % WN;
    const int lrow = lane & 31, lh = lane >> 5, K = g.K;

    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, group, lane, t)) return;
    const int n0 = t.nt * BN;
    const int nk = static_cast<int>(q8_blocks(K)), left = K - (nk - 1) * BK;
    const int steps = (nk + KG - 1) / KG;        // stage kg + KG * step is the group's
    const int lr = lane / CPR;
    // first k of the lane's chunk in an even load's 8 rows; odd: ^ 64
    const int kc0 = 16 * ((lane % CPR) ^ (lr >> 1));
    const uint32_t lda = static_cast<uint32_t>(g.lda);
    const int nrows = g.N - n0 < BN ? g.N - n0 : BN;
    const gb_i32x4 da = gb_desc(g.A + t.m_lo * g.lda, (static_cast<int64_t>(t.rows) - 1) * g.lda + K);
    const gb_i32x4 db = gb_desc(g.B + t.seg * g.b_seg_stride + static_cast<int64_t>(n0) * K,
                                static_cast<int64_t>(nrows) * K);
    // scale words: the first BM / 64 waves fetch those of the rows, the next
    // BN / 64 those of the columns (each its block's)
    const int sr = wave * 64 + lane;
    const bool s_row = wave < BM / 64;
    const gb_i32x4 ds = s_row ? gb_desc(g.SA + t.m_lo * g.sa_ld, static_cast<int64_t>(t.rows) * g.sa_ld)
                              : gb_desc(g.SB + t.seg * g.sb_seg_stride, q8_blocks(g.N) * g.sb_ld);
    const uint32_t vs = s_row ? (sr < t.rows ? static_cast<uint32_t>(sr) * static_cast<uint32_t>(g.sa_ld) : kGbOob)
                              : (sr - BM < BN ? static_cast<uint32_t>((n0 + sr - BM) / kQ8Block) *
                                                    static_cast<uint32_t>(g.sb_ld)
                                              : kGbOob);
    // Load i of a wave brings the rows 8 i + lr from its first one on.  Row r
    // of LDS has its chunk c at c ^ (r / 2 % 8), which for the rows of a load
    // depends on whether it is an even or odd one of the tile.
    constexpr int PA = AL > 1 ? 2 : 1, PB = BL > 1 ? 2 : 1;
    const int oddA = AL == 1 ? wave & 1 : 0, oddB = BL == 1 ? wave & 1 : 0;
    uint32_t va[PA], vb[PB];
    int ka[PA], kb[PB];
#pragma unroll
    for (int p = 0; p < PA; ++p) {
        ka[p] = kc0 ^ (64 * ((p + oddA) & 1));
        va[p] = static_cast<uint32_t>(wave * AL * 8 + lr) * lda + static_cast<uint32_t>(ka[p]);
    }
#pragma unroll
    for (int p = 0; p < PB; ++p) {
        kb[p] = kc0 ^ (64 * ((p + oddB) & 1));
        vb[p] = static_cast<uint32_t>((wave * BL * 8 + lr) * K + kb[p]);
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((gb_lds_u32*)smem)));
    // Stages past the last are issued too (zeros, no memory traffic), so that
    // every wait below counts the same.  Rows past the tile's lie past the
    // descriptor's end.
    auto dma = [&](int step, int b) {
        const int kt = step * KG + kg;
        const bool past = kt >= nk;
        const int soff = __builtin_amdgcn_readfirstlane(past ? 0 : kt * BK);
#pragma unroll
        for (int i = 0; i < AL; ++i) {
            const int p = i % PA;
            const uint32_t v = past || (kt == nk - 1 && ka[p] >= left) ? kGbOob : va[p];
            gb_dma16(da, v + static_cast<uint32_t>(8 * i) * lda, soff,
                     __builtin_amdgcn_readfirstlane(lds0 + b * STAGE + (wave * AL + i) * 1024));
        }
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int p = i % PB;
            const uint32_t v = past || (kt == nk - 1 && kb[p] >= left) ? kGbOob : vb[p];
            gb_dma16(db, v + static_cast<uint32_t>(8 * i * K), soff,
                     __builtin_amdgcn_readfirstlane(lds0 + b * STAGE + STAGE_A + (wave * BL + i) * 1024));
        }
        gb_dma4(ds, past ? kGbOob : vs, __builtin_amdgcn_readfirstlane(past ? 0 : (kt & ~3)),
                __builtin_amdgcn_readfirstlane(lds0 + SOFF + b * SSTAGE + wave * 256));
    };
    // (a word a lane: 256 bytes)
    const uint32_t boff = KG * GROUP + wave * 256;
    if (g.bias != nullptr && kg == 0) q8_bias_dma<TN>(g, t.seg, n0 + wn * TN * 32, lane, lds0 + boff);
#pragma unroll
    for (int s = 0; s < NS; ++s) dma(s, s);

    const int bcol = gb_col_of_slot(lrow);
    uint32_t oa[2], ob[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        oa[s] = static_cast<uint32_t>((wm * TM * 32 + lrow) * SB + (((4 * s + 2 * lh) ^ gb_swz<SB>(lrow)) << 4));
        ob[s] = static_cast<uint32_t>(STAGE_A + (wn * TN * 32 + bcol) * SB +
                                      (((4 * s + 2 * lh) ^ gb_swz<SB>(bcol)) << 4));
    }
    i32x8 fa[2][TM], fb[2][TN];
    uint32_t sa[2][TM], sb[2];                   // by the stage's parity
    auto read = [&](int b, int s) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[s][j] = q8_lds_frag(smem + b * STAGE + j * 32 * SB, ob[s]);
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[s][i] = q8_lds_frag(smem + b * STAGE + i * 32 * SB, oa[s]);
    };
    auto read_scales = [&](int step, int b) {
        const int sh = 8 * ((step * KG + kg) & 3);
        const uint32_t* p = reinterpret_cast<const uint32_t*>(smem + SOFF + b * SSTAGE);
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[b & 1][i] = p[wm * TM * 32 + i * 32 + lrow] >> sh;
        sb[b & 1] = p[BM + wn * TN * 32] >> sh;   // one block
    };
    gb_wait_barrier<(NS - 1) * LPS>();           // the bias and stage 0 have landed
    f32x16 acc[TM][TN];
    if (g.bias != nullptr && kg == 0) q8_start(lane, smem_all + boff, acc);
    else gb_zero(acc);
    read(0, 0);
    read_scales(0, 0);
    f32x16 part[WIDE ? TM : 1][WIDE ? TN : 1];
    for (int k0 = 0; k0 < steps; k0 += NS) {
#pragma unroll
        for (int b = 0; b < NS; ++b) {
            const int kt = k0 + b;
            if (kt >= steps) break;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s == 0) {
                    read(b, 1);
                } else if (kt + 1 < steps) {
                    // stage kt + 1 has landed for every wave, and every wave
                    // is done reading stage kt's buffer, which takes kt + NS
                    gb_wait_barrier<(NS - 2) * LPS>();
                    read((b + 1) % NS, 0);
                    read_scales(kt + 1, (b + 1) % NS);
                    dma(kt + NS, b);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        if constexpr (WIDE) {
                            f32x16& c = part[i][j];
                            if (s == 0)
#pragma unroll
                                for (int v = 0; v < 16; ++v) c[v] = 0.0f;
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q8_widen<FB>(fb[s][j], q),
                                                                            q8_widen<FA>(fa[s][i], q), c, 0, 0, 0);
                            // a lane's results are of the row that its A
                            // fragment has; one factor for both scales unless
                            // it is no normal number
                            if (s == 1) {
                                const uint32_t x = sa[b & 1][i] & 255u, y = sb[b & 1] & 255u;
                                const int e = static_cast<int>(x + y) - 127;
                                if (__ballot(e < 1 || e > 254 || x == 255u || y == 255u) == 0) {
                                    const float f = __uint_as_float(static_cast<uint32_t>(e) << 23);
#pragma unroll
                                    for (int v = 0; v < 16; ++v) acc[i][j][v] = __builtin_fmaf(c[v], f, acc[i][j][v]);
                                } else {
#pragma unroll
                                    for (int v = 0; v < 16; ++v) acc[i][j][v] = q8_add_scaled(acc[i][j][v], c[v], x, y);
                                }
                            }
                        } else {
                            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                                fb[s][j], fa[s][i], acc[i][j], FB, FA, 0, static_cast<int>(sb[b & 1]), 0,
                                static_cast<int>(sa[b & 1][i]));
                        }
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    gb_wait_barrier<0>();                        // the stage buffers are free
    if constexpr (KG > 1) {
        // the groups' sums, in order, through their own buffers
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<f32x4*>(smem + (((wave * TM + i) * TN + j) * 4 + q) * 1024 + lane * 16) =
                            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int o = 1; o < KG; ++o)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 v = *reinterpret_cast<const f32x4*>(
                            smem + o * GROUP + (((wave * TM + i) * TN + j) * 4 + q) * 1024 + lane * 16);
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[i][j][4 * q + c] += v[c];
                    }
    }
    q8_epilogue<TM, TN, OUT, BM, false>(g, t, wm * TM * 32, n0 + wn * TN * 32, wn, lane, smem + wave * (EPI / NW),
                                 reinterpret_cast<float*>(smem + SOFF), acc);
}

// Row tiles that are taken column tile by column tile on one XCD (gb_tile; 1
// to 16 measure the same, and so do stores past the L2).
constexpr int kQ8Group = 4;

template <int FA, int FB, int OUT>
hipError_t q8_duo(const Q8Desc& g, hipStream_t st) {
    const int64_t mt = (g.M + 255) / 256 + (g.seg_offsets != nullptr ? g.nseg : 0);
    const int64_t nt = q8_blocks(g.N);
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q8_duo<FA, FB, OUT>, dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, g,
                  static_cast<int>(mt), static_cast<int>(nt), kQ8Group);
    return hipGetLastError();
}

template <int KG, int WM, int WN, int TM, int TN, int NS, int FA, int FB, int OUT>
hipError_t q8_tile(const Q8Desc& g, hipStream_t st) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    const int64_t mt = (g.M + BM - 1) / BM + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + BN - 1) / BN;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q8_tile<KG, WM, WN, TM, TN, NS, FA, FB, OUT>, dim3(static_cast<unsigned>(grid)), dim3(64 * KG * WM * WN), 0,
                  st, g, static_cast<int>(mt), static_cast<int>(nt), kQ8Group);
    return hipGetLastError();
}

// Tiles of bm x bn of a product; a group ends inside a tile: half a tile more.
int64_t q8_tiles(const Q8Desc& g, int bm, int bn) {
    const int64_t groups = g.seg_offsets != nullptr ? g.nseg : 0;
    return ((g.M + bm - 1) / bm + groups / 2) * ((g.N + bn - 1) / bn);
}

// Which kernel: by the number of tiles, that is by how well each fills the
// chip.  Times in us on an MI355X, N x K of 768 x 3072 and 384 x 1536 to
// bfloat16 and float32, 3072 x 768 and 1536 x 384 with GELU to 8 bits:
//                    rows of A   128        1024         4096         16384
//   bfloat16  16 x 16 (rows)   8.6  4.5  38.0  11.8   141   39
//             64 x 64          8.4  6.0   9.0   6.3    22.9  9.1     80   24
//             128 x 128       15.6  9.7  16.5  10.1    19.1 10.8     56   22
//             256 x 128 (duo) 28.3 16.3  29.4  16.7    32.9 17.3     42   21
//   float32   16 x 16          9.4        39.4        143
//             64 x 64         12.7        13.9         32.5
//             256 x 128                                38.3         108
//   8 bits    64 x 128         7.2  6.0   9.6   6.2    25.1 11.9     89   35
//             256 x 128 (duo) 12.8  9.6  13.4  10.0    20.5 11.0     57   25
Q8Kernel q8_choose(const Q8Desc& g) {
    // bytes: two workgroups of 64 x 128 on every CU, or more rows a workgroup
    if (g.out == kQ8OutE4M3 || g.out == kQ8OutE5M2) return q8_tiles(g, 64, 128) <= 512 ? kQ8Small : kQ8Large;
    if (g.out == kQ8OutF32)
        return q8_tiles(g, 16, 16) <= 800 ? kQ8Rows : q8_tiles(g, 64, 64) <= 1024 ? kQ8Small : kQ8Large;
    return q8_tiles(g, 16, 16) <= 400     ? kQ8Rows
           : q8_tiles(g, 64, 64) <= 640   ? kQ8Small
           : q8_tiles(g, 256, 128) < 192  ? kQ8Middle
                                          : kQ8Large;
}

template <int FA, int FB, int OUT>
hipError_t q8_launch(const Q8Desc& g, hipStream_t st) {
    const Q8Kernel kernel = q8_choose(g);
    if constexpr (OUT == kQ8OutE4M3 || OUT == kQ8OutE5M2) {
        return kernel == kQ8Small ? q8_tile<1, 2, 2, 1, 2, 2, FA, FB, OUT>(g, st) : q8_duo<FA, FB, OUT>(g, st);
    } else {
        if (kernel == kQ8Rows) return q8_rows<FA, FB, OUT == kQ8OutF32>(g, st);
        if (kernel == kQ8Small) return q8_tile<2, 2, 2, 1, 1, 2, FA, FB, OUT>(g, st);
        if constexpr (OUT == kQ8OutF32) return q8_tile<1, 4, 2, 2, 2, 2, FA, FB, OUT>(g, st);
        else
            return kernel == kQ8Middle ? q8_tile<1, 4, 2, 1, 2, 4, FA, FB, OUT>(g, st) : q8_duo<FA, FB, OUT>(g, st);
    }
}

template <int FA, int FB>
hipError_t q8_formats(const Q8Desc& g, hipStream_t st) {
    if (g.out == kQ8OutE4M3) return q8_launch<FA, FB, kQ8OutE4M3>(g, st);
    if (g.out == kQ8OutE5M2) return q8_launch<FA, FB, kQ8OutE5M2>(g, st);
    if (g.out == kQ8OutF32) return q8_launch<FA, FB, kQ8OutF32>(g, st);
    return q8_launch<FA, FB, kQ8OutBf16>(g, st);
}

// The LDS that the quantised form of a few rows may take.
constexpr int64_t kQ8FewLds = 48 << 10;

}  // namespace

Q8Kernel q8_kernel(const Q8Desc& g) { return q8_choose(g); }
bool q8_launch_fits(int64_t M, int N, int groups, int out) {
    // 256 x 128 tiles take whatever is large, over 512 threads for float32
    // results and 256 for others (the grid is rounded up to whole XCDs)
    const int64_t threads = out == kQ8OutF32 ? 512 : 256;
    return ((M + 255) / 256 + groups) * q8_blocks(N) <= (int64_t{1} << 32) / threads - kGbXcds;
}
bool q8_few_supported(int64_t M, int64_t K) {
    const int64_t rows = M < 16 ? M : 16;
    return M <= kQ8FewRows && rows * (q8_blocks(K) * (kQ8Block + 1) + 16) <= kQ8FewLds;
}
hipError_t launch_q8_few(const Q8Desc& g, const void* A, bool a_f32, int K0, hipStream_t st) {
    if (g.M == 0) return hipSuccess;
    if (g.out == kQ8OutF32) return a_f32 ? q8_few<float, float>(g, A, K0, st) : q8_few<bf16_bits, float>(g, A, K0, st);
    return a_f32 ? q8_few<float, bf16_bits>(g, A, K0, st) : q8_few<bf16_bits, bf16_bits>(g, A, K0, st);
}

hipError_t launch_gemm_q8(const Q8Desc& g, hipStream_t st) {
    if (g.M == 0) return hipSuccess;
    if (g.fa == kQ8E4M3) return g.fb == kQ8E4M3 ? q8_formats<kQ8E4M3, kQ8E4M3>(g, st) : q8_formats<kQ8E4M3, kQ8E5M2>(g, st);
    return g.fb == kQ8E4M3 ? q8_formats<kQ8E5M2, kQ8E4M3>(g, st) : q8_formats<kQ8E5M2, kQ8E5M2>(g, st);
}

}  // namespace clearmoe
