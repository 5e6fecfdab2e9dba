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
#include "gemm_tile.h"
#include "q8.h"

namespace clearmoe {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// A few rows: 16 rows x 16 columns (or x 128 for an 8-bit result, whose
// scales need whole blocks), operands straight from memory into registers.
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
// The scale a byte stands for.
__device__ __forceinline__ float q8_scale(uint32_t b) {
    return b == 0 ? 0x1p-127f : b == 255 ? __builtin_nanf("") : __uint_as_float(b << 23);
}

// CW waves side by side along the columns, KW sharing the sum; WIDE: float32
// results.
template <int FA, int FB, int CW, int KW, bool WIDE>
__global__ __launch_bounds__(64 * CW * KW) void k_q8_rows(Q8Desc g, int mtiles, int ntiles) {
    constexpr int BM = 16, BN = 16 * CW, PITCH = BN + 4;
    __shared__ float s_acc[KW][BM][PITCH];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, 1, lane, t)) return;
    const int n0 = t.nt * BN, cw = wave % CW, kw = wave / CW;
    const uint8_t* B = g.B + t.seg * g.b_seg_stride;
    const int n = n0 + cw * 16 + row;
    const bool mok = row < t.rows, nok = n < g.N;
    const uint8_t* ar = g.A + (t.m_lo + (mok ? row : 0)) * g.lda;
    const uint8_t* br = B + static_cast<int64_t>(nok ? n : 0) * g.K;
    const uint8_t* sa = g.SA + (t.m_lo + (mok ? row : 0)) * g.sa_ld;
    // the wave's 16 columns lie in one block
    const uint8_t* sb = g.SB + t.seg * g.sb_seg_stride + (n0 + cw * 16) / kQ8Block * g.sb_ld;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int nk = static_cast<int>(q8_blocks(g.K));
    for (int kb = kw; kb < nk; kb += KW) {
        const i32x8 fa = q8_frag(ar, kb * kQ8Block + grp * 32, g.K, mok);
        const i32x8 fb = q8_frag(br, kb * kQ8Block + grp * 32, g.K, nok);
        if constexpr (WIDE) {
            f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_widen<FB>(fb, i), q8_widen<FA>(fa, i), c, 0, 0, 0);
            // a lane's results are of the row that its A fragment has
            const float ka = q8_scale(sa[kb]), kb_ = q8_scale(sb[kb]);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] += c[v] * ka * kb_;
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc, FB, FA, 0, sb[kb], 0, sa[kb]);
        }
    }
    // result v of a lane: column 4 grp + v of row `row`
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[kw][row][cw * 16 + 4 * grp + v] = acc[v];
    __syncthreads();
    const float* bias = g.bias == nullptr ? nullptr : g.bias + static_cast<int64_t>(t.seg) * g.N;
    auto value = [&](int m, int c) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) v += s_acc[w][m][c];
        if (n0 + c >= g.N) return 0.0f;
        if (bias != nullptr) v += bias[n0 + c];
        return g.gelu ? gelu_erf(v) : v;
    };
    if constexpr (CW == 1) {
        const int m = tid / 16, c = tid % 16;
        if (m < t.rows && n0 + c < g.N) {
            const float v = value(m, c);
            const int64_t at = (t.m_lo + m) * g.ldc + n0 + c;
            if constexpr (WIDE) static_cast<float*>(g.C)[at] = v;
            else static_cast<bf16_bits*>(g.C)[at] = f32_to_bf16(v);
        }
    } else {
        static_assert(CW == 8, "a wave finishes a row of one block");
        const int64_t vcols = q8_cols(g.N), blocks = q8_blocks(g.N);
        for (int m = wave; m < t.rows; m += CW * KW) {
            const int c = 2 * lane;
            const float v0 = value(m, c), v1 = value(m, c + 1);
            float a = fmaxf(q8_mag(v0), q8_mag(v1));
#pragma unroll
            for (int s = 32; s > 0; s >>= 1) a = fmaxf(a, __shfl_xor(a, s));
            const int fmt = g.out == kQ8OutE4M3 ? kQ8E4M3 : kQ8E5M2;
            const int e = q8_exponent(__float_as_uint(a), q8_top_exp(fmt));
            const float k = q8_two_to(-e);
            const uint32_t p = fmt == kQ8E4M3 ? q8_pack4<kQ8E4M3>(v0 * k, v1 * k, 0.0f, 0.0f)
                                              : q8_pack4<kQ8E5M2>(v0 * k, v1 * k, 0.0f, 0.0f);
            if (n0 + c < vcols)
                *reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(g.C) + (t.m_lo + m) * g.ldc + n0 + c) =
                    static_cast<uint16_t>(p);
            if (lane == 0) {
                uint8_t* s = g.SC + (t.m_lo + m) * g.sc_ld;
                s[t.nt] = static_cast<uint8_t>(e + kQ8One);
                if (t.nt == blocks - 1)
                    for (int64_t i = blocks; i < g.sc_ld; ++i) s[i] = kQ8One;
            }
        }
    }
}

template <int FA, int FB, int CW, int KW, bool WIDE>
hipError_t q8_rows(const Q8Desc& g, hipStream_t st) {
    const int64_t mt = (g.M + 15) / 16 + (g.seg_offsets != nullptr ? g.nseg : 0);
    const int64_t nt = (g.N + 16 * CW - 1) / (16 * CW);
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q8_rows<FA, FB, CW, KW, WIDE>, dim3(static_cast<unsigned>(grid)), dim3(64 * CW * KW), 0, st, g,
                  static_cast<int>(mt), static_cast<int>(nt));
    return hipGetLastError();
}

template <int FA, int FB>
hipError_t q8_formats(const Q8Desc& g, hipStream_t st) {
    if (g.out == kQ8OutF32) return q8_rows<FA, FB, 1, 8, true>(g, st);
    if (g.out == kQ8OutBf16) return q8_rows<FA, FB, 1, 8, false>(g, st);
    return q8_rows<FA, FB, 8, 2, false>(g, st);
}

}  // namespace

hipError_t launch_gemm_q8(const Q8Desc& g, hipStream_t st) {
    if (g.M == 0) return hipSuccess;
    if (g.fa == kQ8E4M3) return g.fb == kQ8E4M3 ? q8_formats<kQ8E4M3, kQ8E4M3>(g, st) : q8_formats<kQ8E4M3, kQ8E5M2>(g, st);
    return g.fb == kQ8E4M3 ? q8_formats<kQ8E5M2, kQ8E4M3>(g, st) : q8_formats<kQ8E5M2, kQ8E5M2>(g, st);
}

}  // namespace clearmoe
