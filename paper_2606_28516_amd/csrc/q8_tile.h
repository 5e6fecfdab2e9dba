// What the tiled products of 8-bit (gemm_q8.hip) and 4-bit (gemm_q4.hip)
// matrices share: sums that start at the bias, and the epilogue of a wave.
#pragma once

#include "gemm_tile.h"
#include "q8.h"

namespace clearmoe {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// GELU as v Phi(v) = max(v, 0) - |v| Phi(-|v|), which has no cancellation in
// its negative tail, with Phi(-a) = 2^P(a), P a polynomial near log2 Phi(-a).
// Step by step over the values: an exponential's result may not be used by the
// next instruction.
template <int N, int D>
__device__ __forceinline__ void q8_gelu(const float (&v)[N], const float (&P)[D + 1], float (&y)[N]) {
    float p[N], m[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float a = fabsf(v[i]);
        p[i] = P[D];
#pragma unroll
        for (int k = D - 1; k >= 0; --k) p[i] = __builtin_fmaf(a, p[i], P[k]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = __builtin_amdgcn_exp2f(p[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // (fmaxf takes two instructions: it quiets NaN first)
        asm("v_max_f32 %0, 0, %1" : "=v"(m[i]) : "v"(v[i]));
        y[i] = __builtin_fmaf(-fabsf(v[i]), p[i], m[i]);
    }
}

// For results of 8-bit products that are rounded to 8 bits or bfloat16: degree
// 7, nearest on [0, 6] (5.0e-6, so GELU is off by at most 3.5e-6 of itself
// there; further out P falls on without end): 13 full-rate operations' time
// instead of gelu_erf's 20.  fc1 + GELU over many rows is bound by this vector
// work (50432 x 3072 x 768: 199 us with gelu_erf, 141 without any).  An
// infinite v gives NaN, as gelu_erf does.
constexpr float kQ8Gelu[8] = {-9.99995318e-01f, -1.15125091f,    -4.58464246e-01f, -5.39604758e-02f,
                              8.50815862e-03f,  -9.3060248e-04f, 6.16087855e-05f,  -1.83535093e-06f};

// For all results of 4-bit products: degree 9, nearest on [0, 5] with errors
// weighed down from 2 on, and further out (rare: the whole wave looks again,
// each value by its own place) |v| Phi(-|v|) = 2^(-v^2 log2(e) / 2) T(1 / v^2), T
// of degree 3, nearest on [5, 13.25], where float32's normal numbers end.
// What |v| Phi(-|v|) is off by, of itself, evaluated in float32: 3e-7 for |v| up
// to 1, 5.6e-7 to 2, 1.6e-6 to 4, 3.8e-6 to 5 and 8e-6 beyond; what is below
// 2^-126 may be 0.  So a block of small hidden values is rounded to 4 or 8 bits
// from what GELU is, and few of the others fall on the other side of a tie.
// P(0) is -1 itself: sums of 4-bit products lie on a coarse grid, the halves
// that GELU makes of small ones (below 2^-20) are often ties of the result's
// grid, or six times a power of two, and must not be moved off them.  16
// operations' time: 50432 x 4096 x 1024 to 4 bits takes 192 us with sums of unit
// variance (of variance 2, where a third of the waves look again, 203), 183 with
// the polynomial above, 207 with one of degree 14 for the whole range, 153
// without GELU.
constexpr float kQ4Gelu[10] = {-1.0f,            -1.15111232f,     -0.459147573f,   -0.0526642539f,  0.0072750384f,
                               -0.000269470678f, -0.000147616622f, 3.69796508e-05f, -3.90794594e-06f, 1.65017468e-07f};
constexpr float kQ4GeluTail[4] = {0.3989396095f, -0.3982101083f, 1.1313945055f, -3.517411232f};
constexpr float kQ4GeluFar = 5.0f;

template <int N>
__device__ __forceinline__ void q4_gelu(float (&v)[N]) {
    float y[N], most = 0.0f;
    q8_gelu<N, 9>(v, kQ4Gelu, y);
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(v[i]));
    if (__builtin_expect(__ballot(most > kQ4GeluFar) != 0, 0))
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = v[i] * v[i], r = __builtin_amdgcn_rcpf(s);
            float t = kQ4GeluTail[3];
#pragma unroll
            for (int k = 2; k >= 0; --k) t = __builtin_fmaf(r, t, kQ4GeluTail[k]);
            t *= __builtin_amdgcn_exp2f(s * -0.72134752044448170368f);
            // (NaN of an infinite v)
            const float far = __builtin_fmaf(v[i], 0.0f, fmaxf(v[i], 0.0f) - t);
            y[i] = fabsf(v[i]) > kQ4GeluFar ? far : y[i];
        }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = y[i];
}

// Four floats over a scale -> four bytes (as q8_pack4, the division inside).
template <int FMT>
__device__ __forceinline__ uint32_t q8_pack4_over(float a, float b, float c, float d, float scale) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    s16x2 v = {0, 0};
    if constexpr (FMT == kQ8E4M3) {
        v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a, b, scale, false);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale, true);
    } else {
        v = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(v, a, b, scale, false);
        v = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(v, c, d, scale, true);
    }
    return __builtin_bit_cast(uint32_t, v);
}

// Eight floats over a scale -> eight e2m1 values (as q4_pack8, the division
// inside).
__device__ __forceinline__ uint32_t q4_pack8_over(float a, float b, float c, float d, float e, float f, float g,
                                                  float h, float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c, d, scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e, f, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, g, h, scale, 3);
}

// Sums start at the bias, which saves an addition a value at the end.  Its
// values for a wave's 32 TN columns from c are put in the lanes' order through
// 128 TN bytes of the wave's own LDS (wb): here in registers on the way, or
// fetched by q8_bias_dma and waited for by the caller.
__device__ __forceinline__ gb_i32x4 q8_bias_desc(const Q8Desc& g, int seg) {
    return gb_desc(g.bias + static_cast<int64_t>(seg) * g.N, static_cast<int64_t>(g.N) * 4);
}
template <int TN>
__device__ __forceinline__ void q8_bias_dma(const Q8Desc& g, int seg, int c, int lane, uint32_t wb) {
    const gb_i32x4 d = q8_bias_desc(g, seg);
    static_assert(TN <= 2, "a word a lane");
    gb_dma4(d, lane < 32 * TN ? static_cast<uint32_t>(c + lane) * 4u : kGbOob, 0, __builtin_amdgcn_readfirstlane(wb));
}
template <int TN>
__device__ __forceinline__ void q8_bias_load(const Q8Desc& g, int seg, int c, int lane, unsigned char* wb) {
    const __amdgpu_buffer_rsrc_t rb = raw_rsrc(g.bias + static_cast<int64_t>(seg) * g.N, static_cast<int64_t>(g.N) * 4);
#pragma unroll
    for (int h = 0; h < TN / 2; ++h)
        reinterpret_cast<float*>(wb)[h * 64 + lane] =
            __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rb, (c + h * 64 + lane) * 4, 0, 0));
    __builtin_amdgcn_wave_barrier();
}
template <int TM, int TN>
__device__ __forceinline__ void q8_start(int lane, const unsigned char* wb, f32x16 (&acc)[TM][TN]) {
    const int lh = lane >> 5;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const f32x4 b =
                *reinterpret_cast<const f32x4*>(wb + 4 * (j * 32 + 16 * (h >> 1) + 8 * lh + 4 * (h & 1)));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][4 * h + v] = b[v];
        }
    __builtin_amdgcn_wave_barrier();
}

// Epilogue of one wave: 32 TM rows from rw, 32 TN columns from nw.  Lane l
// holds row i * 32 + l % 32 and, for each half h of a tile's 16 values, eight
// consecutive columns (gb_col_of_slot).  Rows are rounded, put together in 32
// rows of this wave's own LDS (wb) and stored as whole row pieces.  For an
// 8-bit result, 128 / (32 TN) waves side by side share a block: they exchange
// the rows' maxima through s_max [waves side by side][BM], between barriers
// that all waves of the workgroup take.  Q4: the product is a 4-bit one.
template <int TM, int TN, int OUT, int BM, bool Q4>
__device__ __forceinline__ void q8_epilogue(const Q8Desc& g, const GbTile& t, int rw, int nw, int wn, int lane,
                                            unsigned char* wb, float* s_max, f32x16 (&acc)[TM][TN]) {
    constexpr bool F32 = OUT == kQ8OutF32, BF16 = OUT == kQ8OutBf16, E2M1 = OUT == kQ8OutE2M1;
    constexpr int FMT = OUT == kQ8OutE4M3 ? kQ8E4M3 : kQ8E5M2;
    constexpr int RB = E2M1 ? TN * 16 : TN * 32 * (F32 ? 4 : BF16 ? 2 : 1), CH = RB / 16, RPI = 64 / CH > 32 ? 32 : 64 / CH;
    constexpr int SHARE = 4 / TN;
    static_assert(RB >= 16 && 64 % CH == 0 && 32 % RPI == 0, "whole rows per store");
    const int lrow = lane & 31, lh = lane >> 5;
    const int cols = static_cast<int>(q8_cols(g.N));
    if (g.gelu)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; v += Q4 ? 16 : 4) {
                    constexpr int STEP = Q4 ? 16 : 4;
                    float x[STEP], y[STEP];
#pragma unroll
                    for (int c = 0; c < STEP; ++c) x[c] = y[c] = acc[i][j][v + c];
                    if constexpr (Q4) {
                        q4_gelu(y);
                    } else if constexpr (F32) {
#pragma unroll
                        for (int c = 0; c < STEP; ++c) y[c] = gelu_erf(x[c]);
                    } else {
                        q8_gelu<STEP, 7>(x, kQ8Gelu, y);
                    }
#pragma unroll
                    for (int c = 0; c < STEP; ++c) acc[i][j][v + c] = y[c];
                }
    float mx[TM];
    if constexpr (!F32 && !BF16 && !E2M1) {
        // Bytes past N are zeros whatever the row holds (their sums are zeros
        // times A: NaN where A is no number or infinite); 16 of them at most
        // are stored.
        if (cols != g.N && nw + 32 * TN > g.N)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (nw + j * 32 + 16 * (v >> 3) + 8 * lh + (v & 7) >= g.N)
#pragma unroll
                        for (int i = 0; i < TM; ++i) acc[i][j][v] = 0.0f;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            // a lane and the one 32 further hold a row's columns; infinities
            // (rare: the whole wave looks again) do not set the scale
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) m = fmaxf(m, fabsf(acc[i][j][v]));
            if (__ballot(!(m < __builtin_inff())) != 0) {
                m = 0.0f;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) m = fmaxf(m, q8_mag(acc[i][j][v]));
            }
            mx[i] = fmaxf(m, __shfl_xor(m, 32));
            if (SHARE > 1 && lh == 0) s_max[wn * BM + rw + i * 32 + lrow] = mx[i];
        }
        if constexpr (SHARE > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int w = 0; w < SHARE; ++w)
                    mx[i] = fmaxf(mx[i], s_max[(wn / SHARE * SHARE + w) * BM + rw + i * 32 + lrow]);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 w = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    const int ch = j * 8 + 4 * (q >> 1) + 2 * lh + (q & 1);
                    *reinterpret_cast<f32x4*>(wb + lrow * RB + ((ch ^ (lrow % CH)) << 4)) = w;
                }
        } else if constexpr (BF16) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 w;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        w[q] = pack2_bf16(acc[i][j][8 * h + 2 * q], acc[i][j][8 * h + 2 * q + 1]);
                    const int ch = j * 4 + 2 * h + lh;
                    *reinterpret_cast<u32x4*>(wb + lrow * RB + ((ch ^ (lrow % CH)) << 4)) = w;
                }
        } else if constexpr (E2M1) {
            // A block is a tile's 32 columns: a lane and the one 32 further
            // hold a row's.  (Columns past N are zeros, but where the row is
            // no number, and then so is its last block.)
            const int rl = rw + i * 32 + lrow;
            uint32_t scales = 0;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                // the largest magnitude; NaN if one of them is
                float m = 0.0f;
#pragma unroll
                for (int v = 0; v < 16; v += 2)
                    m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(acc[i][j][v]), fabsf(acc[i][j][v + 1])), m);
                m = __builtin_elementwise_maximum(m, __shfl_xor(m, 32));
                const int e = nw + j * 32 < g.N ? q4_exponent(q4_mag(m)) : 0;
                const float k = e == kQ4NaN ? 1.0f : q8_two_to(e);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w =
                        q4_pack8_over(acc[i][j][8 * h], acc[i][j][8 * h + 1], acc[i][j][8 * h + 2], acc[i][j][8 * h + 3],
                                      acc[i][j][8 * h + 4], acc[i][j][8 * h + 5], acc[i][j][8 * h + 6],
                                      acc[i][j][8 * h + 7], k);
                    *reinterpret_cast<uint32_t*>(wb + lrow * RB + ((j ^ (lrow % CH)) << 4) + 8 * h + 4 * lh) =
                        e == kQ4NaN ? 0u : w;
                }
                scales |= static_cast<uint32_t>(e + kQ8One) << (8 * j);
            }
            // TN scales side by side; the last ones fill the row up
            if (lh == 0 && rl < t.rows && nw < g.N) {
                uint8_t* s = g.SC + (t.m_lo + rl) * g.sc_ld + nw / kQ4Block;
                if constexpr (TN == 4) *reinterpret_cast<uint32_t*>(s) = scales;
                else if constexpr (TN == 2) *reinterpret_cast<uint16_t*>(s) = static_cast<uint16_t>(scales);
                else *s = static_cast<uint8_t>(scales);
                if (TN < 4 && nw + TN * 32 >= g.N)
                    for (int64_t p = nw / kQ4Block + TN; p < g.sc_ld; ++p) g.SC[(t.m_lo + rl) * g.sc_ld + p] = kQ8One;
            }
        } else {
            const int e = q8_exponent(__float_as_uint(mx[i]), q8_top_exp(FMT));
            const float k = q8_two_to(e);
            const int rl = rw + i * 32 + lrow;
            if (lh == 0 && rl < t.rows && nw % kQ8Block == 0 && nw < g.N) {
                uint8_t* s = g.SC + (t.m_lo + rl) * g.sc_ld;
                const int blk = nw / kQ8Block;
                s[blk] = static_cast<uint8_t>(e + kQ8One);
                if (nw + kQ8Block >= g.N)                       // the last block fills the row up
                    for (int64_t p = blk + 1; p < g.sc_ld; ++p) s[p] = kQ8One;
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x2 w;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int v = 8 * h + 4 * q;
                        w[q] = q8_pack4_over<FMT>(acc[i][j][v], acc[i][j][v + 1], acc[i][j][v + 2],
                                                  acc[i][j][v + 3], k);
                    }
                    const int ch = j * 2 + h;
                    *reinterpret_cast<u32x2*>(wb + lrow * RB + ((ch ^ (lrow % CH)) << 4) + 8 * lh) = w;
                }
        }
        // one wave's LDS accesses complete in order: only the compiler has to
        // keep them in place
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int it = 0; it < 32 / RPI; ++it) {
            const int rr = it * RPI + lane / CH, ch = lane % CH;
            if (RPI * CH < 64 && lane >= RPI * CH) continue;    // (a row is one piece)
            const u32x4 w = *reinterpret_cast<const u32x4*>(wb + rr * RB + ((ch ^ (rr % CH)) << 4));
            const int rl = rw + i * 32 + rr;
            if (rl >= t.rows) continue;
            if constexpr (F32) {
                const int n = nw + ch * 4;
                float* c = static_cast<float*>(g.C) + (t.m_lo + rl) * g.ldc + n;
                if (g.wide) {
                    if (n < g.N) *reinterpret_cast<u32x4*>(c) = w;
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (n + q < g.N) c[q] = __uint_as_float(w[q]);
                }
            } else if constexpr (BF16) {
                const int n = nw + ch * 8;
                bf16_bits* c = static_cast<bf16_bits*>(g.C) + (t.m_lo + rl) * g.ldc + n;
                if (g.wide) {
                    if (n < g.N) *reinterpret_cast<u32x4*>(c) = w;
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (n + q < g.N) c[q] = static_cast<bf16_bits>(w[q >> 1] >> (16 * (q & 1)));
                }
            } else if constexpr (E2M1) {
                const int n = nw + ch * 32;
                if (n < g.N)
                    *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(g.C) + (t.m_lo + rl) * g.ldc + n / 2) = w;
            } else {
                const int n = nw + ch * 16;
                if (n < cols)
                    *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(g.C) + (t.m_lo + rl) * g.ldc + n) = w;
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace

}  // namespace clearmoe
