// 8- and 4-bit floating point with block scales: internal declarations of the
// quantiser (quantize.hip), the norm with an 8-bit output (norm.hip) and the
// products (gemm_q8.hip, gemm_q4.hip).
//
// 8 bits: a matrix of k columns is held as rows of round_up(k, 16) bytes (zeros past
// k) and, for each block of 128 columns of a row (or of 128 rows), one byte b
// that stands for the scale 2^(b - 127); rows of scales have
// q8_scale_cols(k) bytes, whole 4-byte words.
//
// 4 bits (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives): blocks of 32
// columns of a row, 16 bytes with the even column of a byte in its low half;
// rows of q4_cols(k) bytes (zeros past k) and of q4_scale_cols(k) scales.
#pragma once

#include "kernels.h"

namespace clearmoe {

constexpr int kQ8Block = 128;
constexpr int kQ8One = 127;              // the scale byte of 1

__host__ __device__ inline int64_t q8_cols(int64_t k) { return (k + 15) / 16 * 16; }
__host__ __device__ inline int64_t q8_blocks(int64_t k) { return (k + kQ8Block - 1) / kQ8Block; }
__host__ __device__ inline int64_t q8_scale_cols(int64_t k) { return (q8_blocks(k) + 3) / 4 * 4; }

constexpr int kQ4Block = 32;
__host__ __device__ inline int64_t q4_blocks(int64_t k) { return (k + kQ4Block - 1) / kQ4Block; }
__host__ __device__ inline int64_t q4_cols(int64_t k) { return q4_blocks(k) * (kQ4Block / 2); }
__host__ __device__ inline int64_t q4_scale_cols(int64_t k) { return (q4_blocks(k) + 3) / 4 * 4; }

// Formats, as the matrix instructions number them, and output types.
enum { kQ8E4M3 = 0, kQ8E5M2 = 1, kQ8E2M1 = 4 };
enum { kQ8OutF32 = 0, kQ8OutBf16 = 1, kQ8OutE4M3 = 2, kQ8OutE5M2 = 3, kQ8OutE2M1 = 4 };

// Largest finite value 1.75 * 2^kTopExp of a format.
__host__ __device__ constexpr int q8_top_exp(int fmt) { return fmt == kQ8E4M3 ? 8 : 15; }

// The scale exponent of a block whose largest finite magnitude has the bits u:
// the smallest e with amax <= 1.75 2^(top + e), at least -126; 0 for zeros.
// (Adding 0x1fffff carries into the exponent exactly when the mantissa is
// above 1.75.)
__device__ __forceinline__ int q8_exponent(uint32_t u, int top) {
    if (u == 0) return 0;
    const int e = static_cast<int>((u + 0x1fffffu) >> 23) - 127 - top;
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float q8_two_to(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// The same for e2m1 (amax <= 1.5 2^(2 + e)) of a block's largest magnitude
// bits u, those of NaN and infinity too: 128, the scale that is no number,
// since e2m1 has neither.
constexpr int kQ4NaN = 128;
__device__ __forceinline__ int q4_exponent(uint32_t u) {
    if (u == 0) return 0;
    if (u >= 0x7f800000u) return kQ4NaN;
    const int e = static_cast<int>((u + 0x3fffffu) >> 23) - 127 - 2;
    return e < -126 ? -126 : e;
}
// Bits of |v|, ordered as the magnitudes are, NaN above infinity.
__device__ __forceinline__ uint32_t q4_mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// |v| for the block's maximum: infinities and NaN do not set a scale.
__device__ __forceinline__ float q8_mag(float v) {
    const float m = fabsf(v);
    return m < __builtin_inff() ? m : 0.0f;
}
// Four floats -> four bytes, round to nearest even; infinities become NaN in
// e4m3 (which has none) and stay in e5m2.
template <int FMT>
__device__ __forceinline__ uint32_t q8_pack4(float a, float b, float c, float d) {
    int v = 0;
    if constexpr (FMT == kQ8E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
    }
    return static_cast<uint32_t>(v);
}

// The value of a lane's partner in its row of 16 lanes: the steps of a
// butterfly over 2, 4, 8 and 16 lanes (the last two mirror the halves, which is
// as good once the smaller groups agree).  In the vector unit, without the LDS
// that a shuffle takes.
template <int STEP>
__device__ __forceinline__ int q8_partner(int v) {
    constexpr int CTRL = STEP == 1 ? 0xb1 : STEP == 2 ? 0x4e : STEP == 4 ? 0x141 : 0x140;
    return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
template <int STEP>
__device__ __forceinline__ float q8_partner(float v) {
    return __int_as_float(q8_partner<STEP>(__float_as_int(v)));
}
// The largest of 16 lanes.
__device__ __forceinline__ float q8_max16(float m) {
    m = fmaxf(m, q8_partner<1>(m));
    m = fmaxf(m, q8_partner<2>(m));
    m = fmaxf(m, q8_partner<4>(m));
    return fmaxf(m, q8_partner<8>(m));
}

// A lane's share of a 128-column block when 16 lanes quantise it: columns
// [c, c + 8) of a row, zeros from n on.  (A piece may start at any element:
// the hardware loads it all the same.)
constexpr int kQ8Lanes = 16;
template <typename T>
__device__ __forceinline__ void q8_load8(const T* row, int64_t c, int64_t n, float (&v)[8]) {
    if (c + 8 > n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < n ? Elem<T>::load(row, c + i) : 0.0f;
    } else if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(v, row + c, 32);
    } else {
        u32x4 a;
        __builtin_memcpy(&a, row + c, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
        }
    }
}
// Columns [c, c + 8) of a row, those before n.
template <typename T>
__device__ __forceinline__ void q8_store8(T* row, int64_t c, int64_t n, const float (&v)[8]) {
    if (c + 8 > n) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < n) row[c + i] = Elem<T>::from_f32(v[i]);
    } else if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(row + c, v, 32);
    } else {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = pack2_bf16(v[2 * i], v[2 * i + 1]);
        __builtin_memcpy(row + c, &a, 16);
    }
}
__device__ __forceinline__ float q8_mag8(const float (&v)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, q8_mag(v[i]));
    return m;
}
template <int FMT>
__device__ __forceinline__ uint2 q8_pack8(const float (&v)[8], float s) {
    return make_uint2(q8_pack4<FMT>(v[0] * s, v[1] * s, v[2] * s, v[3] * s),
                      q8_pack4<FMT>(v[4] * s, v[5] * s, v[6] * s, v[7] * s));
}

// Eight floats over 2^e (their block's; e = kQ4NaN: zeros) -> eight e2m1
// values, the first in the lowest bits, round to nearest even.
__device__ __forceinline__ uint32_t q4_pack8(const float (&v)[8], int e) {
    if (e == kQ4NaN) return 0;
    const float s = q8_two_to(-e);               // (a normal number: the product is exact)
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * s, v[1] * s, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * s, v[3] * s, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * s, v[5] * s, 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * s, v[7] * s, 1.0f, 3);
}

// x [batch, rows, cols] (dtype, row stride ldx elements, batches rows * ldx
// apart) -> v, scale; block_rows 1 or 128 (e2m1: 1).
hipError_t launch_quantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                           const void* x, int64_t ldx, uint8_t* v, uint8_t* scale, hipStream_t st);

// v, scale of a format -> y [batch, rows, cols] (dtype, row stride ldy).
hipError_t launch_dequantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                             const uint8_t* v, const uint8_t* scale, void* y, int64_t ldy, hipStream_t st);

// h = x (+ residual), y = h rsqrt(mean h^2 + eps) weight (norm.hip): rows of
// dtype, y of dtype or (out: a byte format) 8-bit with scales of 1 x 128.
struct NormArgs {
    const void* x;
    const void* residual;        // or null
    const float* weight;         // [cols], or null: ones
    void* sum;                   // h, or null
    void* y;                     // 8 bits: rows of ldy bytes
    uint8_t* scale;              // 8 bits: rows of q8_scale_cols(cols) bytes
    int64_t ldx, ldr, lds, ldy;
    int64_t rows;
    int cols;
    float eps;
    double inv_cols;             // 1 / cols
};
hipError_t launch_rms_norm(int dtype, int out, const NormArgs& a, hipStream_t st);

// C[m, n] = epi( sum over blocks of 2^(sa + sb) sum_k A[m, k] B_seg(m)[n, k] ).
struct Q8Desc {
    const uint8_t* A;            // [M, >= K] row stride lda bytes
    int64_t lda;
    const uint8_t* SA;           // [M, sa_ld]
    int64_t sa_ld;
    const uint8_t* B;            // [N, K] per segment
    int64_t b_seg_stride;
    const uint8_t* SB;           // [ceil(N / 128), q8_scale_cols(K)] per segment
    int64_t sb_ld, sb_seg_stride;
    const float* bias;           // [N] per segment, or null
    void* C;                     // row stride ldc elements
    int64_t ldc;
    uint8_t* SC;                 // 8-bit output: its scales, row stride sc_ld
    int64_t sc_ld;
    int out, gelu, fa, fb;
    int wide;                    // C rows can be stored 16 bytes at a time
    int64_t M;
    int N, K;                    // K a multiple of 16
    const int32_t* seg_offsets;  // [nseg + 1] on the device, or null
    int nseg;
    int seg_merge;               // always 0 (the tile search's field)
};
hipError_t launch_gemm_q8(const Q8Desc& g, hipStream_t st);
// The kernel that a product takes: 16 x 16 tiles, 64 x 64 (bytes: 64 x 128),
// 128 x 128 or 256 x 128.
enum Q8Kernel { kQ8Rows, kQ8Small, kQ8Middle, kQ8Large };
Q8Kernel q8_kernel(const Q8Desc& g);
// Whether the product fits one launch: a grid holds less than 2^32 threads,
// and one that asks for more is cut without an error.
bool q8_launch_fits(int64_t M, int N, int groups, int out);

// The same product in e4m3 for a few rows of A that are still float32
// (a_f32) or bfloat16 [M, K0] (row stride K0, K = q8_cols(K0)): every workgroup
// quantises its rows of A itself, in blocks of 128 columns, so that a
// quantising pass over them is not a launch of its own.  float32 or bfloat16
// results; SA, A, lda, fa and fb are not used.
constexpr int64_t kQ8FewRows = 16;       // at most: then a pass of its own costs less
bool q8_few_supported(int64_t M, int64_t K);
hipError_t launch_q8_few(const Q8Desc& g, const void* A, bool a_f32, int K0, hipStream_t st);

// The product of e4m3 or e2m1 rows (fa) and e2m1 matrices (gemm_q4.hip); every
// stride of bytes in bytes: a row of B has q4_cols(K) of them, SB
// q4_scale_cols(K) for each of N, a row of e2m1 results ldc.
hipError_t launch_gemm_q4(const Q8Desc& g, hipStream_t st);
// The kernel that a product takes: 16 x 16 tiles, 64 x 64, 64 x 128 (split: by
// two groups of waves along k), 128 x 128 (deep: 256 of k a stage), or 256 x
// 256 (4-bit rows to bfloat16) and 128 x 256.
enum Q4Kernel { kQ4Rows, kQ4Small, kQ4Split, kQ4Wide, kQ4Middle, kQ4Deep, kQ4Large };
Q4Kernel q4_kernel(const Q8Desc& g);
// The rows that a first launch takes; the others follow in a second one.
int64_t q4_whole_rows(const Q8Desc& g);
// Whether the product fits one launch.
bool q4_launch_fits(int64_t M, int N, int groups);
// As launch_q8_few, the rows quantised to fa.
bool q4_few_supported(int64_t M, int64_t K);
hipError_t launch_q4_few(const Q8Desc& g, const void* A, bool a_f32, int K0, hipStream_t st);

}  // namespace clearmoe
