// 8-bit floating point with block scales: internal declarations of the
// quantiser (quantize.hip) and the products (gemm_q8.hip).
//
// A matrix of k columns is held as rows of round_up(k, 16) bytes (zeros past
// k) and, for each block of 128 columns of a row (or of 128 rows), one byte b
// that stands for the scale 2^(b - 127); rows of scales have
// q8_scale_cols(k) bytes, whole 4-byte words.
#pragma once

#include "kernels.h"

namespace clearmoe {

constexpr int kQ8Block = 128;
constexpr int kQ8One = 127;              // the scale byte of 1

__host__ __device__ inline int64_t q8_cols(int64_t k) { return (k + 15) / 16 * 16; }
__host__ __device__ inline int64_t q8_blocks(int64_t k) { return (k + kQ8Block - 1) / kQ8Block; }
__host__ __device__ inline int64_t q8_scale_cols(int64_t k) { return (q8_blocks(k) + 3) / 4 * 4; }

// Formats, as the matrix instructions number them, and output types.
enum { kQ8E4M3 = 0, kQ8E5M2 = 1 };
enum { kQ8OutF32 = 0, kQ8OutBf16 = 1, kQ8OutE4M3 = 2, kQ8OutE5M2 = 3 };

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

// x [batch, rows, cols] (dtype, row stride ldx elements, batches rows * ldx
// apart) -> v, scale; block_rows 1 or 128.
hipError_t launch_quantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                           const void* x, int64_t ldx, uint8_t* v, uint8_t* scale, hipStream_t st);

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

}  // namespace clearmoe
