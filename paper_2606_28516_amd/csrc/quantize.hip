// 8- and 4-bit floating point with power-of-two block scales (q8.h), and back.
// The scale is exact to divide by, so a value is rounded once, and the matrix
// instructions apply it for nothing.  One read of x, one write of its bytes:
// bound by memory.  Measured on an MI355X, calls in a row (a large copy moves 5.0
// to 5.2 TB/s): rows of 50432 x 768 bfloat16 in 25 us (4.7 TB/s), 12608 x 384 in
// 5, squares of 8 x 1550 x 790 float32 in 15 (3.2 TB/s: a workgroup holds its
// square until the maximum of all of it is known).  4 bits: rows of 50432 x 1024
// bfloat16 in 23 us (5.7 TB/s: part of the rows is still in the last-level
// cache), 8 x 1550 x 790 float32 in 9.0; back to the same types 20.6 and 10.5.
#include "q8.h"

namespace clearmoe {

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = kQ8Lanes;

// 1 x 128 blocks: 16 lanes a block.
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void k_quantize_rows(const T* x, int64_t ldx, int64_t rows, int64_t cols,
                                                            uint8_t* v, uint8_t* scale) {
    const int64_t blocks = q8_blocks(cols), vcols = q8_cols(cols), scols = q8_scale_cols(cols);
    const int sub = threadIdx.x % kLanes;
    const int64_t b = static_cast<int64_t>(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (b >= rows * blocks) return;
    const int64_t row = b / blocks, blk = b - row * blocks, c = blk * kQ8Block + sub * 8;
    float f[8];
    q8_load8(x + row * ldx, c, cols, f);
    const float m = q8_max16(q8_mag8(f));
    const int e = q8_exponent(__float_as_uint(m), q8_top_exp(FMT));
    if (c < vcols) *reinterpret_cast<uint2*>(v + row * vcols + c) = q8_pack8<FMT>(f, q8_two_to(-e));
    if (sub == 0) {
        uint8_t* s = scale + row * scols;
        s[blk] = static_cast<uint8_t>(e + kQ8One);
        if (blk == blocks - 1)
            for (int64_t i = blocks; i < scols; ++i) s[i] = kQ8One;
    }
}

// e2m1: 16 lanes take 128 columns, four blocks of 32, and write their bytes
// and the word of their four scales.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_quantize4(const T* x, int64_t ldx, int64_t rows, int64_t cols,
                                                        uint8_t* v, uint8_t* scale) {
    const int64_t units = q8_blocks(cols), vcols = q4_cols(cols);
    const int sub = threadIdx.x % kLanes;
    const int64_t b = static_cast<int64_t>(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (b >= rows * units) return;
    const int64_t row = b / units, unit = b - row * units, c = unit * kQ8Block + sub * 8;
    float f[8];
    q8_load8(x + row * ldx, c, cols, f);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, q4_mag(f[i]));
    m = max(m, static_cast<uint32_t>(q8_partner<1>(static_cast<int>(m))));
    m = max(m, static_cast<uint32_t>(q8_partner<2>(static_cast<int>(m))));
    const int e = q4_exponent(m);
    if (c / 2 < vcols) *reinterpret_cast<uint32_t*>(v + row * vcols + c / 2) = q4_pack8(f, e);
    // (blocks past the last have no columns: zeros, the scale 1)
    uint32_t w = static_cast<uint32_t>(e + kQ8One) << (8 * (sub / 4));
    w |= static_cast<uint32_t>(q8_partner<4>(static_cast<int>(w)));
    w |= static_cast<uint32_t>(q8_partner<8>(static_cast<int>(w)));
    if (sub == 0) reinterpret_cast<uint32_t*>(scale)[row * units + unit] = w;
}

// The value that a byte (e2m1: eight values, the word of them) stands for,
// times 2^(s - 127).  Exact in float32, and in bfloat16 but where it falls
// below its normal numbers.
template <int FMT>
__device__ __forceinline__ void q8_read8(const uint8_t* p, uint32_t s, float (&f)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 d[4];
    if constexpr (FMT == kQ8E2M1) {
        const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
        d[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 0);
        d[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 1);
        d[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 2);
        d[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(u, 1.0f, 3);
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        const int w[2] = {static_cast<int>(u.x), static_cast<int>(u.y)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if constexpr (FMT == kQ8E4M3) {
                d[2 * i] = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false);
                d[2 * i + 1] = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
            } else {
                d[2 * i] = __builtin_amdgcn_cvt_pk_f32_bf8(w[i], false);
                d[2 * i + 1] = __builtin_amdgcn_cvt_pk_f32_bf8(w[i], true);
            }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = s == 255u ? __builtin_nanf("") : __builtin_ldexpf(d[i / 2][i % 2], static_cast<int>(s) - kQ8One);
}

// Back: a thread takes eight columns.
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void k_dequantize(const uint8_t* v, const uint8_t* scale, int block_rows,
                                                         int64_t rows, int64_t first, int64_t all, int64_t cols,
                                                         T* y, int64_t ldy) {
    constexpr bool E2M1 = FMT == kQ8E2M1;
    const int64_t pieces = (cols + 7) / 8;
    const int64_t i = (first + blockIdx.x) * kThreads + threadIdx.x;
    if (i >= all) return;
    const int64_t row = i / pieces, c = (i - row * pieces) * 8;         // row over all batches
    int64_t srow = row;
    if (block_rows != 1) {
        const int64_t b = row / rows;
        srow = b * ((rows + kQ8Block - 1) / kQ8Block) + (row - b * rows) / kQ8Block;
    }
    const uint32_t s = scale[srow * (E2M1 ? q4_scale_cols(cols) : q8_scale_cols(cols)) + c / (E2M1 ? kQ4Block : kQ8Block)];
    float f[8];
    q8_read8<FMT>(v + row * (E2M1 ? q4_cols(cols) : q8_cols(cols)) + (E2M1 ? c / 2 : c), s, f);
    q8_store8(y + row * ldy, c, cols, f);
}

// 128 x 128 blocks: a workgroup each (from block `first` on), its values in
// registers between the maximum and the rounding.
template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void k_quantize_square(const T* x, int64_t ldx, int64_t rows, int64_t cols,
                                                              int64_t first, uint8_t* v, uint8_t* scale) {
    constexpr int PASS = kThreads / kLanes, NP = kQ8Block / PASS;       // rows a pass, passes
    __shared__ float s_m[kThreads / 64];
    const int64_t blocks = q8_blocks(cols), vcols = q8_cols(cols), scols = q8_scale_cols(cols);
    const int64_t nr = (rows + kQ8Block - 1) / kQ8Block;
    const int sub = threadIdx.x % kLanes, rl = threadIdx.x / kLanes;
    const int64_t at = first + blockIdx.x, br = at / blocks, blk = at - br * blocks;    // row block over all batches
    const int64_t batch = br / nr, r0 = (br - batch * nr) * kQ8Block, c = blk * kQ8Block + sub * 8;
    const T* xb = x + batch * rows * ldx;
    float f[NP][8], m = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int64_t row = r0 + p * PASS + rl;
        q8_load8(xb + (row < rows ? row : 0) * ldx, c, row < rows ? cols : 0, f[p]);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) m = fmaxf(m, q8_mag8(f[p]));
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
    if (threadIdx.x % 64 == 0) s_m[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, s_m[w]);
    const int e = q8_exponent(__float_as_uint(m), q8_top_exp(FMT));
    const float k = q8_two_to(-e);
    uint8_t* vb = v + batch * rows * vcols;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int64_t row = r0 + p * PASS + rl;
        if (row < rows && c < vcols) *reinterpret_cast<uint2*>(vb + row * vcols + c) = q8_pack8<FMT>(f[p], k);
    }
    if (threadIdx.x == 0) {
        uint8_t* s = scale + br * scols;
        s[blk] = static_cast<uint8_t>(e + kQ8One);
        if (blk == blocks - 1)
            for (int64_t i = blocks; i < scols; ++i) s[i] = kQ8One;
    }
}

// Workgroups of a launch: a grid holds less than 2^32 threads.  Larger
// matrices take several launches.
constexpr int64_t kMostGroups = ((int64_t{1} << 32) - 1) / kThreads;

template <typename T, int FMT>
hipError_t quantize(int block_rows, int64_t batch, int64_t rows, int64_t cols, const T* x, int64_t ldx, uint8_t* v,
                    uint8_t* scale, hipStream_t st) {
    constexpr int64_t PER = kThreads / kLanes;                          // row blocks a workgroup
    const int64_t blocks = q8_blocks(cols);
    if (block_rows == 1) {
        const int64_t all = batch * rows, most = kMostGroups * PER / blocks;
        for (int64_t r = 0; r < all; r += most) {
            const int64_t n = all - r < most ? all - r : most, grid = (n * blocks + PER - 1) / PER;
            launch_kernel(k_quantize_rows<T, FMT>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st,
                          x + r * ldx, ldx, n, cols, v + r * q8_cols(cols), scale + r * q8_scale_cols(cols));
        }
    } else {
        const int64_t all = batch * ((rows + kQ8Block - 1) / kQ8Block) * blocks;
        for (int64_t b = 0; b < all; b += kMostGroups) {
            const int64_t grid = all - b < kMostGroups ? all - b : kMostGroups;
            launch_kernel(k_quantize_square<T, FMT>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st, x, ldx,
                          rows, cols, b, v, scale);
        }
    }
    return hipGetLastError();
}

template <typename T>
hipError_t quantize4(int64_t all, int64_t cols, const T* x, int64_t ldx, uint8_t* v, uint8_t* scale, hipStream_t st) {
    constexpr int64_t PER = kThreads / kLanes;
    const int64_t units = q8_blocks(cols), most = kMostGroups * PER / units;
    for (int64_t r = 0; r < all; r += most) {
        const int64_t n = all - r < most ? all - r : most, grid = (n * units + PER - 1) / PER;
        launch_kernel(k_quantize4<T>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st, x + r * ldx, ldx, n,
                      cols, v + r * q4_cols(cols), scale + r * q4_scale_cols(cols));
    }
    return hipGetLastError();
}

template <typename T, int FMT>
hipError_t dequantize(int block_rows, int64_t batch, int64_t rows, int64_t cols, const uint8_t* v,
                      const uint8_t* scale, T* y, int64_t ldy, hipStream_t st) {
    const int64_t all = batch * rows * ((cols + 7) / 8), groups = (all + kThreads - 1) / kThreads;
    for (int64_t b = 0; b < groups; b += kMostGroups) {
        const int64_t grid = groups - b < kMostGroups ? groups - b : kMostGroups;
        launch_kernel(k_dequantize<T, FMT>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st, v, scale,
                      block_rows, rows, b, all, cols, y, ldy);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize(int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols, const uint8_t* v,
                      const uint8_t* scale, void* y, int64_t ldy, hipStream_t st) {
    T* p = static_cast<T*>(y);
    return fmt == kQ8E4M3   ? dequantize<T, kQ8E4M3>(block_rows, batch, rows, cols, v, scale, p, ldy, st)
           : fmt == kQ8E5M2 ? dequantize<T, kQ8E5M2>(block_rows, batch, rows, cols, v, scale, p, ldy, st)
                            : dequantize<T, kQ8E2M1>(block_rows, batch, rows, cols, v, scale, p, ldy, st);
}

}  // namespace

hipError_t launch_dequantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                             const uint8_t* v, const uint8_t* scale, void* y, int64_t ldy, hipStream_t st) {
    if (batch == 0 || rows == 0) return hipSuccess;
    return dtype == 0 ? dequantize<float>(fmt, block_rows, batch, rows, cols, v, scale, y, ldy, st)
                      : dequantize<bf16_bits>(fmt, block_rows, batch, rows, cols, v, scale, y, ldy, st);
}

hipError_t launch_quantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                           const void* x, int64_t ldx, uint8_t* v, uint8_t* scale, hipStream_t st) {
    if (batch == 0 || rows == 0) return hipSuccess;
    if (fmt == kQ8E2M1)
        return dtype == 0 ? quantize4(batch * rows, cols, static_cast<const float*>(x), ldx, v, scale, st)
                          : quantize4(batch * rows, cols, static_cast<const bf16_bits*>(x), ldx, v, scale, st);
    if (dtype == 0) {
        const float* p = static_cast<const float*>(x);
        return fmt == kQ8E4M3 ? quantize<float, kQ8E4M3>(block_rows, batch, rows, cols, p, ldx, v, scale, st)
                              : quantize<float, kQ8E5M2>(block_rows, batch, rows, cols, p, ldx, v, scale, st);
    }
    const bf16_bits* p = static_cast<const bf16_bits*>(x);
    return fmt == kQ8E4M3 ? quantize<bf16_bits, kQ8E4M3>(block_rows, batch, rows, cols, p, ldx, v, scale, st)
                          : quantize<bf16_bits, kQ8E5M2>(block_rows, batch, rows, cols, p, ldx, v, scale, st);
}

}  // namespace clearmoe
