// 8-bit floating point with power-of-two block scales (q8.h).  The scale is
// exact to divide by, so a value is rounded once, and the matrix instructions
// apply it for nothing.  One read of x, one write of its bytes: bound by
// memory.  Measured on an MI355X: rows of 50432 x 768 bfloat16 in 25 us (4.7
// TB/s; a large copy moves 4.8), 12608 x 384 in 5, squares of 8 x 1550 x 790
// float32 in 15 (3.2 TB/s: a workgroup holds its square until the maximum of
// all of it is known).
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
    float m = q8_mag8(f);
#pragma unroll
    for (int s = kLanes / 2; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
    const int e = q8_exponent(__float_as_uint(m), q8_top_exp(FMT));
    if (c < vcols) *reinterpret_cast<uint2*>(v + row * vcols + c) = q8_pack8<FMT>(f, q8_two_to(-e));
    if (sub == 0) {
        uint8_t* s = scale + row * scols;
        s[blk] = static_cast<uint8_t>(e + kQ8One);
        if (blk == blocks - 1)
            for (int64_t i = blocks; i < scols; ++i) s[i] = kQ8One;
    }
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

}  // namespace

hipError_t launch_quantize(int dtype, int fmt, int block_rows, int64_t batch, int64_t rows, int64_t cols,
                           const void* x, int64_t ldx, uint8_t* v, uint8_t* scale, hipStream_t st) {
    if (batch == 0 || rows == 0) return hipSuccess;
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
