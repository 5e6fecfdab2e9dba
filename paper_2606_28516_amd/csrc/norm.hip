// Root-mean-square norm with the residual's addition:
//     h = x + residual (rounded to the rows' type: the stream that goes on),
//     y = h (mean(h^2) + eps)^(-1/2) weight,
// y in the rows' type or in 8 bits with a power-of-two scale for each 128
// columns (q8.h), rounded once from float32.
//
// One read of x and the residual, one write of h and y: bound by memory.  A
// row stays in registers between its sum and its scaling, whatever its width
// (65536 columns are 64 values a thread).
#include "q8.h"

namespace clearmoe {

namespace {

constexpr int kNormThreads = 256;

// TPR threads a row, NP pieces of eight columns a thread: piece p of thread t
// is columns 8 (p TPR + t) on, so that 16 threads side by side hold a block of
// 128.  TPR 64: a wave a row, four rows a workgroup.
template <typename T, int OUT, int TPR, int NP>
__global__ __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) void k_rms_norm(NormArgs a, int64_t first) {
    constexpr int THREADS = TPR > kNormThreads ? TPR : kNormThreads, WAVES = TPR / 64;
    const int t = threadIdx.x % TPR;
    const int64_t row = first + static_cast<int64_t>(blockIdx.x) * (THREADS / TPR) + threadIdx.x / TPR;
    if (TPR == 64 && row >= a.rows) return;      // (a whole wave; else a workgroup has one row, and exists)
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float f[NP][8];
#pragma unroll
    for (int p = 0; p < NP; ++p) q8_load8(x, 8 * (p * TPR + t), a.cols, f[p]);
    if (a.residual != nullptr) {
        const T* r = static_cast<const T*>(a.residual) + row * a.ldr;
        // (at most four pieces on their way: the registers hold no more)
#pragma unroll
        for (int q = 0; q < NP; q += 4) {
            float g[4][8];
#pragma unroll
            for (int p = 0; p < 4 && q + p < NP; ++p) q8_load8(r, 8 * ((q + p) * TPR + t), a.cols, g[p]);
#pragma unroll
            for (int p = 0; p < 4 && q + p < NP; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f[q + p][i] = Elem<T>::to_f32(Elem<T>::from_f32(f[q + p][i] + g[p][i]));
            if (NP > 4) __builtin_amdgcn_sched_barrier(0);
        }
    }
    // in double: no finite row's squares overflow, and the sum of a long row
    // keeps what float32 would drop
    double s = 0.0;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double d = static_cast<double>(f[p][i]);
            s = __builtin_fma(d, d, s);
        }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if constexpr (WAVES > 1) {
        __shared__ double s_sum[WAVES];
        if (threadIdx.x % 64 == 0) s_sum[threadIdx.x / 64] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += s_sum[w];
    }
    // (mean + eps)^(-1/2) in float32 for any exponent: mean + eps = m 4^k with
    // m in [1/4, 1), whose root is the hardware's (1 ulp); k = 0 of NaN and
    // infinity
    const double mean = __builtin_fma(s, a.inv_cols, static_cast<double>(a.eps));
    const int k = (__builtin_amdgcn_frexp_exp(mean) + 1) >> 1;
    const float inv = __builtin_ldexpf(__builtin_amdgcn_rsqf(static_cast<float>(__builtin_ldexp(mean, -2 * k))), -k);
    if (a.sum != nullptr) {
        T* h = static_cast<T*>(a.sum) + row * a.lds;
#pragma unroll
        for (int p = 0; p < NP; ++p) q8_store8(h, 8 * (p * TPR + t), a.cols, f[p]);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        float w[8];
        if (a.weight != nullptr) {
            q8_load8(a.weight, 8 * (p * TPR + t), a.cols, w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 1.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[p][i] = f[p][i] * inv * w[i];
        if (NP > 4) __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (OUT < kQ8OutE4M3) {
        T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
        for (int p = 0; p < NP; ++p) q8_store8(y, 8 * (p * TPR + t), a.cols, f[p]);
    } else {
        constexpr int FMT = OUT == kQ8OutE4M3 ? kQ8E4M3 : kQ8E5M2;
        const int blocks = static_cast<int>(q8_blocks(a.cols)), vcols = static_cast<int>(q8_cols(a.cols));
        const int scols = static_cast<int>(q8_scale_cols(a.cols));
        uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.ldy;
        uint8_t* sc = a.scale + row * scols;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int c = 8 * (p * TPR + t), blk = c / kQ8Block;
            // columns past the last hold zeros, NaN where the row's scale is
            // none: zeros again
            if (c + 8 > a.cols)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i >= a.cols) f[p][i] = 0.0f;
            float m = q8_mag8(f[p]);
#pragma unroll
            for (int o = kQ8Lanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            const int e = q8_exponent(__float_as_uint(m), q8_top_exp(FMT));
            if (c < vcols) *reinterpret_cast<uint2*>(y + c) = q8_pack8<FMT>(f[p], q8_two_to(-e));
            if (t % kQ8Lanes == 0 && blk < blocks) {
                sc[blk] = static_cast<uint8_t>(e + kQ8One);
                if (blk == blocks - 1)
                    for (int i = blocks; i < scols; ++i) sc[i] = kQ8One;
            }
        }
    }
}

template <typename T, int OUT, int TPR, int NP>
hipError_t norm(const NormArgs& a, hipStream_t st) {
    constexpr int THREADS = TPR > kNormThreads ? TPR : kNormThreads, PER = THREADS / TPR;
    // a grid holds less than 2^32 threads: larger ones take several launches
    constexpr int64_t MOST = ((int64_t{1} << 32) - 1) / THREADS;
    for (int64_t r = 0; r < a.rows; r += MOST * PER) {
        const int64_t left = (a.rows - r + PER - 1) / PER, grid = left < MOST ? left : MOST;
        launch_kernel(k_rms_norm<T, OUT, TPR, NP>, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, st, a, r);
    }
    return hipGetLastError();
}

template <typename T, int OUT>
hipError_t norm(const NormArgs& a, hipStream_t st) {
    if (a.cols <= 512) return norm<T, OUT, 64, 1>(a, st);
    if (a.cols <= 1024) return norm<T, OUT, 64, 2>(a, st);
    if (a.cols <= 2048) return norm<T, OUT, 256, 1>(a, st);
    if (a.cols <= 4096) return norm<T, OUT, 256, 2>(a, st);
    if (a.cols <= 8192) return norm<T, OUT, 256, 4>(a, st);
    if (a.cols <= 16384) return norm<T, OUT, 1024, 2>(a, st);
    if (a.cols <= 32768) return norm<T, OUT, 1024, 4>(a, st);
    return norm<T, OUT, 1024, 8>(a, st);
}

}  // namespace

hipError_t launch_rms_norm(int dtype, int out, const NormArgs& a, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    if (dtype == 0)
        return out == kQ8OutE4M3   ? norm<float, kQ8OutE4M3>(a, st)
               : out == kQ8OutE5M2 ? norm<float, kQ8OutE5M2>(a, st)
                                   : norm<float, kQ8OutF32>(a, st);
    return out == kQ8OutE4M3   ? norm<bf16_bits, kQ8OutE4M3>(a, st)
           : out == kQ8OutE5M2 ? norm<bf16_bits, kQ8OutE5M2>(a, st)
                               : norm<bf16_bits, kQ8OutBf16>(a, st);
}

}  // namespace clearmoe
