// Root-mean-square norm with the residual's addition:
//     h = x + residual (rounded to the rows' type: the stream that goes on),
//     y = h (mean(h^2) + eps)^(-1/2) weight,
// y in the rows' type or in 8 bits with a power-of-two scale for each 128
// columns (q8.h), rounded once from float32.
//
// One read of x and the residual, one write of h and y: bound by memory.  A
// row stays in registers between its sum and its scaling, up to 32768 columns
// (32 values a thread; of wider rows some spill).  Measured on an MI355X: 50432 x
// 1024 bfloat16 with the residual to e4m3 in 64 us (5.7 TB/s, where a large copy
// moves 5.0 to 5.2: part of the rows is still in the last-level cache), 1 x 768
// in 2.7 where an empty kernel takes 2.3.
#include "q8.h"

namespace clearmoe {

namespace {

constexpr int kNormThreads = 256;

// Eight elements from p on (any element).
__device__ __forceinline__ void norm_load8(const float* p, float (&v)[8]) { __builtin_memcpy(v, p, 32); }
__device__ __forceinline__ void norm_load8(const bf16_bits* p, float (&v)[8]) {
    u32x4 a;
    __builtin_memcpy(&a, p, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}

// N pieces of a row: piece p is its columns from c0 + step p on, zeros from
// cols on.  WHOLE (cols a multiple of 8): a piece is there or is not, and all
// loads are on their way before the first is used (a lane without one reads
// the row's last).
template <bool WHOLE, int N, typename T>
__device__ __forceinline__ void norm_load(const T* row, int c0, int step, int cols, float (&f)[N][8]) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int c = c0 + p * step;
        if constexpr (WHOLE) norm_load8(row + (c < cols ? c : cols - 8), f[p]);
        else q8_load8(row, c, cols, f[p]);
    }
    if constexpr (WHOLE)
#pragma unroll
        for (int p = 0; p < N; ++p)
            if (c0 + p * step >= cols)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[p][i] = 0.0f;
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void norm_store(T* row, int c, int cols, const float (&v)[8]) {
    if (!WHOLE || c < cols) q8_store8(row, c, WHOLE ? c + 8 : cols, v);
}

// h = f + g rounded to T.
template <typename T>
__device__ __forceinline__ void norm_add(float (&f)[8], const float (&g)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        f[i] += g[i];
        f[i + 1] += g[i + 1];
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = pack2_bf16(f[i], f[i + 1]);
            f[i] = __uint_as_float(w << 16);
            f[i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
}

// A wave's sum, the same in every lane.
template <int STEP>
__device__ __forceinline__ double norm_partner(double v) {
    const int2 w = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(double, make_int2(q8_partner<STEP>(w.x), q8_partner<STEP>(w.y)));
}
__device__ __forceinline__ double norm_sum(double s) {
    s += norm_partner<1>(s);
    s += norm_partner<2>(s);
    s += norm_partner<4>(s);
    s += norm_partner<8>(s);
    s += __shfl_xor(s, 16);
    return s + __shfl_xor(s, 32);
}

// TPR threads a row, NP pieces of eight columns a thread: piece p of thread t
// is columns 8 (p TPR + t) on, so that 16 threads side by side hold a block of
// 128.  TPR 64: a wave a row, four rows a workgroup.
template <typename T, int OUT, int TPR, int NP, bool WHOLE>
__global__ __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) void k_rms_norm(NormArgs a, int64_t first) {
    constexpr int THREADS = TPR > kNormThreads ? TPR : kNormThreads, WAVES = TPR / 64, STEP = 8 * TPR;
    // the weights are there when the sum is, and at most four pieces of a
    // second tensor on their way: the registers hold no more
    constexpr bool EARLY = NP <= 2;
    constexpr int G = NP < 4 ? NP : 4;
    const int t = threadIdx.x % TPR, c0 = 8 * t;
    const int64_t row = first + static_cast<int64_t>(blockIdx.x) * (THREADS / TPR) + threadIdx.x / TPR;
    if (TPR == 64 && row >= a.rows) return;      // (a whole wave; else a workgroup has one row, and exists)
    float f[NP][8], w[EARLY ? NP : 1][8];
    norm_load<WHOLE>(static_cast<const T*>(a.x) + row * a.ldx, c0, STEP, a.cols, f);
    if (EARLY && a.weight != nullptr) norm_load<WHOLE>(a.weight, c0, STEP, a.cols, w);
    if (a.residual != nullptr) {
        const T* r = static_cast<const T*>(a.residual) + row * a.ldr;
#pragma unroll
        for (int q = 0; q < NP; q += G) {
            float g[G][8];
            norm_load<WHOLE>(r, c0 + q * STEP, STEP, a.cols, g);
#pragma unroll
            for (int p = 0; p < G; ++p) norm_add<T>(f[q + p], g[p]);
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
    s = norm_sum(s);
    if constexpr (WAVES > 1) {
        __shared__ double s_sum[WAVES];
        if (threadIdx.x % 64 == 0) s_sum[threadIdx.x / 64] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) s += s_sum[v];
    }
    // (mean + eps)^(-1/2) in float32: mean + eps = m 4^k with m in [1/4, 1),
    // whose root is the hardware's (1 ulp); k = 0 of NaN and infinity
    const double mean = __builtin_fma(s, a.inv_cols, static_cast<double>(a.eps));
    int k = (__builtin_amdgcn_frexp_exp(mean) + 1) >> 1;
    const float root = __builtin_amdgcn_rsqf(static_cast<float>(__builtin_ldexp(mean, -2 * k)));
    if (a.sum != nullptr) {
        T* h = static_cast<T*>(a.sum) + row * a.lds;
#pragma unroll
        for (int p = 0; p < NP; ++p) norm_store<WHOLE>(h, c0 + p * STEP, a.cols, f[p]);
    }
    // root 2^-k is no normal number for the largest rows: those come down by
    // 2^8 first (what that rounds is far below their results' range)
    if (k > 126) {
        k -= 8;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[p][i] *= 0x1p-8f;
    }
    const float inv = __builtin_ldexpf(root, -k);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[p][i] *= inv;
    if (a.weight != nullptr) {
        if constexpr (EARLY) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[p][i] *= w[p][i];
        } else {
#pragma unroll
            for (int q = 0; q < NP; q += G) {
                float u[G][8];
                norm_load<WHOLE>(a.weight, c0 + q * STEP, STEP, a.cols, u);
#pragma unroll
                for (int p = 0; p < G; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[q + p][i] *= u[p][i];
                if (NP > 4) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if constexpr (OUT < kQ8OutE4M3) {
        T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
        for (int p = 0; p < NP; ++p) norm_store<WHOLE>(y, c0 + p * STEP, a.cols, f[p]);
    } else {
        constexpr int FMT = OUT == kQ8OutE4M3 ? kQ8E4M3 : kQ8E5M2;
        const int blocks = static_cast<int>(q8_blocks(a.cols)), vcols = static_cast<int>(q8_cols(a.cols));
        const int scols = static_cast<int>(q8_scale_cols(a.cols));
        uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.ldy;
        uint8_t* sc = a.scale + row * scols;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int c = c0 + p * STEP, blk = c / kQ8Block;
            // columns past the last hold zeros, NaN where the row's scale is
            // none: zeros again
            if (c + 8 > a.cols)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i >= a.cols) f[p][i] = 0.0f;
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[p][i]));
            // (infinities, which do not set a scale, are rare: the whole wave
            // looks again)
            if (__ballot(!(m < __builtin_inff())) != 0) m = q8_mag8(f[p]);
            m = q8_max16(m);
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
        launch_kernel(a.cols % 8 == 0 ? k_rms_norm<T, OUT, TPR, NP, true> : k_rms_norm<T, OUT, TPR, NP, false>,
                      dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, st, a, r);
    }
    return hipGetLastError();
}

// Threads a row.  More of them mean less work one after the other, which is
// what a few rows wait for, but also fewer rows at a time on a CU.  us on an
// MI355X, rows of bfloat16 with the residual to e4m3 (a wave; 256 threads;
// 1024):
//                  1 row              64 rows             many (50432 x 1024 values)
//   512      2.2   2.3   3.2    2.7   2.8   3.6    70   144   587
//   768      3.5   2.7   3.2    3.5   3.5   3.8    75   111   412
//   1024     2.7   2.4   3.3    3.2   2.8   3.6    64    86   302
//   2048     3.6   2.4   3.1    4.0   2.8   3.5    68    64   160
//   4096           3.3   3.2          3.5   3.7          68    96
//   8192           3.9   3.5          4.4   3.9          69    76
//   16384                4.2                4.9                81
//   32768                6.5                7.6                80
//   65536               16.8               20.7               112 (registers spill)
template <typename T, int OUT>
hipError_t norm(const NormArgs& a, hipStream_t st) {
    const bool few = a.rows <= 1024;
    if (a.cols <= 512) return norm<T, OUT, 64, 1>(a, st);
    if (a.cols <= 1024 && !few) return norm<T, OUT, 64, 2>(a, st);
    if (a.cols <= 2048) return norm<T, OUT, 256, 1>(a, st);
    if (a.cols <= 4096) return norm<T, OUT, 256, 2>(a, st);
    if (a.cols <= 8192 && !few) return norm<T, OUT, 256, 4>(a, st);
    if (a.cols <= 8192) return norm<T, OUT, 1024, 1>(a, st);
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
