// The whole CLEAR-MoE layer for a few tokens in two kernels (gfx950).
//
//     z = GELU(x W1^T + b1),  t = Vt z,  u_j = Q_{a_j} z        k_few_hidden
//     y = US t + b2 + sum_j gate_j P_{a_j} u_j                  k_few_out
//
// One token needs every weight of the shared path once and nothing twice, so
// what counts is how many dependent trips to memory a call makes, not its
// arithmetic.  The hidden width is cut into slices: a workgroup of the first
// kernel computes its slice of z (all of D is the sum), and from it the
// slice's share of t and u, which is summed over slices by the second kernel:
// z never leaves the chip and no workgroup waits for another.  Every
// workgroup routes for itself (E D products a token, in double), which costs
// less than a launch before it.
#include "few.h"

namespace clearmoe {

namespace {

constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64;
constexpr int kOutThreads = 512;
constexpr int kFewExperts = 64;

// 16 bytes per lane of each operand are one step along the sum: 32 bf16 or 16
// float32 of a 16-row tile.  Which of the step's values a lane holds does not
// matter as long as both operands agree: lane l has row l % 16 and the 16
// bytes at 16 (l / 16).
template <typename T> struct FewMfma;
template <> struct FewMfma<bf16_bits> {
    static constexpr int step = 32;
    __device__ static f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                       c, 0, 0, 0);
    }
};
template <> struct FewMfma<float> {
    static constexpr int step = 16;
    __device__ static f32x4 mma(const u32x4& a, const u32x4& b, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
};

// The 16 bytes of row elements [c, c + per16) (zeros from column n on, or
// with ok false).  VEC: rows are whole 16-byte pieces.
template <typename T, bool VEC>
__device__ __forceinline__ u32x4 few_load(const T* row, int64_t c, int64_t n, bool ok) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (VEC) {
        if (ok && c < n) v = *reinterpret_cast<const u32x4*>(row + c);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ok && c + i < n) v[i] = __float_as_uint(row[c + i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (ok && c + i < n) v[i >> 1] |= static_cast<uint32_t>(row[c + i]) << (16 * (i & 1));
    }
    return v;
}

__device__ __forceinline__ float few_elem(const u32x4& v, int i, float) { return __uint_as_float(v[i]); }
__device__ __forceinline__ float few_elem(const u32x4& v, int i, bf16_bits) {
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
}

// Choice of one token from its logits: the rule of the routers (by logit
// descending, ties to the lower index; a NaN never wins over the first expert
// left; adaptive and gate rules as clearmoe_router documents).
__device__ void few_select(const double* lg, const FewArgs& a, int32_t* idx, float* gate) {
    const int E = a.E, k = a.k;
    auto best_of = [&](uint64_t taken) {
        int best = -1;
        for (int e = 0; e < E; ++e)
            if (!((taken >> e) & 1u) && (best < 0 || lg[e] > lg[best])) best = e;
        return best;
    };
    const int top = best_of(0);
    double all = 0.0;                       // softmax denominator over every expert
    if (a.adaptive || !a.renorm) {
        double hi = lg[0];
        for (int e = 1; e < E; ++e)
            if (lg[e] > hi) hi = lg[e];
        for (int e = 0; e < E; ++e) all += exp(lg[e] - hi);
    }
    const int kk = a.adaptive && 1.0 / all >= a.tau ? 1 : k;
    uint64_t taken = 0;
    double den = 0.0;
    for (int j = 0; j < kk; ++j) {
        const int e = best_of(taken);
        taken |= uint64_t{1} << e;
        idx[j] = e;
        if (kk > 1) den += exp(lg[e] - lg[top]);
    }
    if (kk == 1 && a.renorm) {
        gate[0] = 1.0f;                     // whatever the logit
    } else {
        if (!a.renorm) den = all;
        for (int j = 0; j < kk; ++j) gate[j] = static_cast<float>(exp(lg[idx[j]] - lg[top]) / den);
    }
    for (int j = kk; j < k; ++j) {
        idx[j] = -1;
        gate[j] = 0.0f;
    }
}

// Workgroup (slice, token group): z of HS hidden units for up to 16 tokens,
// then its share of t and the u_j.
template <typename T, bool VEC, int HS>
__global__ __launch_bounds__(kFewThreads) void k_few_hidden(FewArgs a) {
    constexpr int STEP = FewMfma<T>::step, PER16 = Elem<T>::per16;
    constexpr int HT = HS / 16, KW = kFewWaves / HT;          // row tiles of the slice, waves along D
    static_assert(kFewWaves % HT == 0 && HS % STEP == 0, "waves and steps of a slice");
    constexpr int ZP = HS + PER16;                             // pitch of z rows: 16 bytes more
    constexpr bool LO = sizeof(T) == 2;
    __shared__ double s_lg[kFewGroup][kFewExperts + 1];
    __shared__ float s_acc[KW][kFewGroup][HS + 1];
    __shared__ __attribute__((aligned(16))) T s_z[LO ? 2 : 1][kFewGroup][ZP];
    __shared__ int32_t s_idx[kFewGroup][kFewExperts];
    __shared__ float s_gate[kFewGroup][kFewExperts];
    __shared__ unsigned long long s_used;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    const int t0 = blockIdx.y * kFewGroup;
    const int nt = a.T - t0 < kFewGroup ? a.T - t0 : kFewGroup;
    const int h0 = blockIdx.x * HS;
    const int D = a.D, H = a.H, E = a.E, k = a.k;
    const T* x = static_cast<const T*>(a.x) + static_cast<int64_t>(t0) * D;

    // ---- hidden slice: rows h of W1 times the tokens
    const int ht = wave % HT, kw = wave / HT;
    const int h = h0 + ht * 16 + row;
    const T* wrow = static_cast<const T*>(a.W1) + static_cast<int64_t>(h < H ? h : 0) * D;
    const T* xrow = x + static_cast<int64_t>(row < nt ? row : 0) * D;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (D + STEP - 1) / STEP;
    constexpr int UN = 8;
    for (int s0 = kw; s0 < steps; s0 += KW * UN) {
        u32x4 wv[UN], xv[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int64_t c = static_cast<int64_t>(s0 + i * KW) * STEP + grp * PER16;
            wv[i] = few_load<T, VEC>(wrow, c, D, h < H);
            xv[i] = few_load<T, VEC>(xrow, c, D, row < nt);
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) acc = FewMfma<T>::mma(wv[i], xv[i], acc);
    }
    // result v of a lane: hidden unit 4 grp + v, token row
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[kw][row][ht * 16 + 4 * grp + v] = acc[v];

    // ---- routing of the group's tokens
    if (!a.routed) {
        for (int p = wave; p < nt * E; p += kFewWaves) {
            const int t = p / E, e = p - t * E;
            const T* xr = x + static_cast<int64_t>(t) * D;
            const T* wr = static_cast<const T*>(a.Wg) + static_cast<int64_t>(e) * D;
            double s = 0.0;
            for (int64_t c = lane * PER16; c < D; c += 64 * PER16) {
                const u32x4 xv = few_load<T, VEC>(xr, c, D, true), wv = few_load<T, VEC>(wr, c, D, true);
#pragma unroll
                for (int i = 0; i < PER16; ++i)
                    s += static_cast<double>(few_elem(xv, i, T{})) * static_cast<double>(few_elem(wv, i, T{}));
            }
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
            if (lane == 0) s_lg[t][e] = s + (a.bg != nullptr ? static_cast<double>(a.bg[e]) : 0.0);
        }
    }
    if (tid == 0) s_used = 0;
    __syncthreads();
    // z: the waves' sums, bias, GELU.  In bfloat16 z is kept as two parts, the
    // rounded value and what the rounding left, and both are multiplied: twice
    // the (idle) matrix instructions, and t and u keep float32's accuracy.
    for (int i = tid; i < kFewGroup * HS; i += kFewThreads) {
        const int t = i / HS, c = i - t * HS;
        float v = a.b1 != nullptr && h0 + c < H ? a.b1[h0 + c] : 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) v += s_acc[w][t][c];
        v = h0 + c < H && t < nt ? gelu_erf(v) : 0.0f;
        const T hi = Elem<T>::from_f32(v);
        s_z[0][t][c] = hi;
        if constexpr (LO) {
            const float f = Elem<T>::to_f32(hi);
            s_z[1][t][c] = Elem<T>::from_f32(fabsf(f) < __builtin_inff() ? v - f : 0.0f);
        }
    }
    // the choice: a lane per token of the last wave
    const int ct = tid - (kFewThreads - 64);
    if (ct >= 0 && ct < nt) {
        int32_t* gi = a.idx + static_cast<int64_t>(t0 + ct) * k;
        uint64_t used = 0;
        if (!a.routed) {
            float* gg = a.gate + static_cast<int64_t>(t0 + ct) * k;
            few_select(s_lg[ct], a, s_idx[ct], s_gate[ct]);
            if (blockIdx.x == 0)
                for (int j = 0; j < k; ++j) {
                    gi[j] = s_idx[ct][j];
                    gg[j] = s_gate[ct][j];
                }
        } else {
            for (int j = 0; j < k; ++j) s_idx[ct][j] = gi[j];
        }
        for (int j = 0; j < k; ++j)
            if (s_idx[ct][j] >= 0) used |= uint64_t{1} << s_idx[ct][j];
        atomicOr(&s_used, static_cast<unsigned long long>(used));
    }
    __syncthreads();

    // ---- shares of t (rows of Vt) and of u (rows of the chosen experts' Q)
    const int r = a.r, q = a.q, R = r + k * q;
    float* part = a.part + (static_cast<int64_t>(blockIdx.x) * a.T + t0) * R;
    const int nvt = (r + 15) / 16, nq = (q + 15) / 16;
    const uint64_t used = s_used;
    const int tiles = nvt + __popcll(used) * nq;
    for (int tile = wave; tile < tiles; tile += kFewWaves) {
        int e = -1, row0 = tile * 16, n = r;
        const T* m = static_cast<const T*>(a.Vt);
        if (tile >= nvt) {
            uint64_t left = used;
            int s = (tile - nvt) / nq;
            while (s-- > 0) left &= left - 1;
            e = __builtin_ctzll(left);
            row0 = ((tile - nvt) % nq) * 16;
            n = q;
            m = static_cast<const T*>(a.Q) + static_cast<int64_t>(e) * q * H;
        }
        const T* mrow = m + static_cast<int64_t>(row0 + row < n ? row0 + row : 0) * H;
        f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < HS / STEP; ++s) {
            const u32x4 v = few_load<T, VEC>(mrow, h0 + s * STEP + grp * PER16, H, row0 + row < n);
            c = FewMfma<T>::mma(v, *reinterpret_cast<const u32x4*>(&s_z[0][row][s * STEP + grp * PER16]), c);
            if constexpr (LO)
                c = FewMfma<T>::mma(v, *reinterpret_cast<const u32x4*>(&s_z[1][row][s * STEP + grp * PER16]), c);
        }
        // Matrix instructions work for all lanes: they and the loads of their
        // operands must not be moved behind the branch below, which only some
        // lanes take.
        asm volatile("" : "+v"(c));
        // result v of a lane: matrix row row0 + 4 grp + v, token row
        if (row < nt) {
            float* pt = part + static_cast<int64_t>(row) * R;
            if (e < 0) {
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (row0 + 4 * grp + v < r) pt[row0 + 4 * grp + v] = c[v];
            } else {
                for (int j = 0; j < k; ++j)
                    if (s_idx[row][j] == e) {
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (row0 + 4 * grp + v < q) pt[r + j * q + row0 + 4 * grp + v] = c[v];
                    }
            }
        }
    }
}

// Workgroup (rows of y, token): sums the slices' shares, then its rows of
// US t + sum_j gate_j P u_j + b2 in float32.
template <typename T, bool VEC>
__global__ __launch_bounds__(kOutThreads) void k_few_out(FewArgs a, int S, int rows) {
    constexpr int PER16 = Elem<T>::per16;
    extern __shared__ __attribute__((aligned(16))) float s_v[];     // [r + k q]: t, then gate_j u_j
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int t = blockIdx.y, r = a.r, q = a.q, k = a.k, R = r + k * q, D = a.D;
    const int32_t* idx = a.idx + static_cast<int64_t>(t) * k;
    for (int c = tid; c < R; c += kOutThreads) {
        const int j = c < r ? -1 : (c - r) / q;
        float v = 0.0f;
        if (j < 0 || idx[j] >= 0) {
            const float* p = a.part + static_cast<int64_t>(t) * R + c;
            const int64_t step = static_cast<int64_t>(a.T) * R;
#pragma unroll 16
            for (int s = 0; s < S; ++s) v += p[s * step];
            if (j >= 0) v *= a.gate[static_cast<int64_t>(t) * k + j];
        }
        s_v[c] = v;
    }
    __syncthreads();
    // 16 lanes a row, four rows a wave
    const int sub = lane & 15;
    const int d1 = (blockIdx.x + 1) * rows < D ? (blockIdx.x + 1) * rows : D;
    for (int d0 = blockIdx.x * rows + wave * 4; d0 < d1; d0 += kOutThreads / 16) {
        const int d = d0 + (lane >> 4);
        const bool in = d < d1;
        float v = 0.0f;
        const T* us = static_cast<const T*>(a.US) + static_cast<int64_t>(in ? d : 0) * r;
        for (int c = sub * PER16; c < r; c += 16 * PER16) {
            const u32x4 w = few_load<T, VEC>(us, c, r, in);
#pragma unroll
            for (int i = 0; i < PER16; ++i)
                if (c + i < r) v += few_elem(w, i, T{}) * s_v[c + i];
        }
        for (int j = 0; j < k; ++j) {
            const int e = idx[j];
            if (e < 0) continue;
            const T* p = static_cast<const T*>(a.P) + (static_cast<int64_t>(e) * D + (in ? d : 0)) * q;
            for (int c = sub * PER16; c < q; c += 16 * PER16) {
                const u32x4 w = few_load<T, VEC>(p, c, q, in);
#pragma unroll
                for (int i = 0; i < PER16; ++i)
                    if (c + i < q) v += few_elem(w, i, T{}) * s_v[r + j * q + c + i];
            }
        }
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) v += __shfl_xor(v, m);
        if (in && sub == 0)
            static_cast<T*>(a.y)[static_cast<int64_t>(t) * D + d] =
                Elem<T>::from_f32(v + (a.b2 != nullptr ? a.b2[d] : 0.0f));
    }
}

constexpr int kSlice = 32;
constexpr int kOutRows = 32;

template <typename T, bool VEC>
hipError_t few_hidden(const FewArgs& a, hipStream_t st) {
    const dim3 grid((a.H + kSlice - 1) / kSlice, (a.T + kFewGroup - 1) / kFewGroup);
    launch_kernel(k_few_hidden<T, VEC, kSlice>, grid, dim3(kFewThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T, bool VEC>
hipError_t few_out(const FewArgs& a, hipStream_t st) {
    const dim3 grid((a.D + kOutRows - 1) / kOutRows, a.T);
    const size_t lds = sizeof(float) * (a.r + static_cast<size_t>(a.k) * a.q);
    launch_kernel(k_few_out<T, VEC>, grid, dim3(kOutThreads), lds > 0 ? lds : 4, st, a,
                  (a.H + kSlice - 1) / kSlice, kOutRows);
    return hipGetLastError();
}

}  // namespace

int few_slices(int, int H) { return (H + kSlice - 1) / kSlice; }
size_t few_part_bytes(int dtype, int64_t T, int H, int r, int k, int q) {
    return sizeof(float) * static_cast<size_t>(few_slices(dtype, H)) * static_cast<size_t>(T) *
           (static_cast<size_t>(r) + static_cast<size_t>(k) * static_cast<size_t>(q));
}
hipError_t launch_few_hidden(int dtype, bool aligned, const FewArgs& a, hipStream_t st) {
    if (dtype == 0) return aligned ? few_hidden<float, true>(a, st) : few_hidden<float, false>(a, st);
    return aligned ? few_hidden<bf16_bits, true>(a, st) : few_hidden<bf16_bits, false>(a, st);
}
hipError_t launch_few_out(int dtype, bool aligned, const FewArgs& a, hipStream_t st) {
    if (dtype == 0) return aligned ? few_out<float, true>(a, st) : few_out<float, false>(a, st);
    return aligned ? few_out<bf16_bits, true>(a, st) : few_out<bf16_bits, false>(a, st);
}

}  // namespace clearmoe
