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
// workgroup chooses the tokens' experts for itself, which costs less than a
// launch before it: logits by the matrix instructions on the x it holds
// anyway, with a bound on their error, and in double where the choice does not
// clear it.  The routing that is given out (and the gates, which need double)
// comes from workgroups beside, one a token, which only do that.
//
// Both kernels wait for memory (us on an MI355X under a profiler, where an
// empty kernel takes 2.3 to 2.8; the bytes alone 0.4 to 2.2 for both):
//                                                  hidden    out
//   1 token, 384 -> 1536, E = 8, k = 1, bfloat16     6.6     5.2
//   1 token, 768 -> 3072, E = 8, k = 2, bfloat16     8.2     5.3 to 6.4
//   16 tokens of these, adaptive router             12.6     7.6
// More tokens choose more experts: a wave has six 16-row tiles of Vt and Q
// where one token gives it three, which is most of what the first kernel grows
// by.  (Both experts of a token count, also where the adaptive router drops
// the second.)
// Slices of 16 or 64 hidden units, 256 or 1024 threads and the logits in double
// on the matrix instructions (2.2 us more) were slower.
#include "few.h"

namespace clearmoe {

namespace {

constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64;
constexpr int kOutThreads = 512;
constexpr int kSlice = 32;                // hidden units of a workgroup
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

__device__ __forceinline__ float few_elem(const u32x4& v, int i, float) { return __uint_as_float(v[i]); }
__device__ __forceinline__ float few_elem(const u32x4& v, int i, bf16_bits) {
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
}

// How rows are read: whole 16-byte pieces; pieces that may start at any
// element (the hardware loads them all the same); or, for rows shorter than a
// piece, element by element.
enum { kFewWhole, kFewPieces, kFewElems };

// Row elements [c, c + per16), zeros from column n on or with ok false.  The
// row's last, cut piece is read element by element.
template <typename T, int MODE>
__device__ __forceinline__ u32x4 few_load(const T* row, int64_t c, int64_t n, bool ok) {
    constexpr int PER16 = Elem<T>::per16;
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (MODE == kFewWhole) {
        if (ok && c < n) v = *reinterpret_cast<const u32x4*>(row + c);
    } else if (MODE == kFewPieces && ok && c + PER16 <= n) {
        __builtin_memcpy(&v, row + c, 16);
    } else if (ok && c < n) {
#pragma unroll
        for (int i = 0; i < PER16; ++i) {
            if (c + i >= n) break;
            if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(row[c + i]);
            else v[i >> 1] |= static_cast<uint32_t>(row[c + i]) << (16 * (i & 1));
        }
    }
    return v;
}
// The same for an operand whose partner is read in the same way, so that only
// the pairs of elements count: a cut last piece is the row's last whole one
// without the elements that came before.  (No branch: a load that some lanes
// take apart costs more than the rest of a step.)
template <typename T, int MODE>
__device__ __forceinline__ u32x4 few_pair(const T* row, int64_t c, int64_t n, bool ok) {
    constexpr int PER16 = Elem<T>::per16;
    if constexpr (MODE != kFewPieces) return few_load<T, MODE>(row, c, n, ok);
    u32x4 v = {0u, 0u, 0u, 0u};
    const int64_t at = c + PER16 <= n ? c : n - PER16;
    if (ok && c < n) __builtin_memcpy(&v, row + at, 16);
    const int skip = static_cast<int>(c - at);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4) v[w] = w >= skip ? v[w] : 0u;
        else v[w] = 2 * w >= skip ? v[w] : 2 * w + 1 >= skip ? v[w] & 0xffff0000u : 0u;
    }
    return v;
}

// |v| of each element of a piece.
__device__ __forceinline__ u32x4 few_abs(u32x4 v, float) { return v & 0x7fffffffu; }
__device__ __forceinline__ u32x4 few_abs(u32x4 v, bf16_bits) { return v & 0x7fff7fffu; }

// Logits of one token in double into lg[0 .. E) (LDS): an expert a wave.
template <typename T, int MODE>
__device__ __forceinline__ void few_logits(const FewArgs& a, const T* x, int wave, int lane, double* lg) {
    constexpr int PER16 = Elem<T>::per16;
    for (int e = wave; e < a.E; e += kFewWaves) {
        const T* w = static_cast<const T*>(a.Wg) + static_cast<int64_t>(e) * a.D;
        double s = 0.0;
        for (int64_t c = lane * PER16; c < a.D; c += 64 * PER16) {
            const u32x4 xv = few_pair<T, MODE>(x, c, a.D, true), wv = few_pair<T, MODE>(w, c, a.D, true);
#pragma unroll
            for (int i = 0; i < PER16; ++i)
                s += static_cast<double>(few_elem(xv, i, T{})) * static_cast<double>(few_elem(wv, i, T{}));
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
        if (lane == 0) lg[e] = s + (a.bg != nullptr ? static_cast<double>(a.bg[e]) : 0.0);
    }
}
// The k experts of logits lg[0 .. E) (LDS) into idx, by logit descending, ties
// to the lower index; all threads call it, barriers before and after are the
// caller's.  With NaN among them the routers' rule decides: one pick after the
// other, each from the first expert that is left on, which only a larger logit
// replaces.
__device__ __forceinline__ void few_choose(const double* lg, int E, int k, int tid, int32_t* idx) {
    if (tid >= E) return;
    const double l = lg[tid];
    int rank = 0;
    bool nan = false;
    for (int o = 0; o < E; ++o) {
        const double m = lg[o];
        rank += m > l || (m == l && o < tid);
        nan = nan || m != m;
    }
    if (!nan) {
        if (rank < k) idx[rank] = tid;
    } else if (tid == 0) {
        uint64_t taken = 0;
        for (int j = 0; j < k; ++j) {
            int best = -1;
            for (int e = 0; e < E; ++e)
                if ((taken >> e & 1u) == 0 && (best < 0 || lg[e] > lg[best])) best = e;
            taken |= 1ull << best;
            idx[j] = best;
        }
    }
}

// Routing of token t for the caller and the second kernel: choice and gates by
// the rule of the routers, all in double.
template <typename T, int MODE>
__device__ __forceinline__ void few_route(const FewArgs& a, int t, double* lg, double* ex, int32_t* idx) {
    const int tid = threadIdx.x, E = a.E, k = a.k;
    few_logits<T, MODE>(a, static_cast<const T*>(a.x) + static_cast<int64_t>(t) * a.D, tid >> 6, tid & 63, lg);
    __syncthreads();
    few_choose(lg, E, k, tid, idx);
    __syncthreads();
    if (tid < E) ex[tid] = exp(lg[tid] - lg[idx[0]]);
    __syncthreads();
    if (tid < k) {
        double all = 0.0, mine = 0.0;
        for (int e = 0; e < E; ++e) all += ex[e];
        const int kk = a.adaptive && 1.0 / all >= a.tau ? 1 : k;
        for (int j = 0; j < kk; ++j) mine += ex[idx[j]];
        const int64_t o = static_cast<int64_t>(t) * k + tid;
        a.idx[o] = tid < kk ? idx[tid] : -1;
        // a single renormalised expert has gate 1 whatever its logit
        a.gate[o] = tid >= kk ? 0.0f
                    : kk == 1 && a.renorm ? 1.0f
                                          : static_cast<float>(ex[idx[tid]] / (a.renorm ? mine : all));
    }
}

// Workgroup (slice, token group): z of HS hidden units for up to 16 tokens,
// then its share of t and the u_j.  The first `routes` workgroups of a group
// route a token each instead.  EG: 16-expert groups.
template <typename T, int MODE, int EG, int HS>
__global__ __launch_bounds__(kFewThreads) void k_few_hidden(FewArgs a, int routes) {
    constexpr int STEP = FewMfma<T>::step, PER16 = Elem<T>::per16;
    constexpr int HT = HS / 16, KW = kFewWaves / HT;          // row tiles of the slice, waves along D
    static_assert((HT == 2 || HT == 4) && kFewGroup * HS % kFewThreads == 0, "waves and values of z");
    constexpr int ZP = HS + PER16;                             // pitch of z rows: 16 bytes more
    constexpr bool LO = sizeof(T) == 2, VEC = MODE == kFewWhole;
    constexpr int NV = 2;                                      // tiles of Vt a wave fetches ahead
    __shared__ float s_part[2][kFewWaves][kFewGroup][16 * EG + 1];
    __shared__ __attribute__((aligned(16))) float s_lf[2][kFewGroup][16 * EG];
    __shared__ uint32_t s_key[kFewGroup][16 * EG];
    __shared__ double s_lg[kFewExperts], s_ex[kFewExperts];
    __shared__ float s_acc[KW][kFewGroup][HS + 1];
    __shared__ __attribute__((aligned(16))) T s_z[LO ? 2 : 1][kFewGroup][ZP];
    __shared__ int32_t s_idx[kFewGroup][kFewExperts];
    __shared__ unsigned long long s_used;
    __shared__ unsigned s_unsure;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    const int t0 = blockIdx.y * kFewGroup;
    const int nt = a.T - t0 < kFewGroup ? a.T - t0 : kFewGroup;
    const int slice = static_cast<int>(blockIdx.x) - routes;
    if (slice < 0) {
        if (static_cast<int>(blockIdx.x) < nt) few_route<T, MODE>(a, t0 + blockIdx.x, s_lg, s_ex, s_idx[0]);
        return;
    }
    const int h0 = slice * HS;
    const int D = a.D, H = a.H, E = a.E, k = a.k, r = a.r, q = a.q;
    const T* x = static_cast<const T*>(a.x) + static_cast<int64_t>(t0) * D;
    if (tid == 0) {
        s_used = 0;
        s_unsure = 0;
    }

    // ---- hidden slice: rows h of W1 times the tokens, and the logits: the HT
    // waves that hold the same part of x share it
    const int ht = wave % HT, kw = wave / HT;
    const int h = h0 + ht * 16 + row;
    const T* wrow = static_cast<const T*>(a.W1) + static_cast<int64_t>(h < H ? h : 0) * D;
    const T* xrow = x + static_cast<int64_t>(row < nt ? row : 0) * D;
    const T* Wg = static_cast<const T*>(a.Wg);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 lg[EG], lm[EG];                                      // logits, and the sums of magnitudes
#pragma unroll
    for (int g = 0; g < EG; ++g) lg[g] = lm[g] = acc;
    const int steps = (D + STEP - 1) / STEP;
    constexpr int UN = 8;
    u32x4 vt[NV];
    for (int s0 = kw; s0 < steps; s0 += KW * UN) {
        u32x4 wv[UN], xv[UN], gv[UN / HT];
        auto column = [&](int i) { return static_cast<int64_t>(s0 + i * KW) * STEP + grp * PER16; };
        auto experts = [&](int g) {
            const int e = 16 * g + row;
#pragma unroll
            for (int i = 0; i < UN / HT; ++i)
                gv[i] = few_pair<T, MODE>(Wg + static_cast<int64_t>(e < E ? e : 0) * D, column(HT * i + ht), D, e < E);
        };
#pragma unroll
        for (int i = 0; i < UN; ++i) wv[i] = few_pair<T, MODE>(wrow, column(i), D, h < H);
#pragma unroll
        for (int i = 0; i < UN; ++i) xv[i] = few_pair<T, MODE>(xrow, column(i), D, row < nt);
        if (!a.routed) experts(0);
        if (s0 == kw) {
            // what the second half needs first, in flight with the rest
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int n = (wave + v * kFewWaves) * 16 + row;
                vt[v] = few_load<T, MODE>(static_cast<const T*>(a.Vt) + static_cast<int64_t>(n < r ? n : 0) * H,
                                         h0 + grp * PER16, H, n < r);
            }
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) acc = FewMfma<T>::mma(wv[i], xv[i], acc);
        if (!a.routed) {
#pragma unroll
            for (int g = 0; g < EG; ++g) {
                if (16 * g >= E) break;
                if (g > 0) experts(g);
#pragma unroll
                for (int i = 0; i < UN / HT; ++i) {
                    u32x4 xs = xv[HT * i];
#pragma unroll
                    for (int w = 1; w < HT; ++w)
#pragma unroll
                        for (int c = 0; c < 4; ++c) xs[c] = ht == w ? xv[HT * i + w][c] : xs[c];
                    lg[g] = FewMfma<T>::mma(gv[i], xs, lg[g]);
                    lm[g] = FewMfma<T>::mma(few_abs(gv[i], T{}), few_abs(xs, T{}), lm[g]);
                }
            }
        }
    }
    // result v of a lane: hidden unit (expert) 4 grp + v, token row
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[kw][row][ht * 16 + 4 * grp + v] = acc[v];
    if (!a.routed)
#pragma unroll
        for (int g = 0; g < EG; ++g)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                s_part[0][wave][row][16 * g + 4 * grp + v] = lg[g][v];
                s_part[1][wave][row][16 * g + 4 * grp + v] = lm[g][v];
            }
    constexpr int ZN = kFewGroup * HS / kFewThreads;
    float bias[ZN];
#pragma unroll
    for (int i = 0; i < ZN; ++i) {
        const int c = h0 + (i * kFewThreads + tid) % HS;
        bias[i] = a.b1 != nullptr && c < H ? a.b1[c] : 0.0f;
    }
    __syncthreads();
    // z: the waves' sums, bias, GELU.  In bfloat16 z is kept as two parts, the
    // rounded value and what the rounding left (rounded too: 16 bits in all),
    // and both are multiplied: twice the (idle) matrix instructions, and t and u
    // are off by 2^-16 of z at most beside float32's sums.
#pragma unroll
    for (int i = 0; i < ZN; ++i) {
        const int t = (i * kFewThreads + tid) / HS, c = (i * kFewThreads + tid) % HS;
        float v = bias[i];
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
    // logits of (token, expert) and how far they may be off: a wave adds up
    // the products of its steps and then the waves' sums are added, each
    // addition off by 2^-23 of the magnitudes' sum at most (the instructions
    // may truncate), itself off as little; and what of a product or an addition
    // lies below the normal numbers may be lost, from the magnitudes too
    const float slack = static_cast<float>(STEP * (steps / kFewWaves + 2) + 2 * kFewWaves) * (0x1p-23f * 1.01f);
    const float lost = static_cast<float>(2 * STEP * steps + 4 * kFewWaves) * 0x1p-126f;
    if (!a.routed)
        for (int p = tid; p < nt * 16 * EG; p += kFewThreads) {
            const int t = p / (16 * EG), e = p % (16 * EG);
            float l = 0.0f, m = 0.0f;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                l += s_part[0][w][t][e];
                m += s_part[1][w][t][e];
            }
            const float b = a.bg != nullptr && e < E ? a.bg[e] : 0.0f;
            l += b;
            // keys order as the logits do (-0 is 0, NaN lowest); past the
            // last expert: below all of them, and far from everything
            const uint32_t u = __float_as_uint(l + 0.0f);
            s_key[t][e] = e >= E || l != l ? 0u : (u & 0x80000000u) != 0 ? ~u : u | 0x80000000u;
            s_lf[0][t][e] = e < E ? l : 0.0f;
            s_lf[1][t][e] = e < E ? (m + fabsf(b)) * slack + lost : -__builtin_inff();
        }
    __syncthreads();
    if (!a.routed) {
        for (int p = tid; p < nt * 16 * EG; p += kFewThreads) {
            const int t = p / (16 * EG), e = p % (16 * EG);
            if (e >= E) continue;
            // rank by logit descending, ties to the lower index; certain if
            // the logit differs from every other by more than both may be off
            // (never with NaN or infinities)
            const uint32_t key = s_key[t][e];
            const float l = s_lf[0][t][e], b = s_lf[1][t][e];
            int rank = 0, near = 0;
#pragma unroll
            for (int g = 0; g < EG; ++g) {
                if (16 * g >= E) break;
#pragma unroll
                for (int o4 = 0; o4 < 4; ++o4) {
                    const u32x4 ko = *reinterpret_cast<const u32x4*>(&s_key[t][16 * g + 4 * o4]);
                    const f32x4 lo = *reinterpret_cast<const f32x4*>(&s_lf[0][t][16 * g + 4 * o4]);
                    const f32x4 bo = *reinterpret_cast<const f32x4*>(&s_lf[1][t][16 * g + 4 * o4]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        rank += ko[i] > key || (ko[i] == key && 16 * g + 4 * o4 + i < e);
                        near += !(fabsf(lo[i] - l) > b + bo[i]);         // itself always
                    }
                }
            }
            if (rank >= k) continue;
            s_idx[t][rank] = e;
            if (near != 1) atomicOr(&s_unsure, 1u << t);
            else atomicOr(&s_used, 1ull << e);
        }
        __syncthreads();
        // the others again, in double
        for (unsigned left = s_unsure; left != 0; left &= left - 1) {
            const int t = __builtin_ctz(left);
            few_logits<T, MODE>(a, x + static_cast<int64_t>(t) * D, wave, lane, s_lg);
            __syncthreads();
            few_choose(s_lg, E, k, tid, s_idx[t]);
            __syncthreads();
            if (tid < k) atomicOr(&s_used, 1ull << s_idx[t][tid]);
            __syncthreads();
        }
    } else {
        for (int p = tid; p < nt * k; p += kFewThreads) {
            const int32_t e = a.idx[static_cast<int64_t>(t0) * k + p];
            s_idx[p / k][p % k] = e;
            if (e >= 0 && e < E) atomicOr(&s_used, 1ull << e);
        }
        __syncthreads();
    }

    // ---- shares of t (rows of Vt) and of u (rows of the chosen experts' Q)
    const int R = r + k * q;
    float* part = a.part + (static_cast<int64_t>(slice) * a.T + t0) * R;
    const int nvt = (r + 15) / 16, nq = (q + 15) / 16;
    u32x4 zf[LO ? 2 : 1][HS / STEP];
#pragma unroll
    for (int p = 0; p < (LO ? 2 : 1); ++p)
#pragma unroll
        for (int s = 0; s < HS / STEP; ++s)
            zf[p][s] = *reinterpret_cast<const u32x4*>(&s_z[p][row][s * STEP + grp * PER16]);
    constexpr int KS = 2;                                      // slots whose experts are held in registers
    int mine[KS];
#pragma unroll
    for (int j = 0; j < KS; ++j) mine[j] = j < k && row < nt ? s_idx[row][j] : -1;

    // The tiles of 16 rows: nvt of Vt, then nq of each chosen expert's Q; a
    // wave takes every kFewWaves-th of them.
    struct Tile {
        const T* m;           // its matrix
        int n, row0, e;       // rows of the matrix, first row of the tile, expert (-1: Vt)
    };
    uint64_t left = s_used;
    int at = wave;                                             // tile within the current matrix
    bool q_now = false;
    auto next = [&](Tile& t) {                                 // false: no more
        if (!q_now) {
            if (at < nvt) {
                t = Tile{static_cast<const T*>(a.Vt), r, at * 16, -1};
                at += kFewWaves;
                return true;
            }
            at -= nvt;
            q_now = true;
        }
        if (nq == 0) return false;
        while (left != 0 && at >= nq) {
            at -= nq;
            left &= left - 1;
        }
        if (left == 0) return false;
        const int e = __builtin_ctzll(left);
        t = Tile{static_cast<const T*>(a.Q) + static_cast<int64_t>(e) * q * H, q, at * 16, e};
        at += kFewWaves;
        return true;
    };
    auto load = [&](const Tile& t, int s) {
        const bool in = t.row0 + row < t.n;
        return few_load<T, MODE>(t.m + static_cast<int64_t>(in ? t.row0 + row : 0) * H, h0 + s * STEP + grp * PER16, H, in);
    };
    auto finish = [&](const Tile& t, const u32x4 (&v)[HS / STEP]) {
        f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < HS / STEP; ++s)
#pragma unroll
            for (int p = 0; p < (LO ? 2 : 1); ++p) c = FewMfma<T>::mma(v[s], zf[p][s], c);
        // Matrix instructions work for all lanes: they and the loads of their
        // operands must not be moved behind the branch below, which only some
        // lanes take.
        asm volatile("" : "+v"(c));
        // result v of a lane: matrix row row0 + 4 grp + v, token row
        if (row >= nt) return;
        float* pt = part + static_cast<int64_t>(row) * R;
        const int c0 = t.row0 + 4 * grp;
        auto store = [&](float* p) {
            if (VEC && c0 < t.n) {                             // whole groups of four, R a multiple of four
                *reinterpret_cast<f32x4*>(p + c0) = c;
            } else {
#pragma unroll
                for (int v2 = 0; v2 < 4; ++v2)
                    if (c0 + v2 < t.n) p[c0 + v2] = c[v2];
            }
        };
        if (t.e < 0) {
            store(pt);
        } else {
#pragma unroll
            for (int j = 0; j < KS; ++j)
                if (mine[j] == t.e) store(pt + r + j * q);
            for (int j = KS; j < k; ++j)
                if (s_idx[row][j] == t.e) store(pt + r + j * q);
        }
    };
    // A queue of tiles, the first of Vt fetched before: the loads of NQ tiles
    // are in flight while one is finished.  (One copy of the code: cold
    // instruction fetches are a good part of so short a kernel.)
    constexpr int NQ = 4;
    Tile tq[NQ];
    u32x4 mq[NQ][HS / STEP];
    int queued = 0;                                            // tiles not yet finished
#pragma unroll
    for (int b = 0; b < NQ; ++b)
        if (next(tq[b])) {
            ++queued;
#pragma unroll
            for (int s = 0; s < HS / STEP; ++s)
                mq[b][s] = s == 0 && b < NV && tq[b].e < 0 ? vt[b < NV ? b : 0] : load(tq[b], s);
        }
#pragma unroll 1
    for (; queued > 0; --queued) {
        finish(tq[0], mq[0]);
#pragma unroll
        for (int b = 0; b + 1 < NQ; ++b) {
            tq[b] = tq[b + 1];
#pragma unroll
            for (int s = 0; s < HS / STEP; ++s) mq[b][s] = mq[b + 1][s];
        }
        if (queued >= NQ && next(tq[NQ - 1])) {
            ++queued;
#pragma unroll
            for (int s = 0; s < HS / STEP; ++s) mq[NQ - 1][s] = load(tq[NQ - 1], s);
        }
    }
}

// Workgroup (rows of y, token): sums the slices' shares, then its rows of
// US t + sum_j gate_j P u_j + b2 in float32.  Its time is two trips to memory
// (routing and shares, the rows of US being fetched along with them; then P)
// and the sum's.
template <typename T, int MODE>
__global__ __launch_bounds__(kOutThreads) void k_few_out(FewArgs a, int S, int rows) {
    constexpr int PER16 = Elem<T>::per16, SPAN = 16 * PER16;    // columns that 16 lanes read at once
    constexpr bool VEC = MODE == kFewWhole;
    constexpr int W = VEC ? 4 : 1;                              // columns of the sums a thread takes
    constexpr int PU = 4;
    __shared__ __attribute__((aligned(16))) float s_red[kOutThreads * W];
    extern __shared__ __attribute__((aligned(16))) float s_v[];     // [r + k q]: t, then gate_j u_j
    typedef float vec __attribute__((ext_vector_type(W)));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // (the tokens are the grid's first dimension: the workgroups of one are on
    // one XCD when their number is a multiple of eight, and read its shares
    // from memory once)
    const int t = blockIdx.x, r = a.r, q = a.q, k = a.k, R = r + k * q, D = a.D;
    const int32_t* idx = a.idx + static_cast<int64_t>(t) * k;
    const float* gate = a.gate + static_cast<int64_t>(t) * k;
    // 16 lanes a row, four rows a wave: the first rows of US on their way
    const int sub = lane & 15;
    const int d0 = blockIdx.y * rows + wave * 4 + (lane >> 4);
    const int d1 = (blockIdx.y + 1) * rows < D ? (blockIdx.y + 1) * rows : D;
    u32x4 us[PU];
#pragma unroll
    for (int i = 0; i < PU; ++i)
        us[i] = few_load<T, MODE>(static_cast<const T*>(a.US) + static_cast<int64_t>(d0 < d1 ? d0 : 0) * r,
                                 sub * PER16 + i * SPAN, r, d0 < d1);
    const float bias = a.b2 != nullptr && d0 < d1 ? a.b2[d0] : 0.0f;
    // and the first pieces of P for the first slots
    constexpr int KS = 2;
    u32x4 ps[KS];
#pragma unroll
    for (int j = 0; j < KS; ++j) {
        const int e = j < k ? idx[j] : -1;
        const bool in = d0 < d1 && e >= 0 && e < a.E;
        ps[j] = few_load<T, MODE>(static_cast<const T*>(a.P) + (in ? static_cast<int64_t>(e) * D + d0 : 0) * q, sub * PER16, q, in);
    }

    // ---- the sums, S of them over G groups of threads
    const int C = R / W, G = C > 0 && C < kOutThreads ? kOutThreads / C : 1;
    const int g = C > 0 ? tid / C : 0;
    for (int c = G > 1 ? tid - g * C : tid; c < C && g < G; c += kOutThreads) {
        const float* p = a.part + static_cast<int64_t>(t) * R + c * W;
        const int64_t step = static_cast<int64_t>(a.T) * R;
        constexpr int UN = 24;                                 // loads in flight
        vec v = {};
        for (int s0 = g; s0 < S; s0 += UN * G) {
            vec m[UN];
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                m[i] = vec{};
                if (s0 + i * G < S) m[i] = *reinterpret_cast<const vec*>(p + (s0 + i * G) * step);
            }
#pragma unroll
            for (int i = 0; i < UN; ++i) v += m[i];
        }
        *reinterpret_cast<vec*>((G > 1 ? s_red + g * R : s_v) + c * W) = v;
        if (G > 1) break;
    }
    __syncthreads();
    for (int c = tid; c < R; c += kOutThreads) {
        float v = 0.0f;
        if (G > 1) {
            for (int i = 0; i < G; ++i) v += s_red[i * R + c];
        } else {
            v = s_v[c];
        }
        if (c >= r) {
            const int j = (c - r) / q;
            v = idx[j] >= 0 ? v * gate[j] : 0.0f;              // an empty slot's share was never summed
        }
        s_v[c] = v;
    }
    __syncthreads();
    for (int d = d0; d - (lane >> 4) < d1; d += kOutThreads / 16) {
        const bool in = d < d1;
        float v = 0.0f;
        auto add = [&](const u32x4& w, int c, int n, int at) {
#pragma unroll
            for (int i = 0; i < PER16; ++i)
                if (VEC ? c < n : c + i < n) v += few_elem(w, i, T{}) * s_v[at + c + i];
        };
        const T* row = static_cast<const T*>(a.US) + static_cast<int64_t>(in ? d : 0) * r;
        if (d == d0)
#pragma unroll
            for (int i = 0; i < PU; ++i) add(us[i], sub * PER16 + i * SPAN, r, 0);
        for (int c = sub * PER16 + (d == d0 ? PU * SPAN : 0); c < r; c += SPAN) add(few_load<T, MODE>(row, c, r, in), c, r, 0);
        for (int j = 0; j < k; ++j) {
            const int e = idx[j];
            if (e < 0 || e >= a.E) continue;
            const T* p = static_cast<const T*>(a.P) + (static_cast<int64_t>(e) * D + (in ? d : 0)) * q;
            if (d == d0 && j < KS) add(j == 0 ? ps[0] : ps[1], sub * PER16, q, r + j * q);
            for (int c = sub * PER16 + (d == d0 && j < KS ? SPAN : 0); c < q; c += SPAN)
                add(few_load<T, MODE>(p, c, q, in), c, q, r + j * q);
        }
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) v += __shfl_xor(v, m);
        if (in && sub == 0)
            static_cast<T*>(a.y)[static_cast<int64_t>(t) * D + d] =
                Elem<T>::from_f32(v + (d == d0 ? bias : a.b2 != nullptr ? a.b2[d] : 0.0f));
    }
}

template <typename T, int MODE>
hipError_t few_hidden(const FewArgs& a, hipStream_t st) {
    const int routes = a.routed ? 0 : a.T < kFewGroup ? a.T : kFewGroup;
    const dim3 grid(few_slices(a.H) + routes, (a.T + kFewGroup - 1) / kFewGroup);
    if (a.E <= 16) launch_kernel(k_few_hidden<T, MODE, 1, kSlice>, grid, dim3(kFewThreads), 0, st, a, routes);
    else launch_kernel(k_few_hidden<T, MODE, 4, kSlice>, grid, dim3(kFewThreads), 0, st, a, routes);
    return hipGetLastError();
}
template <typename T, int MODE>
hipError_t few_out(const FewArgs& a, hipStream_t st) {
    // rows of y a workgroup: a wave's passes take four rows each, and every
    // workgroup sums all shares again, so there are about as many workgroups
    // as compute units
    const int pass = kOutThreads / 16;
    const int most = 256 / a.T > 0 ? 256 / a.T : 1;
    const int rows = ((a.D + most - 1) / most + pass - 1) / pass * pass;
    const dim3 grid(a.T, (a.D + rows - 1) / rows);
    const size_t lds = sizeof(float) * (a.r + static_cast<size_t>(a.k) * a.q);
    launch_kernel(k_few_out<T, MODE>, grid, dim3(kOutThreads), lds > 0 ? lds : 4, st, a,
                  few_slices(a.H), rows);
    return hipGetLastError();
}

}  // namespace

int few_slices(int H) { return (H + kSlice - 1) / kSlice; }
size_t few_part_bytes(int64_t T, int H, int r, int k, int q) {
    return sizeof(float) * static_cast<size_t>(few_slices(H)) * static_cast<size_t>(T) *
           (static_cast<size_t>(r) + static_cast<size_t>(k) * static_cast<size_t>(q));
}
hipError_t launch_few_hidden(int dtype, bool whole, const FewArgs& a, hipStream_t st) {
    if (dtype == 0)
        return whole                      ? few_hidden<float, kFewWhole>(a, st)
               : a.D >= Elem<float>::per16 ? few_hidden<float, kFewPieces>(a, st)
                                           : few_hidden<float, kFewElems>(a, st);
    return whole                          ? few_hidden<bf16_bits, kFewWhole>(a, st)
           : a.D >= Elem<bf16_bits>::per16 ? few_hidden<bf16_bits, kFewPieces>(a, st)
                                           : few_hidden<bf16_bits, kFewElems>(a, st);
}
hipError_t launch_few_out(int dtype, bool whole, const FewArgs& a, hipStream_t st) {
    if (dtype == 0) return whole ? few_out<float, kFewWhole>(a, st) : few_out<float, kFewPieces>(a, st);
    return whole ? few_out<bf16_bits, kFewWhole>(a, st) : few_out<bf16_bits, kFewPieces>(a, st);
}

}  // namespace clearmoe
