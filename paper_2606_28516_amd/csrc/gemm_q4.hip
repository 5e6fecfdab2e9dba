// Products with 4-bit matrices (q8.h: e2m1, a power-of-two scale for each 32
// values of k) on CDNA4's scaled matrix instructions: the scales of a block are
// operands of the instruction, so the sum stays in its float32 accumulators
// from the first block to the last.
//
// What those instructions add up exactly: eight products that follow each
// other along k are aligned to the largest of them and cut 14 bits below it,
// before the float32 sum.  Products of two e2m1 values lie between 2^-2 and 36
// in whole quarters, so none of them is cut: 4-bit rows give float32 sums.
// With 8-bit rows (e4m3) one instruction would lose 1.2e-5 of the result's norm
// on normal data, and small products beside large ones that cancel altogether.
// So products of them take two, one for the rows' values from 2 on (products
// from 2^-3 to 2688, in whole eighths) and one for those below (up to 11.25, in
// whole 2^-10), each of which cuts nothing.  That is the price of float32 sums:
// 32768 x 1024 x 4096 takes 177 us instead of 112.
#include <type_traits>

#include "q8_tile.h"

namespace clearmoe {

namespace {

__device__ __forceinline__ i32x8 q4_wide(const u32x4& a) {
    i32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = static_cast<int>(a[i]);
        f[i + 4] = 0;                            // (not read in the 4-bit form)
    }
    return f;
}
__device__ __forceinline__ i32x8 q4_join(const u32x4& a, const u32x4& b) {
    i32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = static_cast<int>(a[i]);
        f[i + 4] = static_cast<int>(b[i]);
    }
    return f;
}

// The e4m3 bytes of f whose magnitude is at least 2 (bit 6; NaN too), and the
// others: a mask of whole bytes from their bits 6, which the byte permutation
// spreads (its selectors 8 .. 11 are the signs of bytes 1 and 3).
__device__ __forceinline__ void q4_split(const i32x8& f, i32x8& high, i32x8& low) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = static_cast<uint32_t>(f[i]), m = __builtin_amdgcn_perm(u << 1, u << 9, 0x0b090a08u);
        high[i] = static_cast<int>(u & m);
        low[i] = static_cast<int>(u & ~m);
    }
}

// Words of four scale bytes whose blocks are not all there: 1 in the place of
// those past the end (their values are zeros, but their bytes may say NaN).
__device__ __forceinline__ uint32_t q4_scale_mask(int blocks) {
    return blocks >= 4 ? 0xffffffffu : blocks <= 0 ? 0u : (1u << (8 * blocks)) - 1;
}
__device__ __forceinline__ uint32_t q4_masked(uint32_t w, uint32_t mask) { return (w & mask) | (0x7f7f7f7fu & ~mask); }

template <int N>
__device__ __forceinline__ void q4_words(const unsigned char* p, uint32_t (&w)[N]) {
    __builtin_memcpy(w, __builtin_assume_aligned(p, N * 4), N * 4);
}

// How the instructions lay out k (measured): of a 4-bit operand, lane group g
// holds values 32 g .. 32 g + 31, of an 8-bit one 16 g .. 16 g + 15 and the
// sixteen that are half the instruction's k further; the scale of the block of
// 32 with the number g is lane group g's.

// ---------------------------------------------------------------------------
// A few rows: 16 rows x 16 columns, operands straight from memory into
// registers; eight waves share the sum (1 x 1536 x 384: 2.7 us in a graph, as
// an empty kernel).
// ---------------------------------------------------------------------------
__device__ __forceinline__ u32x4 q4_piece(const uint8_t* row, int64_t at, int64_t n, bool ok) {
    u32x4 a = {0u, 0u, 0u, 0u};
    if (ok && at < n) a = *reinterpret_cast<const u32x4*>(row + at);
    return a;
}

// a times b, all of it; 8-bit rows in the two parts.
template <int FA>
__device__ __forceinline__ f32x4 q4_mfma16(const i32x8& b, const i32x8& a, f32x4 acc, int sb, int sa) {
    if constexpr (FA != kQ8E2M1) {
        i32x8 h, l;
        q4_split(a, h, l);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, h, acc, kQ8E2M1, FA, 0, sb, 0, sa);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, l, acc, kQ8E2M1, FA, 0, sb, 0, sa);
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, kQ8E2M1, FA, 0, sb, 0, sa);
    }
}

// What a row tile's results are after the sums: bias, GELU, the row's type.
template <typename TC, int KW>
__device__ __forceinline__ void q4_rows_end(const Q8Desc& g, const GbTile& t, int n0, int tid,
                                            const float (&s_acc)[KW][16][20]) {
    const int m = tid / 16, c = tid % 16;
    if (m < t.rows && n0 + c < g.N) {
        float v = g.bias != nullptr ? g.bias[static_cast<int64_t>(t.seg) * g.N + n0 + c] : 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) v += s_acc[w][m][c];
        if (g.gelu) {
            float x[1] = {v};
            q4_gelu(x);
            v = x[0];
        }
        static_cast<TC*>(g.C)[(t.m_lo + m) * g.ldc + n0 + c] = Elem<TC>::from_f32(v);
    }
}

template <int FA, typename TC>
__global__ __launch_bounds__(512) void k_q4_rows(Q8Desc g, int mtiles, int ntiles) {
    constexpr int BM = 16, BN = 16, KW = 8, K128 = 128;
    constexpr bool A4 = FA == kQ8E2M1;
    __shared__ float s_acc[KW][BM][BN + 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, 1, lane, t)) return;
    const int n0 = t.nt * BN, n = n0 + row;
    const bool mok = row < t.rows, nok = n < g.N;
    const int64_t kb = q4_cols(g.K), ka = A4 ? kb : g.K;
    const int blocks = static_cast<int>(q4_blocks(g.K));
    const uint8_t* ar = g.A + (t.m_lo + (mok ? row : 0)) * g.lda;
    const uint8_t* br = g.B + t.seg * g.b_seg_stride + (nok ? n : 0) * kb;
    const uint8_t* sa = g.SA + (t.m_lo + (mok ? row : 0)) * g.sa_ld;
    const uint8_t* sb = g.SB + t.seg * g.sb_seg_stride + (nok ? n : 0) * g.sb_ld;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int nk = static_cast<int>(q8_blocks(g.K));
    for (int i = wave; i < nk; i += KW) {
        const bool in = 4 * i + grp < blocks;
        const i32x8 fb = q4_wide(q4_piece(br, static_cast<int64_t>(i) * 64 + grp * 16, kb, nok));
        const int xb = in ? sb[4 * i + grp] : kQ8One;
        i32x8 fa;
        int xa;
        if constexpr (A4) {
            fa = q4_wide(q4_piece(ar, static_cast<int64_t>(i) * 64 + grp * 16, ka, mok));
            xa = in ? sa[4 * i + grp] : kQ8One;
        } else {
            fa = q4_join(q4_piece(ar, static_cast<int64_t>(i) * K128 + grp * 16, ka, mok),
                         q4_piece(ar, static_cast<int64_t>(i) * K128 + 64 + grp * 16, ka, mok));
            xa = sa[i];
        }
        acc = q4_mfma16<FA>(fb, fa, acc, xb, xa);
    }
    // result v of a lane: column 4 grp + v of row `row`
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[wave][row][4 * grp + v] = acc[v];
    __syncthreads();
    q4_rows_end<TC, KW>(g, t, n0, tid < BM * BN ? tid : 16 * BM, s_acc);
}

template <int FA, typename TC>
hipError_t q4_rows(const Q8Desc& g, hipStream_t st) {
    const int64_t mt = (g.M + 15) / 16 + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + 15) / 16;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q4_rows<FA, TC>, dim3(static_cast<unsigned>(grid)), dim3(512), 0, st, g, static_cast<int>(mt),
                  static_cast<int>(nt));
    return hipGetLastError();
}

// A few rows of float32 or bfloat16, quantised by every workgroup for itself
// into LDS (rows of `pitch` bytes, then rows of `spitch` scale bytes), then as
// k_q4_rows.  The first blocks of B are on their way meanwhile, so a call is
// two trips to memory at most, which is what bounds it: 1 x 4096 x 1024 takes
// 4.3 us under a profiler and 1 x 1024 x 4096 5.8, the weights' bytes 0.45.
template <int FA, typename TA, typename TC>
__global__ __launch_bounds__(512) void k_q4_few(Q8Desc g, const TA* A, int K0, int mtiles, int ntiles, int pitch,
                                                int spitch) {
    constexpr int BM = 16, BN = 16, KW = 8, AHEAD = 4;
    constexpr bool A4 = FA == kQ8E2M1;
    extern __shared__ __attribute__((aligned(16))) unsigned char s_a[];
    __shared__ float s_acc[KW][BM][BN + 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, grp = lane >> 4;
    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, 1, lane, t)) return;
    const int n0 = t.nt * BN, n = n0 + row, nk = static_cast<int>(q8_blocks(g.K));
    const int blocks = static_cast<int>(q4_blocks(g.K));
    const int64_t kb = q4_cols(g.K);
    const bool nok = n < g.N, mok = row < t.rows;
    const uint8_t* br = g.B + t.seg * g.b_seg_stride + (nok ? n : 0) * kb;
    const uint8_t* sb = g.SB + t.seg * g.sb_seg_stride + (nok ? n : 0) * g.sb_ld;
    u32x4 fb[AHEAD];
    int xb[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int u = wave + i * KW;
        fb[i] = q4_piece(br, static_cast<int64_t>(u) * 64 + grp * 16, kb, nok);
        xb[i] = 4 * u + grp < blocks ? sb[4 * u + grp] : kQ8One;
    }
    // 16 lanes take 128 columns
    unsigned char* s_sa = s_a + t.rows * pitch;
    for (int u = tid / kQ8Lanes; u < t.rows * nk; u += 512 / kQ8Lanes) {
        const int m = u / nk, blk = u - m * nk, sub = tid % kQ8Lanes;
        float f[8];
        q8_load8(A + (t.m_lo + m) * K0, blk * kQ8Block + sub * 8, K0, f);
        if constexpr (A4) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w = max(w, q4_mag(f[i]));
            w = max(w, static_cast<uint32_t>(q8_partner<1>(static_cast<int>(w))));
            w = max(w, static_cast<uint32_t>(q8_partner<2>(static_cast<int>(w))));
            const int e = q4_exponent(w);
            *reinterpret_cast<uint32_t*>(s_a + m * pitch + blk * 64 + sub * 4) = q4_pack8(f, e);
            if (sub % 4 == 0) s_sa[m * spitch + blk * 4 + sub / 4] = static_cast<unsigned char>(e + kQ8One);
        } else {
            const float a = q8_max16(q8_mag8(f));
            const int e = q8_exponent(__float_as_uint(a), q8_top_exp(kQ8E4M3));
            *reinterpret_cast<uint2*>(s_a + m * pitch + blk * kQ8Block + sub * 8) =
                q8_pack8<kQ8E4M3>(f, q8_two_to(-e));
            if (sub == 0) s_sa[m * spitch + blk] = static_cast<unsigned char>(e + kQ8One);
        }
    }
    __syncthreads();
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const unsigned char* pa = s_a + (mok ? row : 0) * pitch;
    const unsigned char* ps = s_sa + (mok ? row : 0) * spitch;
    auto step = [&](int u, const u32x4& b, int scale) {
        i32x8 a;
        int xa;
        const u32x4 none = {0u, 0u, 0u, 0u};
        if constexpr (A4) {
            const u32x4 p = *reinterpret_cast<const u32x4*>(pa + u * 64 + grp * 16);
            a = q4_wide(mok ? p : none);
            xa = ps[u * 4 + grp];
        } else {
            const u32x4 p = *reinterpret_cast<const u32x4*>(pa + u * 128 + grp * 16);
            const u32x4 q = *reinterpret_cast<const u32x4*>(pa + u * 128 + 64 + grp * 16);
            a = q4_join(mok ? p : none, mok ? q : none);
            xa = ps[u];
        }
        acc = q4_mfma16<FA>(q4_wide(b), a, acc, scale, xa);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * KW < nk) step(wave + i * KW, fb[i], xb[i]);
    for (int u = wave + AHEAD * KW; u < nk; u += KW)
        step(u, q4_piece(br, static_cast<int64_t>(u) * 64 + grp * 16, kb, nok),
             4 * u + grp < blocks ? sb[4 * u + grp] : kQ8One);
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[wave][row][4 * grp + v] = acc[v];
    __syncthreads();
    q4_rows_end<TC, KW>(g, t, n0, tid < BM * BN ? tid : 16 * BM, s_acc);
}

// LDS bytes of a row quantised there: values (a whole number of 128 columns,
// and 16 so that rows do not share banks) and scales.
int64_t q4_few_pitch(int fa, int64_t K) { return q8_blocks(K) * (fa == kQ8E2M1 ? 64 : 128) + 16; }
int64_t q4_few_spitch(int fa, int64_t K) { return q8_blocks(K) * (fa == kQ8E2M1 ? 4 : 1); }

template <int FA, typename TA, typename TC>
hipError_t q4_few(const Q8Desc& g, const void* A, int K0, hipStream_t st) {
    const int64_t mt = (g.M + 15) / 16 + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + 15) / 16;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    const int64_t pitch = q4_few_pitch(FA, g.K), spitch = q4_few_spitch(FA, g.K), rows = g.M < 16 ? g.M : 16;
    launch_kernel(k_q4_few<FA, TA, TC>, dim3(static_cast<unsigned>(grid)), dim3(512),
                  static_cast<size_t>(rows * (pitch + spitch)), st, g, static_cast<const TA*>(A), K0,
                  static_cast<int>(mt), static_cast<int>(nt), static_cast<int>(pitch), static_cast<int>(spitch));
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Many rows: tiles through LDS.
// ---------------------------------------------------------------------------
template <int FA, int OB, int OA>
__device__ __forceinline__ f32x16 q4_mfma32(const i32x8& b, const i32x8& a, f32x16 acc, uint32_t sb, uint32_t sa) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, acc, kQ8E2M1, FA, OB, static_cast<int>(sb), OA,
                                                           static_cast<int>(sa));
}

// An operand's share of a stage in LDS: rows of SB bytes, their 16-byte chunks
// swizzled (gb_swz), brought by 16-byte loads, a wave of them at a time: RP
// rows.  koff: the byte of the row that a lane's chunk of an even or odd load
// is.
template <int SB>
struct Q4Rows {
    static constexpr int CPR = SB / 16, RP = 64 / CPR;
    static __device__ __forceinline__ int koff(int lane, int load) {
        const int lr = lane / CPR;
        return 16 * ((lane % CPR) ^ gb_swz<SB>(load * RP + lr));
    }
};

// KG groups of WM x WN waves of TM x TN MFMA tiles (32 x 32), KS values of k a
// stage, two stages in LDS for each group.  Scales come for 512 values of k at
// a time (16 bytes a row of a 4-bit operand, 4 of an 8-bit one: a load of one
// word of every row costs as much as 16 bytes), two such pieces in LDS.  The
// groups take the pieces of 512 in turn and their sums are added at the end.
//
// Measured on an MI355X, calls in a row: 4-bit rows 8192 x 8192 x 8192 to
// bfloat16 276 us (3980 TFLOP/s), 50432 x 1024 x 4096 126 (140 in one launch),
// 50432 x 4096 x 1024 with GELU to 4 bits 198; 8-bit rows, two instructions a
// product, 675 (1630), 300, and to e4m3 337.  Bounds: the large one takes 185 us
// without its matrix instructions (what 256 CUs take from the L2s) and 219
// without its loads (the card's power: these instructions alone, from registers,
// reach 6900 TFLOP/s on such data and 9900 on zeros), and the two overlap in
// part; over a short k the epilogue's vector work and stores: without GELU 155 of
// the 198, and 122 of those without the matrix instructions; of 8-bit rows the
// matrix instructions: 564 of the 675 without the loads, 271 without them.
// Four stages of half the k, loads and reads between the single matrix
// instructions, 16 waves on a CU, and workgroups that start half a tile apart
// were no faster.
template <int KG, int WM, int WN, int TM, int TN, int KS, int FA, int OUT, int WPE>
__global__ __launch_bounds__(64 * KG * WM * WN) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
void k_q4_tile(Q8Desc g, int mtiles, int ntiles, int group) {
    constexpr bool A4 = FA == kQ8E2M1;
    constexpr int NW = WM * WN, BM = WM * TM * 32, BN = WN * TN * 32;
    constexpr int SA = A4 ? KS / 2 : KS, SB = KS / 2;                   // bytes of a stage row
    constexpr int PER = 512 / KS, STEPS = KS / 64;                      // stages of a piece of scales, steps of a stage
    using RA = Q4Rows<SA>;
    using RB = Q4Rows<SB>;
    constexpr int AL = BM / (RA::RP * NW), BL = BN / (RB::RP * NW);
    static_assert((SA == 64 || SA == 128) && (SB == 64 || SB == 128), "a stage row is a line or half of one");
    static_assert(AL * RA::RP * NW == BM && BL * RB::RP * NW == BN, "whole loads per wave");
    static_assert(BM % 64 == 0 && BN % 64 == 0 && BM / 64 <= 2 * NW && BN / 64 <= 2 * NW, "scale loads");
    static_assert(kQ8Block % (TN * 32) == 0 && (OUT == kQ8OutF32 || OUT == kQ8OutBf16 || OUT == kQ8OutE2M1 ||
                                                BN % kQ8Block == 0),
                  "a wave's columns lie in one block, an 8-bit tile has whole blocks");
    static_assert(KG == 1 || OUT != kQ8OutE4M3, "the 8-bit epilogue has a barrier for all waves");
    constexpr int STAGE_A = BM * SA, STAGE = BM * SA + BN * SB, SOFF = 2 * STAGE;
    constexpr int SCA = BM * (A4 ? 16 : 4), SCALES = SCA + BN * 16;     // a piece of scales
    constexpr int EPI = NW * 32 * TN * 32 * (OUT == kQ8OutF32 ? 4 : OUT == kQ8OutBf16 ? 2 : 1);
    constexpr int SSIZE = 2 * SCALES > WN * BM * 4 ? 2 * SCALES : WN * BM * 4;
    constexpr int GROUP = SOFF + SSIZE, SUMS = NW * 64 * TM * TN * 64;
    static_assert(SOFF >= EPI && (KG == 1 || SOFF >= SUMS), "the epilogue's rows and the sums fit the stages");
    // the bias waits in the second piece's place, which is filled after the
    // first stage: whole loads of a word a lane
    constexpr int BIAS = TN <= 2 ? 256 : TN * 128, BOFF = SOFF + SCALES;
    static_assert(NW * BIAS <= SCALES, "a wave's columns each");
    __shared__ __attribute__((aligned(1024))) unsigned char smem_all[KG * GROUP];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave_all / NW, wave = wave_all % NW;
    unsigned char* smem = smem_all + kg * GROUP;
    const int wm = wave / WN, wn = wave % WN;
    const int lrow = lane & 31, lh = lane >> 5, K = g.K;

    GbTile t;
    if (!gb_tile<BM>(g, mtiles, ntiles, group, lane, t)) return;
    const int n0 = t.nt * BN;
    const int kb = static_cast<int>(q4_cols(K)), ka = A4 ? kb : K;      // bytes of a row
    const int blocks = static_cast<int>(q4_blocks(K));
    const int nk = (K + KS - 1) / KS, pieces = (nk + PER - 1) / PER;    // stages, pieces
    const int left_a = ka - (nk - 1) * SA, left_b = kb - (nk - 1) * SB; // bytes of the last stage
    // a group's pieces are kg, kg + KG ..; every group takes as many steps as
    // the first, which has the most stages (the barriers are for all)
    const int round = (pieces + KG - 1) / KG - 1, rest = nk - round * KG * PER;
    const int most = round * PER + (rest < PER ? rest : PER);
    auto stage_of = [&](int s) { return (s / PER * KG + kg) * PER + s % PER; };
    const uint32_t lda = static_cast<uint32_t>(g.lda);
    const int nrows = g.N - n0 < BN ? g.N - n0 : BN;
    const gb_i32x4 da = gb_desc(g.A + t.m_lo * g.lda, (static_cast<int64_t>(t.rows) - 1) * g.lda + ka);
    const gb_i32x4 db = gb_desc(g.B + t.seg * g.b_seg_stride + static_cast<int64_t>(n0) * kb,
                                static_cast<int64_t>(nrows) * kb);
    const gb_i32x4 dsa = gb_desc(g.SA + t.m_lo * g.sa_ld, static_cast<int64_t>(t.rows) * g.sa_ld);
    const gb_i32x4 dsb = gb_desc(g.SB + t.seg * g.sb_seg_stride + static_cast<int64_t>(n0) * g.sb_ld,
                                 static_cast<int64_t>(nrows) * g.sb_ld);
    constexpr int PA = AL > 1 ? 2 : 1, PB = BL > 1 ? 2 : 1;
    uint32_t va[PA], vb[PB];
    int ca[PA], cb[PB];                          // bytes of the row
#pragma unroll
    for (int p = 0; p < PA; ++p) {
        ca[p] = RA::koff(lane, wave * AL + p);
        va[p] = static_cast<uint32_t>(wave * AL * RA::RP + lane / RA::CPR) * lda + static_cast<uint32_t>(ca[p]);
    }
#pragma unroll
    for (int p = 0; p < PB; ++p) {
        cb[p] = RB::koff(lane, wave * BL + p);
        vb[p] = static_cast<uint32_t>((wave * BL * RB::RP + lane / RB::CPR) * kb + cb[p]);
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((gb_lds_u32*)smem)));
    // Rows past the tile's lie past the descriptors' ends and read zeros, and
    // so do the chunks past the end of a row in its last stage.
    auto dma = [&](int s, int b) {
        const int kt = stage_of(s);
        if (kt >= nk) return;
        const int soa = __builtin_amdgcn_readfirstlane(kt * SA), sob = __builtin_amdgcn_readfirstlane(kt * SB);
#pragma unroll
        for (int i = 0; i < AL; ++i) {
            const uint32_t v = kt == nk - 1 && ca[i % PA] >= left_a ? kGbOob : va[i % PA];
            gb_dma16(da, v + static_cast<uint32_t>(RA::RP * i) * lda, soa,
                     __builtin_amdgcn_readfirstlane(lds0 + b * STAGE + (wave * AL + i) * 1024));
        }
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const uint32_t v = kt == nk - 1 && cb[i % PB] >= left_b ? kGbOob : vb[i % PB];
            gb_dma16(db, v + static_cast<uint32_t>(RB::RP * i * kb), sob,
                     __builtin_amdgcn_readfirstlane(lds0 + b * STAGE + STAGE_A + (wave * BL + i) * 1024));
        }
        if (s % PER != 0) return;
        // a piece of scales: 64 rows a load
        const int p = kt / PER;
        const uint32_t at = lds0 + SOFF + ((s / PER) & 1) * SCALES;
#pragma unroll
        for (int i = 0; i < BM / 64; ++i)
            if (i % NW == wave) {
                const uint32_t v = static_cast<uint32_t>(i * 64 + lane) * static_cast<uint32_t>(g.sa_ld);
                if constexpr (A4)
                    gb_dma16(dsa, v, __builtin_amdgcn_readfirstlane(p * 16),
                             __builtin_amdgcn_readfirstlane(at + i * 1024));
                else
                    gb_dma4(dsa, v, __builtin_amdgcn_readfirstlane(p * 4),
                            __builtin_amdgcn_readfirstlane(at + i * 256));
            }
#pragma unroll
        for (int i = 0; i < BN / 64; ++i)
            if ((i + BM / 64) % NW == wave)
                gb_dma16(dsb, static_cast<uint32_t>(i * 64 + lane) * static_cast<uint32_t>(g.sb_ld),
                         __builtin_amdgcn_readfirstlane(p * 16),
                         __builtin_amdgcn_readfirstlane(at + SCA + i * 1024));
    };
    // the bias of the wave's columns (zeros past N)
    const uint32_t boff = BOFF + wave * BIAS;
    if (g.bias != nullptr && kg == 0) {
        const gb_i32x4 d = q8_bias_desc(g, t.seg);
#pragma unroll
        for (int h = 0; h < BIAS / 256; ++h)
            gb_dma4(d, static_cast<uint32_t>(n0 + wn * TN * 32 + h * 64 + lane) * 4u, 0,
                    __builtin_amdgcn_readfirstlane(lds0 + boff + h * 256));
    }
    dma(0, 0);
    dma(1, 1);

    const int bcol = gb_col_of_slot(lrow);
    // offsets of a step's chunks in a stage buffer (8 bits: of the first of the
    // two, the other is 32 bytes away)
    uint32_t oa[STEPS], ob[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int chunk = A4 ? 2 * s + lh : 4 * s + lh;
        oa[s] = static_cast<uint32_t>((wm * TM * 32 + lrow) * SA + ((chunk ^ gb_swz<SA>(lrow)) << 4));
        ob[s] = static_cast<uint32_t>(STAGE_A + (wn * TN * 32 + bcol) * SB + (((2 * s + lh) ^ gb_swz<SB>(bcol)) << 4));
    }
    u32x4 fa[2][A4 ? 1 : 2][TM], fb[2][TN];
    // scale words of the stage at hand, a lane's own byte first, and of the
    // next as they are read
    constexpr int SW = KS / 128, SWA = A4 ? SW : 1;
    uint32_t sa[TM][SWA], sb[TN][SW], ra[TM][SWA], rb[TN][SW];
    auto read = [&](int b, int s) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
            fb[s & 1][j] = *reinterpret_cast<const u32x4*>(smem + b * STAGE + ob[s] + j * 32 * SB);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            fa[s & 1][0][i] = *reinterpret_cast<const u32x4*>(smem + b * STAGE + oa[s] + i * 32 * SA);
            if constexpr (!A4)
                fa[s & 1][1][i] = *reinterpret_cast<const u32x4*>(smem + b * STAGE + (oa[s] ^ 32u) + i * 32 * SA);
        }
    };
    auto read_scales = [&](int s) {
        const unsigned char* p = smem + SOFF + ((s / PER) & 1) * SCALES;
        const int at = s % PER;                                         // stage of its piece
#pragma unroll
        for (int j = 0; j < TN; ++j)
            q4_words<SW>(p + SCA + (wn * TN * 32 + j * 32 + bcol) * 16 + at * SW * 4, rb[j]);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            q4_words<SWA>(p + (wm * TM * 32 + i * 32 + lrow) * (A4 ? 16 : 4) + (A4 ? at * SW * 4 : 0), ra[i]);
    };
    // what was read of stage s; past the last block, scales of 1
    auto take_scales = [&](int s) {
        const int have = blocks - stage_of(s) * SW * 4;
        if (have < SW * 4) {
#pragma unroll
            for (int w = 0; w < SW; ++w) {
                const uint32_t mask = q4_scale_mask(have - w * 4);
#pragma unroll
                for (int j = 0; j < TN; ++j) rb[j][w] = q4_masked(rb[j][w], mask);
                if constexpr (A4)
#pragma unroll
                    for (int i = 0; i < TM; ++i) ra[i][w] = q4_masked(ra[i][w], mask);
            }
        }
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int w = 0; w < SW; ++w) sb[j][w] = rb[j][w] >> (8 * lh);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int w = 0; w < SWA; ++w) sa[i][w] = ra[i][w] >> (A4 ? 8 * lh : 8 * (s % PER));
    };
    gb_wait_barrier<0>();                        // the bias and two stages have landed
    f32x16 acc[TM][TN];
    if (g.bias != nullptr && kg == 0) q8_start(lane, smem + boff, acc);
    else gb_zero(acc);
    read(0, 0);
    read_scales(0);
    auto mm = [&](auto step) {
        constexpr int S = decltype(step)::value, W = S / 2, OB = 2 * (S % 2), OA = A4 ? OB : 0;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (A4) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    acc[i][j] = q4_mfma32<FA, OB, OA>(q4_wide(fb[S & 1][j]), q4_wide(fa[S & 1][0][i]), acc[i][j],
                                                      sb[j][W], sa[i][W]);
        } else {
            // (row by row: both parts of one fragment at a time in registers)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                i32x8 part[2];
                q4_split(q4_join(fa[S & 1][0][i], fa[S & 1][1][i]), part[0], part[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = q4_mfma32<FA, OB, OA>(q4_wide(fb[S & 1][j]), part[h], acc[i][j], sb[j][W], sa[i][0]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int s0 = 0; s0 < most; s0 += 2) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int s = s0 + b;
            if (s >= most) break;
            const bool have = stage_of(s) < nk, next = s + 1 < most;
            take_scales(s);
            auto step = [&](auto at) {
                constexpr int S = decltype(at)::value;
                if constexpr (S + 1 < STEPS) {
                    read(b, S + 1);
                } else if (next) {
                    // stage s + 1 has landed for every wave, and every wave is
                    // done reading stage s's buffer, which takes s + 2
                    gb_wait_barrier<0>();
                    read(b ^ 1, 0);
                    read_scales(s + 1);
                    if (s + 2 < most) dma(s + 2, b);
                }
                if (have) mm(at);
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            if constexpr (STEPS == 4) {
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
            }
        }
    }
    gb_wait_barrier<0>();                        // the stage buffers are free
    if constexpr (KG > 1) {
        // the groups' sums, in order, through their own buffers
        if (kg > 0)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<f32x4*>(smem + (((wave * TM + i) * TN + j) * 4 + q) * 1024 + lane * 16) =
                            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int o = 1; o < KG; ++o)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 v = *reinterpret_cast<const f32x4*>(
                            smem + o * GROUP + (((wave * TM + i) * TN + j) * 4 + q) * 1024 + lane * 16);
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[i][j][4 * q + c] += v[c];
                    }
    }
    q8_epilogue<TM, TN, OUT, BM, true>(g, t, wm * TM * 32, n0 + wn * TN * 32, wn, lane, smem + wave * (EPI / NW),
                                 reinterpret_cast<float*>(smem + SOFF), acc);
}

// Row tiles that are taken column tile by column tile on one XCD (gb_tile).
constexpr int kQ4Group = 4;

template <int KG, int WM, int WN, int TM, int TN, int KS, int FA, int OUT, int WPE>
hipError_t q4_tile(const Q8Desc& g, hipStream_t st) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    const int64_t mt = (g.M + BM - 1) / BM + (g.seg_offsets != nullptr ? g.nseg : 0), nt = (g.N + BN - 1) / BN;
    const int64_t grid = (mt * nt + kGbXcds - 1) / kGbXcds * kGbXcds;
    launch_kernel(k_q4_tile<KG, WM, WN, TM, TN, KS, FA, OUT, WPE>, dim3(static_cast<unsigned>(grid)),
                  dim3(64 * KG * WM * WN), 0, st, g, static_cast<int>(mt), static_cast<int>(nt), kQ4Group);
    return hipGetLastError();
}

// Tiles of bm x bn of a product; a group ends inside a tile: half a tile more.
int64_t q4_tiles(const Q8Desc& g, int bm, int bn) {
    const int64_t groups = g.seg_offsets != nullptr ? g.nseg : 0;
    return ((g.M + bm - 1) / bm + groups / 2) * ((g.N + bn - 1) / bn);
}

// Which kernel: by the number of tiles, that is by how well each fills the
// chip's 256 CUs, and by k.  Times in us on an MI355X (calls in a row, N x K):
//   4-bit rows, bfloat16          rows of A   64     512    2048    8192   32768
//     1536 x 384    16 x 16 (rows)          3.7     6.7    20.4
//                   64 x 64 (small)         3.9     4.2     9.9    34.4     130
//                   64 x 128 (wide)         4.0     4.3     5.6    13.2    43.2
//                   128 x 128, 128 of k     4.7     4.9     5.6     9.3    26.7
//                   128 x 128, 256 of k     4.8     5.0     5.8    11.2    30.3
//                   256 x 256               7.1     8.3     8.9    10.7    29.9
//     1024 x 4096   16 x 16                 6.2    30.4     114
//                   64 x 64                 6.6     7.1    15.0    59.4     214
//                   64 x 128                9.7     9.9    11.6    31.6     122
//                   128 x 128, 128 of k    15.8    16.0    16.7    28.7     109
//                   128 x 128, 256 of k    12.9    13.2    13.9    24.1    89.6
//                   256 x 256              26.6    28.0    28.4    31.1    77.8
//   by tiles of 128 x 128 (256 x 256: a quarter), eight groups from 1056 on (with the second k)
//                                              320     512     600     752    1056    1360    2128    3200
//     K 576, 544    128 x 128, 128 of k          8.3     9.5    10.5    11.4    18.5    20.8    29.0    40.9
//                   128 x 128, 256 of k          8.6     9.7    12.5    12.9    19.5    22.9    31.6    43.8
//                   256 x 256                   10.9    11.7    11.8    12.4    24.1    24.1    35.8    47.7
//     K 2048, 4096  128 x 128, 128 of k         13.6    16.2    19.6    22.1    62.3    76.8     114     168
//                   128 x 128, 256 of k         12.4    14.6    19.7    20.7   57.3    65.7    99.9     141
//                   256 x 256                   17.5    19.0    19.3    20.0   66.8    67.6     103     141
//   the same, GELU, to 4 bits
//     4096 x 1024   128 x 128, 256 of k     7.9     8.2    11.5    36.4     136
//                   128 x 256              12.2    12.4    13.4    34.5     126
//                   256 x 256              16.1    16.8    17.2    35.1     135
//   8-bit rows, bfloat16
//     1536 x 384    16 x 16                 3.7     8.5    24.4
//                   64 x 64                 4.5     4.8    12.0
//                   64 x 128                4.9     5.1     6.7    17.2    54.0
//                   128 x 128               6.4     6.6     7.3    14.5    42.8
//                   128 x 256               8.9     9.2     9.9    15.5    38.4
//     1024 x 4096   16 x 16                 6.9    38.1     143
//                   64 x 64                12.0    12.6    25.7
//                   64 x 128               22.4    22.7    23.5    64.1     229
//                   64 x 128, two groups   15.7    15.9    18.0
//                   128 x 128              33.7    34.1    34.6    55.4     209
//                   128 x 256              50.7    51.2    51.9    54.4     177
//   by tiles of 128 x 256 (at N 384 a quarter of their columns is past N)
//                                             256     384     420     512     560     768    1024    1536
//     384 x 1536    128 x 128              22.9    33.6    33.3    34.5    41.8    52.7    65.2    96.2
//                   128 x 256              24.4    34.8    34.9    36.2    50.9    52.4    67.9    99.7
//     1024 x 1024   128 x 128              17.8    24.9    30.1    30.9    37.0    44.8    58.8    89.3
//                   128 x 256              19.1    26.2    26.4    27.9    37.9    40.0    51.2    76.0
//   8-bit rows, float32
//     1550 x 1200   64 x 64                 7.1     8.5    28.9    88.9
//                   64 x 128               10.7    11.1    16.5    49.4
//                   64 x 128, two groups    9.4     9.9    20.6    66.2
//                   128 x 128              14.9    16.6    18.9    49.1
//   64 x 128 and two groups along k, 2048 rows
//     8-bit rows    1024 x 640, 768, 1024, 2064     7.8   7.9,   8.3   8.2,   9.5   8.5,  14.6  11.9
//     4-bit rows    1024 x 1536, 2048, 4096         6.5   6.8,   7.4   7.3,  11.1  10.6
Q4Kernel q4_choose(const Q8Desc& g) {
    const bool a4 = g.fa == kQ8E2M1, f32 = g.out == kQ8OutF32, floats = f32 || g.out == kQ8OutBf16;
    if (floats && q4_tiles(g, 16, 16) <= 320) return kQ4Rows;
    // an 8-bit result's block needs 128 columns of a tile and all its waves
    const bool parts = g.out != kQ8OutE4M3;
    if (parts && q4_tiles(g, 64, 64) <= 256) return kQ4Small;
    const int64_t wide = q4_tiles(g, 64, 128);
    // (with a workgroup alone on its CU and a long sum, two groups of waves
    // along k)
    if (parts && wide <= 256 && g.K > (a4 ? 2048 : 640)) return kQ4Split;
    if (wide <= (a4 ? 400 : 512)) return kQ4Wide;
    if (f32) return a4 && g.K > 512 ? kQ4Deep : kQ4Middle;
    const int64_t tiles = q4_tiles(g, 128, 128);
    if (!a4) {
        // 512 places for 128 x 256, 768 for 128 x 128, of which the larger are
        // better by a tenth: not where a quarter of their columns lie past N
        const int64_t large = q4_tiles(g, 128, 256);
        return large >= 400 && tiles * 5 >= large * 8 ? kQ4Large : kQ4Middle;
    }
    // 4-bit rows: a CU holds three workgroups of 128 x 128 with stages of 128 of
    // k, two with 256 or of 128 x 256, one of 256 x 256; what runs in one round
    // of the chip less wins, but a long sum wants the larger tile or stage
    if (g.K <= 512) return kQ4Middle;
    if (tiles <= 512) return kQ4Deep;
    if (tiles <= 768 && g.K < 2048) return kQ4Middle;
    if (!floats) return q4_tiles(g, 128, 256) >= 400 ? kQ4Large : kQ4Deep;
    const int64_t large = q4_tiles(g, 256, 256), rounds = (large + 255) / 256;
    if (rounds == 1) return kQ4Large;
    if (g.K <= 640) return kQ4Middle;
    // three quarters of the rounds' places taken, or the last round's rows in a
    // launch of their own (q4_whole)
    if (large * 4 >= rounds * 768 || (g.seg_offsets == nullptr && (g.K >= 2048 || rounds > 2))) return kQ4Large;
    return kQ4Deep;
}

// 256 x 256 tiles, one a CU: a few more than the CUs have in whole rounds take
// a round of their own, so the rows past the whole rounds become a product of
// their own with the tiles that suit them, up to a quarter of a round or, with
// a sum long enough to hide the second launch, half of one.  One launch and two,
// us on an MI355X, N = 1024:
//   tiles / 256     1.02          1.12          1.25          1.5           3.08
//   K  544      24.1  19.9    23.8  21.1    23.7  22.9    24.3  25.8    46.9  43.7
//   K 2048      38.5  30.1    37.8  32.9    38.3  35.2    40.4  40.2    82.0  76.1
//   K 4096      65.1  48.3    64.8  53.0    65.3  58.0    68.3  66.2     140   127
// Tiles of 128 x 256, two a CU, win at 1.02 only (79 -> 71) and lose from 1.25 on
// (81 -> 85); a group's rows are not known here.
int64_t q4_whole(const Q8Desc& g) {
    if (q4_choose(g) != kQ4Large || g.fa != kQ8E2M1 || g.out != kQ8OutBf16 || g.seg_offsets != nullptr) return g.M;
    const int64_t nt = (g.N + 255) / 256, tiles = (g.M + 255) / 256 * nt;
    const int64_t whole = tiles / 256 * 256 / nt, rest = tiles - whole * nt;      // rows of tiles, tiles
    return whole > 0 && rest > 0 && rest <= (g.K >= 2048 ? 128 : 64) ? whole * 256 : g.M;
}

template <int FA, int OUT>
hipError_t q4_launch(const Q8Desc& g, hipStream_t st) {
    constexpr bool A4 = FA == kQ8E2M1, F32 = OUT == kQ8OutF32, BF16 = OUT == kQ8OutBf16;
    constexpr int KS = A4 ? 256 : 128;
    const Q4Kernel kernel = q4_choose(g);
    if constexpr (F32 || BF16)
        if (kernel == kQ4Rows) return q4_rows<FA, typename std::conditional<F32, float, bf16_bits>::type>(g, st);
    if constexpr (OUT != kQ8OutE4M3) {
        if (kernel == kQ4Small) return q4_tile<2, 2, 2, 1, 1, KS, FA, OUT, 2>(g, st);
        if (kernel == kQ4Split) return q4_tile<2, 2, 2, 1, 2, KS, FA, OUT, 2>(g, st);
    }
    if (kernel == kQ4Wide) return q4_tile<1, 2, 2, 1, 2, KS, FA, OUT, 2>(g, st);
    if constexpr (A4)
        if (kernel == kQ4Deep) return q4_tile<1, 2, 2, 2, 2, 256, FA, OUT, 2>(g, st);
    if constexpr (A4 && BF16)
        if (kernel == kQ4Large) return q4_tile<1, 2, 4, 4, 2, 256, FA, OUT, 2>(g, st);
    if constexpr (!F32 && !(A4 && BF16))
        if (kernel == kQ4Large) return q4_tile<1, 2, 2, 2, 4, 128, FA, OUT, 2>(g, st);
    return q4_tile<1, 2, 2, 2, 2, 128, FA, OUT, 3>(g, st);               // three workgroups on a CU
}

template <int FA>
hipError_t q4_out(const Q8Desc& g, hipStream_t st) {
    return g.out == kQ8OutF32    ? q4_launch<FA, kQ8OutF32>(g, st)
           : g.out == kQ8OutBf16 ? q4_launch<FA, kQ8OutBf16>(g, st)
           : g.out == kQ8OutE4M3 ? q4_launch<FA, kQ8OutE4M3>(g, st)
                                 : q4_launch<FA, kQ8OutE2M1>(g, st);
}

// The LDS that the quantised form of a few rows may take.
constexpr int64_t kQ4FewLds = 48 << 10;

template <int FA>
hipError_t q4_few_out(const Q8Desc& g, const void* A, bool a_f32, int K0, hipStream_t st) {
    if (g.out == kQ8OutF32)
        return a_f32 ? q4_few<FA, float, float>(g, A, K0, st) : q4_few<FA, bf16_bits, float>(g, A, K0, st);
    return a_f32 ? q4_few<FA, float, bf16_bits>(g, A, K0, st) : q4_few<FA, bf16_bits, bf16_bits>(g, A, K0, st);
}

}  // namespace

Q4Kernel q4_kernel(const Q8Desc& g) { return q4_choose(g); }
int64_t q4_whole_rows(const Q8Desc& g) { return q4_whole(g); }
bool q4_launch_fits(int64_t M, int N, int groups) {
    // many rows take 128 x 128 tiles over 256 threads at the least, or 256 x 256
    // over 512, for which a group's half tile more counts twice (the grid is
    // rounded up to whole XCDs)
    return ((M + 127) / 128 + 2 * static_cast<int64_t>(groups)) * q8_blocks(N) <= (int64_t{1} << 32) / 256 - 4 * kGbXcds;
}
bool q4_few_supported(int64_t M, int64_t K) {
    const int64_t rows = M < 16 ? M : 16;
    return M <= kQ8FewRows && rows * (q4_few_pitch(kQ8E4M3, K) + q4_few_spitch(kQ8E4M3, K)) <= kQ4FewLds;
}
hipError_t launch_q4_few(const Q8Desc& g, const void* A, bool a_f32, int K0, hipStream_t st) {
    if (g.M == 0) return hipSuccess;
    return g.fa == kQ8E2M1 ? q4_few_out<kQ8E2M1>(g, A, a_f32, K0, st) : q4_few_out<kQ8E4M3>(g, A, a_f32, K0, st);
}

hipError_t launch_gemm_q4(const Q8Desc& g, hipStream_t st) {
    if (g.M == 0) return hipSuccess;
    if (const int64_t rows = q4_whole(g); rows < g.M) {
        Q8Desc first = g, rest = g;              // (bfloat16)
        first.M = rows;
        rest.M -= rows;
        rest.A += rows * g.lda;
        rest.SA += rows * g.sa_ld;
        rest.C = static_cast<bf16_bits*>(g.C) + rows * g.ldc;
        const hipError_t e = q4_out<kQ8E2M1>(first, st);
        return e != hipSuccess ? e : q4_out<kQ8E2M1>(rest, st);
    }
    return g.fa == kQ8E2M1 ? q4_out<kQ8E2M1>(g, st) : q4_out<kQ8E4M3>(g, st);
}

}  // namespace clearmoe
