// Parts that the hand-scheduled MFMA products share (gfx950): buffer loads
// into LDS with counted waits, the swizzle of LDS rows, and the mapping of
// workgroups to tiles of (grouped) rows and columns.
#pragma once

#include "kernels.h"

namespace clearmoe {

namespace {

constexpr int kGbRow = 128;                      // bytes of k per stage row
constexpr int kGbXcds = 8;                       // MI355X: 8 XCDs of 32 CUs
constexpr uint32_t kGbOob = 0x80000000u;         // an offset past every operand here

typedef __attribute__((address_space(3))) uint32_t gb_lds_u32;
typedef int gb_i32x4 __attribute__((ext_vector_type(4)));

// Buffer descriptor of `bytes` bytes at p (uniform values): a load at an
// offset outside it returns zeros.
__device__ __forceinline__ gb_i32x4 gb_desc(const void* p, int64_t bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    gb_i32x4 d;
    d.x = __builtin_amdgcn_readfirstlane(static_cast<int>(a & 0xffffffffu));
    d.y = __builtin_amdgcn_readfirstlane(static_cast<int>((a >> 32) & 0xffffu));   // stride 0
    d.z = __builtin_amdgcn_readfirstlane(static_cast<int>(bytes));
    d.w = kRawWord3;
    return d;
}

// 16 bytes per lane, buffer -> LDS at m0 + 16 * lane.  Inline asm: the
// compiler does not count these loads, the pipeline's explicit waits do.
__device__ __forceinline__ void gb_dma16(const gb_i32x4& d, uint32_t voff, uint32_t soff, uint32_t m0) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(d), "s"(soff)
                 : "memory", "m0");
}

// 4 bytes per lane, buffer -> LDS at m0 + 4 * lane.
__device__ __forceinline__ void gb_dma4(const gb_i32x4& d, uint32_t voff, uint32_t soff, uint32_t m0) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :
                 : "s"(m0), "v"(voff), "s"(d), "s"(soff)
                 : "memory", "m0");
}

// Store of a finished row piece; nt: a streaming store past the L2.
__device__ __forceinline__ void gb_store(u32x4* p, const u32x4& v, bool nt) {
    if (nt) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// This wave's outstanding loads down to N, its LDS reads done, then the
// workgroup barrier.
template <int N>
__device__ __forceinline__ void gb_wait_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

// LDS rows of SB bytes hold their 16-byte chunk c at slot c ^ gb_swz(row):
// 16 consecutive rows of one chunk hit 16 different 16-byte bank groups.
template <int SB>
__device__ __forceinline__ int gb_swz(int r) {
    constexpr int CPR = SB / 16, RW = 16 / CPR;
    return (r / RW) % CPR;
}

// Column (within 32) that MFMA row slot s reads.  With B as the MFMA's first
// operand a lane's result v is row slot 8 (v/4) + 4 (lane/32) + v%4, so this
// order makes it column 16 (v/8) + 8 (lane/32) + v%8: eight consecutive
// columns per half of v.  (16 lanes still read 16 neighbouring rows.)
__device__ __forceinline__ int gb_col_of_slot(int s) {
    return 16 * (s >> 4) + 8 * ((s >> 2) & 1) + 4 * ((s >> 3) & 1) + (s & 3);
}

__device__ __forceinline__ int gb_incl_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);   // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);   // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);   // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31
    return v;
}

// Row tiles of bm rows that a segment takes (unsigned: of almost 2^31 rows the
// sum would pass an int).
__host__ __device__ constexpr int gb_row_tiles(int rows, int bm) {
    return static_cast<int>((static_cast<uint32_t>(rows) + static_cast<uint32_t>(bm - 1)) / static_cast<uint32_t>(bm));
}

// What a workgroup works on: rows [m_lo, m_lo + rows) of segment seg, column
// tile nt.
struct GbTile {
    int64_t m_lo;
    int rows, seg, nt;
};

// The tile of this workgroup (false: none, uniform over the workgroup); of g
// the rows M and the segments count (seg_offsets, nseg, seg_merge).
template <int BM, typename Desc>
__device__ __forceinline__ bool gb_tile(const Desc& g, int mtiles, int ntiles, int group, int lane,
                                        GbTile& t) {
    // XCD x = workgroup % 8 owns the row tiles x, x + 8, ... and takes them in
    // groups, column tile by column tile (shared A and B rows in its L2;
    // leading row tiles on every XCD); the last mtiles % 8 row tiles are
    // spread tile by tile, so that every XCD has its share
    const int xcd = blockIdx.x % kGbXcds, local = blockIdx.x / kGbXcds;
    const int m8 = mtiles / kGbXcds, full = m8 / group;
    int mt, nt;
    if (local < m8 * ntiles) {
        int mi;
        if (local < full * group * ntiles) {
            const int gi = local / (group * ntiles), r = local - gi * group * ntiles;
            mi = gi * group + r % group;
            nt = r / group;
        } else {
            const int r = local - full * group * ntiles, gm = m8 - full * group;
            mi = full * group + r % gm;
            nt = r / gm;
        }
        mt = mi * kGbXcds + xcd;
    } else {
        // the last mtiles % 8 row tiles, spread tile by tile over the XCDs
        const int r = (local - m8 * ntiles) * kGbXcds + xcd;
        mt = m8 * kGbXcds + r / ntiles;
        nt = r % ntiles;
        if (mt >= mtiles) return false;
    }
    int64_t m_lo, m_hi;
    int seg = 0;
    if (g.seg_offsets != nullptr && !g.seg_merge) {
        // lane s holds segment s (at most 64): a prefix sum of the segments'
        // row tiles and a ballot find this tile's segment.  Offsets are
        // clamped to [0, M]: bad ones cannot reach outside the buffers.
        const int M = static_cast<int>(g.M);
        int lo = lane < g.nseg ? g.seg_offsets[lane] : 0, hi = lane < g.nseg ? g.seg_offsets[lane + 1] : 0;
        lo = lo < 0 ? 0 : (lo > M ? M : lo);
        hi = hi < lo ? lo : (hi > M ? M : hi);
        const int n_t = gb_row_tiles(hi - lo, BM);
        const int tend = gb_incl_scan(n_t);
        const uint64_t hit = __ballot(lane < g.nseg && mt < tend);
        if (hit == 0) return false;
        seg = __builtin_ctzll(hit);
        const int t0 = __builtin_amdgcn_readlane(tend - n_t, seg);
        m_lo = __builtin_amdgcn_readlane(lo, seg) + static_cast<int64_t>(mt - t0) * BM;
        m_hi = __builtin_amdgcn_readlane(hi, seg);
    } else {
        int64_t lo = 0, hi = g.M;
        if (g.seg_offsets != nullptr) {
            lo = __builtin_amdgcn_readfirstlane(g.seg_offsets[0]);
            hi = __builtin_amdgcn_readfirstlane(g.seg_offsets[g.nseg]);
            lo = lo < 0 ? 0 : (lo > g.M ? g.M : lo);
            hi = hi < lo ? lo : (hi > g.M ? g.M : hi);
        }
        m_lo = lo + static_cast<int64_t>(mt) * BM;
        m_hi = hi;
        if (m_lo >= hi) return false;
    }
    t.m_lo = m_lo;
    t.rows = static_cast<int>(m_hi - m_lo < BM ? m_hi - m_lo : BM);
    t.seg = seg;
    t.nt = nt;
    return true;
}

template <int TM, int TN>
__device__ __forceinline__ void gb_zero(f32x16 (&acc)[TM][TN]) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
}

}  // namespace

}  // namespace clearmoe
