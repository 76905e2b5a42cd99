// Products of matrices in bfloat16 with float32 sums on the matrix cores of gfx950, for all workers in one launch.
//
//   C[m][n] = sum over segments, sum over k of A_seg[m][k] B_seg[n][k]
//
// Either operand may be stored with k contiguous ([m][k]) or with m contiguous ([k][m], template flags AT and BT).  A segment is a
// pair of operands of the same shape; several of them make a sum of products (dG Wg + dU Wu), and the float32 form, where a number
// is held as three bfloat16 terms and the six largest products of the terms are added: hi lo, lo hi, mid mid, hi mid, mid hi, hi hi.
//
// A block makes a tile of BM x BN with WM x WN waves.  Tiles of 64 along k go from memory straight into LDS (two buffers), 16 bytes a
// lane.  Bounds are those of the buffer descriptor: rows and columns that a matrix does not have come as zeros in both operands, so
// that nothing beyond an edge is read and no NaN that stands there reaches a sum.
// LDS layout, k contiguous: rows of 128 bytes, the 16-byte piece c of row r at place c ^ (r % 8), so that the sixteen rows that a
// fragment is read from fall on different banks.  m contiguous: 64 rows of BM elements, read by the transposing LDS load, piece c of
// row r at place c ^ 2 (r % 4 + 4 (r / 8 % 2)): the eight rows that half a wave reads from fall on different banks.
// Fragments go into the instruction as (B, A): a lane then has four consecutive n of one m, and after an exchange between the
// quarters of the wave sixteen, which it stores by 16 bytes.
#pragma once
#include "grawa_elements.h"
#include "grawa_sublayer.h"

typedef float grawa_f32x4 __attribute__((ext_vector_type(4)));
typedef short grawa_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 grawa_bf16x4 __attribute__((ext_vector_type(4)));

#define GRAWA_MAX_SEGS 12
#define GRAWA_BK 64

struct GrawaSeg {
    const char *p;  // worker 0
    int64_t worker; // bytes
};

struct GrawaGemm {
    int K;            // workers
    int M, N;         // of one worker; with two B operands N counts the columns of one
    int len;          // k of a segment, > 0; where k is contiguous a row holds zeros from there to the next multiple of 8
    int nseg;
    int64_t lda, ldb; // bytes between rows as stored, times 256 below 2^31
    GrawaSeg a[GRAWA_MAX_SEGS], b[GRAWA_MAX_SEGS]; // two B operands: the second's segments from nseg on
};

#define GRAWA_LDS __attribute__((address_space(3)))

// One operand's tile on its way to LDS.  R: rows (m or n) of the tile; NW: waves that share the loads.
template <bool TR, int R, int NW> struct GrawaTileLoad {
    static constexpr int LOADS = R * 128 / 1024 / NW;
    static_assert(LOADS * NW * 1024 == R * 128, "whole loads");
    static_assert(!TR || R >= 128, "the swizzle of a transposed tile takes sixteen pieces");
    uint32_t off[LOADS];
    uint32_t ld;
    int kpiece; // first k of the lane's piece (k contiguous only)

    __device__ __forceinline__ void init(int wave, int lane, uint32_t ld_)
    {
        ld = ld_;
        if constexpr (!TR) {
            const int c = (lane & 7) ^ (lane >> 3);
            kpiece = c * 8;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) off[i] = (uint32_t)((wave + NW * i) * 8 + (lane >> 3)) * ld + c * 16;
        } else {
            constexpr int PIECES = R / 8, RPL = 64 / PIECES;
            kpiece = 0;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = (wave + NW * i) * RPL + lane / PIECES, p = lane % PIECES;
                const int c = p ^ (((row & 3) | (((row >> 3) & 1) << 2)) << 1);
                off[i] = (uint32_t)row * ld + c * 16;
            }
        }
    }

    // base: of the tile's first row (k contiguous) or column (m contiguous) at k = 0; rows: of it that the matrix has, > 0; krem: k
    // that are left, > 0.  I0, I1: which of the loads.
    template <int I0, int I1> __device__ __forceinline__ void go(char *lds, int wave, const char *base, int k0, int rows, int krem) const
    {
        const char *b = TR ? base + (int64_t)k0 * ld : base + (int64_t)k0 * 2;
        const uint32_t valid = TR ? (uint32_t)((krem < GRAWA_BK ? krem : GRAWA_BK) - 1) * ld + (uint32_t)(((rows < R ? rows : R) + 7) & ~7) * 2
                                  : (uint32_t)((rows < R ? rows : R) - 1) * ld + (uint32_t)(((krem < GRAWA_BK ? krem : GRAWA_BK) + 7) & ~7) * 2;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)b, 0, valid, 0x00020000);
        const bool tail = !TR && krem < GRAWA_BK;
#pragma unroll
        for (int i = I0; i < I1; ++i) {
            uint32_t o = off[i];
            if (tail && kpiece >= krem) o = 0x80000000u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (GRAWA_LDS void *)(lds + (wave + NW * i) * 1024), 16, o, 0, 0, 0);
        }
    }
};

// Fragments of an operand's tile in LDS: 16 rows from row0 + 16 i on, k = 32 ks + 8 (lane / 16) ...
template <bool TR, int R, int N> struct GrawaFrag {
    uint32_t at[TR ? N : 2];

    __device__ __forceinline__ void init(int lane, int row0)
    {
        if constexpr (!TR) {
            const uint32_t p = ((uint32_t)(lane >> 4) ^ (lane & 7)) << 4;
            at[0] = (uint32_t)(row0 + (lane & 15)) * 128 + p;
            at[1] = at[0] ^ 64;
        } else {
            const int s = lane & 15, q = lane >> 4;
            const uint32_t key = (uint32_t)((s >> 2) | ((q & 1) << 2)) << 1;
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = (uint32_t)(q * 8 + (s >> 2)) * (R * 2) + ((((uint32_t)(row0 / 8 + 2 * i) + ((s & 3) >> 1)) ^ key) << 4) + (s & 1) * 8;
        }
    }

    __device__ __forceinline__ grawa_bf16x8 get(const char *lds, int i, int ks) const
    {
        if constexpr (!TR) {
            return *(const grawa_bf16x8 *)(lds + at[ks] + i * 2048);
        } else {
            const char *p = lds + at[i] + ks * 32 * R * 2;
            const grawa_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GRAWA_LDS grawa_s16x4 *)p);
            const grawa_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GRAWA_LDS grawa_s16x4 *)(p + 4 * R * 2));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(grawa_bf16x8, v);
        }
    }
};

// Which tile a block makes.  Blocks go round the eight XCDs; each XCD gets a run of consecutive tiles, in which GROUP rows of tiles
// are walked column by column, so that the tiles that are worked on at a time share rows and columns in that XCD's L2.
struct GrawaTile2 {
    int k, m, n;
};

__device__ __forceinline__ GrawaTile2 grawa_tile_of(uint32_t id, uint32_t total, uint32_t tm, uint32_t tn)
{
    constexpr uint32_t GROUP = 8;
    const uint32_t q = total / 8, r = total % 8, xcd = id % 8;
    const uint32_t t = xcd * q + (xcd < r ? xcd : r) + id / 8;
    const uint32_t k = t / (tm * tn), u = t - k * (tm * tn);
    const uint32_t g = u / (GROUP * tn), rows = tm - g * GROUP < GROUP ? tm - g * GROUP : GROUP, v = u - g * GROUP * tn;
    return GrawaTile2{(int)k, (int)(g * GROUP + v % rows), (int)(v / rows)};
}

// Rows of sixteen lanes: the odd ones of a change places with the even ones of b.
__device__ __forceinline__ void swap16(float &a, float &b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}

// The upper half of a changes places with the lower half of b.
__device__ __forceinline__ void swap32(float &a, float &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}

// The kernel.  DUAL: B is two operands, BN / 2 columns of each.  Epi: what becomes of the sums, see grawa_ffn.hip:
//   epi.tile(worker)                       once
//   epi.put16(m, n, v)                     sixteen columns from n on, m < M, n < N
//   epi.put8(m, n, v, u)                   DUAL: eight columns of both products
template <int BM, int BN, int WM, int WN, bool AT, bool BT, bool DUAL, class Epi>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_gemm(GrawaGemm g, Epi epi)
{
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
    static_assert(NI == 4, "a wave has 64 columns");
    constexpr int BR = DUAL ? BN / 2 : BN; // columns of B operand in a tile
    constexpr int ABYTES = BM * 128, BBYTES = BN * 128;
    __shared__ __attribute__((aligned(1024))) char buf0[ABYTES + BBYTES];
    __shared__ __attribute__((aligned(1024))) char buf1[ABYTES + BBYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const uint32_t tm = (uint32_t)(g.M + BM - 1) / BM, tn = (uint32_t)(g.N + BR - 1) / BR;
    const GrawaTile2 tile = grawa_tile_of(blockIdx.x, gridDim.x, tm, tn);
    const int m0 = tile.m * BM, n0 = tile.n * BR;

    GrawaTileLoad<AT, BM, NW> la;
    GrawaTileLoad<BT, BR, NW> lb; // of each B operand
    la.init(wave, lane, (uint32_t)g.lda);
    lb.init(wave, lane, (uint32_t)g.ldb);
    GrawaFrag<AT, BM, MI> fa;
    GrawaFrag<BT, BR, NI> fb;
    fa.init(lane, wm * TM);
    fb.init(lane, DUAL ? wn * (TN / 2) : wn * TN); // DUAL: fragments 0, 1 of the first operand, 2, 3 of the second

    const int64_t aoff = AT ? (int64_t)m0 * 2 : (int64_t)m0 * g.lda, boff = BT ? (int64_t)n0 * 2 : (int64_t)n0 * g.ldb;
    const int mrows = g.M - m0, nrows = g.N - n0;
    const int kt = (g.len + GRAWA_BK - 1) / GRAWA_BK, tiles = kt * g.nseg;
    int seg = 0, k0 = 0; // of the next tile to load
    auto load = [&](char *buf) {
        const char *pa = g.a[seg].p + tile.k * g.a[seg].worker + aoff, *pb = g.b[seg].p + tile.k * g.b[seg].worker + boff;
        const int krem = g.len - k0;
        la.template go<0, la.LOADS>(buf, wave, pa, k0, mrows, krem);
        lb.template go<0, lb.LOADS>(buf + ABYTES, wave, pb, k0, nrows, krem);
        if constexpr (DUAL) {
            const char *pc = g.b[g.nseg + seg].p + tile.k * g.b[g.nseg + seg].worker + boff;
            lb.template go<0, lb.LOADS>(buf + ABYTES + BR * 128, wave, pc, k0, nrows, krem);
        }
        k0 += GRAWA_BK;
        if (k0 >= g.len) {
            k0 = 0;
            ++seg;
        }
    };
    grawa_f32x4 acc[MI][NI] = {};
    auto compute = [&](const char *buf) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            grawa_bf16x8 b[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j)
                b[j] = DUAL ? fb.get(buf + ABYTES + (j >= 2 ? BR * 128 : 0), j & 1, ks) : fb.get(buf + ABYTES, j, ks);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const grawa_bf16x8 a = fa.get(buf, i, ks);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a, acc[i][j], 0, 0, 0);
            }
        }
    };
    load(buf0);
    __syncthreads(); // waits for the loads into LDS too
    for (int t = 0;;) {
        if (t + 1 < tiles) load(buf1);
        compute(buf0);
        __syncthreads();
        if (++t >= tiles) break;
        if (t + 1 < tiles) load(buf0);
        compute(buf1);
        __syncthreads();
        if (++t >= tiles) break;
    }

    epi.tile(tile.k);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int m = m0 + wm * TM + i * 16 + (lane & 15);
        float v[NI][4];
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) v[j][r] = acc[i][j][r];
        // Lane quarter q has n = 16 j + 4 q + r.
        if constexpr (DUAL) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                swap16(v[0][r], v[1][r]);
                swap16(v[2][r], v[3][r]);
            }
            const int q = lane >> 4, n = n0 + wn * (TN / 2) + ((q & 1) << 4) + ((q >> 1) << 3);
            if (m < g.M && n < g.N) epi.put8(m, n, v[0], v[2]); // v[0], v[1] and v[2], v[3] follow each other
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                swap32(v[0][r], v[2][r]);
                swap32(v[1][r], v[3][r]);
                swap16(v[0][r], v[1][r]);
                swap16(v[2][r], v[3][r]);
            }
            const int n = n0 + wn * TN + ((lane >> 4) << 4);
            if (m < g.M && n < g.N) epi.put16(m, n, v[0]);
        }
    }
}
