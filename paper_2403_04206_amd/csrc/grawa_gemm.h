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
// Fragments go into the instruction as (B, A): a lane then has four consecutive n of one m.
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
    int K;            // workers; from `one` on those of a second product of the same shape with the same B
    int one;
    int M, N;         // of one worker; with two B operands N counts the columns of one
    int len;          // k of a segment, > 0; where k is contiguous a row holds zeros from there to the next multiple of 8
    int nseg;
    int splits;       // blocks that share a tile's sum, each a run of its tiles of 64 k
    int64_t lda, ldb; // bytes between rows as stored, times 256 below 2^31
    GrawaSeg a[GRAWA_MAX_SEGS], b[GRAWA_MAX_SEGS]; // a second product's A, two B operands: the second's segments from nseg on
};

#define GRAWA_LDS __attribute__((address_space(3)))

// One operand's tile on its way to LDS.  R: rows (m or n) of the tile; NW: waves that share the loads.
template <bool TR, int R, int NW> struct GrawaTileLoad {
    static constexpr int LOADS = R * 128 / 1024 / NW;
    static_assert(LOADS * NW * 1024 == R * 128, "whole loads");
    static_assert(!TR || R >= 128, "the swizzle of a transposed tile takes sixteen pieces");
    uint32_t first; // byte offset of the lane's piece in the wave's first load
    uint32_t odd;   // where loads take turns between two swizzles, that of the second
    uint32_t ld, step;
    int kpiece;     // first k of the lane's piece (k contiguous only)

    __device__ __forceinline__ void init(int wave, int lane, uint32_t ld_)
    {
        ld = ld_;
        if constexpr (!TR) {
            const int c = (lane & 7) ^ (lane >> 3);
            kpiece = c * 8;
            odd = 0;
            first = (uint32_t)(wave * 8 + (lane >> 3)) * ld + c * 16;
            step = NW * 8 * ld;
        } else {
            const int row = row_of(wave, lane), p = lane % (R / 8);
            kpiece = 0;
            first = (uint32_t)row * ld + (uint32_t)(p ^ key(row)) * 16;
            odd = TURN ? (uint32_t)(row + 8) * ld + (uint32_t)(p ^ key(row + 8)) * 16 : 0;
            step = (TURN ? 16 : NW * RPL) * ld;
        }
    }

    static constexpr int RPL = 512 / R;                    // rows of a transposed tile in a load
    static constexpr bool TURN = TR && NW * RPL == 8;      // a wave's loads are 8 rows apart: every other one has another swizzle
    static_assert(!TR || TURN || NW * RPL % 16 == 0, "the swizzles of a wave's loads");
    static __device__ __forceinline__ int row_of(int wave, int lane) { return wave * RPL + lane / (R / 8); }
    static __device__ __forceinline__ int key(int row) { return ((row & 3) | (((row >> 3) & 1) << 2)) << 1; }

    // Descriptor of what the tile has: b is the address of its first row (k contiguous) or column (m contiguous) at its first k, rows
    // (> 0) what the matrix has from there on, krem the k that are left; none: all comes as zeros and nothing is read.
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const char *b, int rows, int krem) const
    {
        const int kn = krem < GRAWA_BK ? krem : GRAWA_BK, rn = rows < R ? rows : R;
        const uint32_t valid = TR ? (uint32_t)(kn - 1) * ld + (uint32_t)((rn + 7) & ~7) * 2 : (uint32_t)(rn - 1) * ld + (uint32_t)((kn + 7) & ~7) * 2;
        return __builtin_amdgcn_make_buffer_rsrc((void *)b, 0, krem > 0 ? valid : 0, 0x00020000);
    }

    // Offset of the 128-byte line that a lane below PF asks for when a quarter of a tile's lines is fetched into L2 ahead of its loads.
    static constexpr int PF = R / 4 / NW;
    static __device__ __forceinline__ uint32_t line(int quarter, int wave, int lane, uint32_t ld)
    {
        const int i = quarter * (R / 4) + wave * PF + lane;
        return lane < PF ? (TR ? (uint32_t)(i / (R / 64)) * ld + (uint32_t)(i % (R / 64)) * 128 : (uint32_t)i * ld) : 0x80000000u;
    }
    static __device__ __forceinline__ void fetch(char *lds, __amdgpu_buffer_rsrc_t r, uint32_t at)
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (GRAWA_LDS void *)lds, 4, at, 0, 0, 0);
    }

    // Where the lane's first piece of a tile is; a piece behind the last k is another row's and comes as zeros, in this load and in those
    // that add a multiple of `step` (below 2^31) to it.
    __device__ __forceinline__ uint32_t place(int krem) const { return !TR && kpiece >= krem ? 0x80000000u : first; }

    template <int AUX = 0> __device__ __forceinline__ void go(int i, char *lds, int wave, __amdgpu_buffer_rsrc_t r, uint32_t at) const
    {
        if (TURN && i % 2) at = odd;
        asm("" : "+v"(at)); // the sum is formed where it is used: held in registers the sums would not fit
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (GRAWA_LDS void *)(lds + (wave + NW * i) * 1024), 16, at + (uint32_t)(TURN ? i / 2 : i) * step, 0, 0, AUX);
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
    int k, m, n, split;
};

__device__ __forceinline__ GrawaTile2 grawa_tile_of(uint32_t id, uint32_t total, uint32_t tm, uint32_t tn, uint32_t workers)
{
    constexpr uint32_t GROUP = 8;
    const uint32_t q = total / 8, r = total % 8, xcd = id % 8;
    const uint32_t t = xcd * q + (xcd < r ? xcd : r) + id / 8;
    const uint32_t ks = t / (tm * tn), u = t - ks * (tm * tn), split = ks / workers, k = ks - split * workers;
    const uint32_t g = u / (GROUP * tn), rows = tm - g * GROUP < GROUP ? tm - g * GROUP : GROUP, v = u - g * GROUP * tn;
    return GrawaTile2{(int)k, (int)(g * GROUP + v % rows), (int)(v / rows), (int)split};
}

// All but the wave's last N loads into LDS have landed and its reads from LDS are done; then the other waves' too.
template <int N> __device__ __forceinline__ void grawa_landed()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// c += a b with the sums where they are.  The builtin leaves it to the register allocator whether a sum stays in its registers; it moves
// them about, and the fragments then do not fit beside them.  The operands are waited for as any others' are.  What the compiler does
// not see is that c is still being written when the next instruction starts: between the first of these and the wait behind the last
// nothing else may touch a sum, a spill to memory least of all, and tests/test_product_kernels.py looks for that in what is built.
__device__ __forceinline__ void mfma_in_place(grawa_f32x4 &c, const grawa_bf16x8 &a, const grawa_bf16x8 &b)
{
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
}

// What becomes of the sums is up to an epilogue, see grawa_ffn.hip:
//   epi.tile(worker, split)              once
//   epi.ahead(mb, nb, lane, r)           asks for what the epilogue needs for a fragment, which is sixteen rows (and more) from its turn
//   epi.fragment(mb, nb, lane, r, v, u)  a fragment of 16 x 16 sums, rows 16 mb ..., columns 16 nb ...: the lane has row lane % 16, columns
//                                        4 (lane / 16) ...; v the product, u the second one where there are two.  Leaves in v, and
//                                        with OUTS = 2 in u, what goes on to
//   epi.put(o, m, n, v)                  VEC columns from n on of row m of output o; m < M, n < N
// Sixteen rows of NJ fragments of a wave.  A lane has four consecutive columns of one row of every fragment.  What goes to rows in memory
// passes through a corner of LDS of the wave's own, so that a store instruction writes whole runs of a row: straight from the
// fragments it would write 64 separate pieces of 16 bytes.  The 16-byte piece c of row r stands at place c ^ r.
struct GrawaNothing {};

template <int NJ, class Epi>
__device__ __forceinline__ void grawa_ahead(const Epi &epi, int m1, int n1, int lane, int M, int N, typename Epi::Ahead (&r)[NJ])
{
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        if (m1 < M && n1 + j * 16 < N) epi.ahead(m1 >> 4, (n1 >> 4) + j, lane, r[j]);
}

template <int NJ, class Epi>
__device__ __forceinline__ void grawa_finish(const Epi &epi, float *corner, int m1, int n1, int lane, int M, int N, const typename Epi::Ahead (&r)[NJ],
                                             grawa_f32x4 (&v)[NJ], grawa_f32x4 (&u)[NJ])
{
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        if (n1 + j * 16 < N) epi.fragment(m1 >> 4, (n1 >> 4) + j, lane, r[j], v[j], u[j]);
    if constexpr (Epi::OUTS > 0) {
        constexpr int COLS = NJ * 16, PIECES = COLS / 4, LPR = COLS / Epi::VEC, ROWS = 64 / LPR < 16 ? 64 / LPR : 16;
#pragma unroll
        for (int o = 0; o < Epi::OUTS; ++o)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int r = lane & 15, c = 4 * j + (lane >> 4);
                *(grawa_f32x4 *)(corner + o * 16 * COLS + r * COLS + (c ^ (r & (PIECES - 1))) * 4) = o ? u[j] : v[j];
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int o = 0; o < Epi::OUTS; ++o)
#pragma unroll
            for (int q = 0; q < 16 / ROWS; ++q) {
                const int r = q * ROWS + lane / LPR, n = n1 + lane % LPR * Epi::VEC;
                if (ROWS * LPR < 64 && lane >= ROWS * LPR) break;
                float w[Epi::VEC];
#pragma unroll
                for (int x = 0; x < Epi::VEC / 4; ++x) {
                    const int c = lane % LPR * (Epi::VEC / 4) + x;
                    const grawa_f32x4 t = *(const grawa_f32x4 *)(corner + o * 16 * COLS + r * COLS + (c ^ (r & (PIECES - 1))) * 4);
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[4 * x + y] = t[y];
                }
                if (m1 + r < M && n < N) epi.put(o, m1 + r, n, w);
            }
        __builtin_amdgcn_wave_barrier();
    }
}

namespace {

// The kernel: a tile a block.  DUAL: B is two operands, BN / 2 columns of each.  PAST: B is read past the caches.
// Bound by the matrix cores, and by the power that they draw: a tile of 256 x 256 reads an element from memory or L2 once for 256 products
// and from LDS once for 64 to 128, and its 128 KiB of two buffers leave a CU one block.  Reached with 8192 tokens, 4096 x 11264, in
// TFLOP/s: gate and up 1325, down 1397, dx 1442, weights' gradients 1290; a loop of nothing but matrix instructions 1600.  With a k as short
// as 1024 the epilogues, which nothing overlaps, take as long as the products: 8 x 2048 tokens, 1024 x 4096, gate and up 870, dH 515.
template <int BM, int BN, int WM, int WN, bool PAST, bool AT, bool BT, bool DUAL, class Epi>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_gemm([[maybe_unused]] GrawaGemm g, [[maybe_unused]] Epi epi)
{
#ifdef __HIP_DEVICE_COMPILE__ // the host pass needs the signature alone; given this body it leaves the launch stubs out without a word
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
    constexpr int NG = DUAL ? NI / 2 : NI; // fragments of a B operand
    constexpr int BR = DUAL ? BN / 2 : BN; // columns of B operand in a tile
    constexpr int ABYTES = BM * 128, BBYTES = BN * 128;
    __shared__ __attribute__((aligned(1024))) char buf0[ABYTES + BBYTES];
    __shared__ __attribute__((aligned(1024))) char buf1[ABYTES + BBYTES];
    __shared__ __attribute__((aligned(1024))) char unread[NW * 256]; // where lines that are only asked for go
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const uint32_t tm = (uint32_t)(g.M + BM - 1) / BM, tn = (uint32_t)(g.N + BR - 1) / BR;
    const GrawaTile2 tile = grawa_tile_of(blockIdx.x, gridDim.x, tm, tn, (uint32_t)g.K);
    const int m0 = tile.m * BM, n0 = tile.n * BR;
    const int worker = tile.k < g.one ? tile.k : tile.k - g.one, a_seg = tile.k < g.one ? 0 : g.nseg;

    GrawaTileLoad<AT, BM, NW> la;
    GrawaTileLoad<BT, BR, NW> lb; // of each B operand
    la.init(wave, lane, (uint32_t)g.lda);
    lb.init(wave, lane, (uint32_t)g.ldb);
    GrawaFrag<AT, BM, MI> fa;
    GrawaFrag<BT, BR, NG> fb;
    fa.init(lane, wm * TM);
    fb.init(lane, wn * NG * 16); // DUAL: the first NG fragments are of the first operand

    const int64_t aoff = AT ? (int64_t)m0 * 2 : (int64_t)m0 * g.lda, boff = BT ? (int64_t)n0 * 2 : (int64_t)n0 * g.ldb;
    const int mrows = g.M - m0, nrows = g.N - n0;
    const int kt = (g.len + GRAWA_BK - 1) / GRAWA_BK, all = kt * g.nseg;
    const int t0 = (int)((int64_t)all * tile.split / g.splits), tiles = (int)((int64_t)all * (tile.split + 1) / g.splits) - t0;
    const int64_t astep = AT ? GRAWA_BK * g.lda : GRAWA_BK * 2, bstep = BT ? GRAWA_BK * g.ldb : GRAWA_BK * 2;
    int seg = t0 / kt, skip = t0 - seg * kt, todo = tiles, krem = 0; // of the next tile to load
    const char *pa = nullptr, *pb = nullptr, *pc = nullptr;
    __amdgpu_buffer_rsrc_t ra, rb, rc;
    int kload = 0;             // k that the tile in the descriptors has
    uint32_t oa = 0, ob = 0;   // the lane's places in it
    // The next tile's descriptors, in steps that find room between matrix instructions.
    auto prepare = [&](int what) {
        if (what == 0) {
            if (krem <= 0 && todo > 0) {
                pa = g.a[a_seg + seg].p + worker * g.a[a_seg + seg].worker + aoff + skip * astep;
                pb = g.b[seg].p + worker * g.b[seg].worker + boff + skip * bstep;
                if (DUAL) pc = g.b[g.nseg + seg].p + worker * g.b[g.nseg + seg].worker + boff + skip * bstep;
                krem = g.len - skip * GRAWA_BK;
                skip = 0;
                ++seg;
            }
            kload = todo > 0 ? krem : 0;
            krem -= GRAWA_BK;
            --todo;
        } else if (what == 1) {
            ra = la.rsrc(pa, mrows, kload);
            oa = la.place(kload);
            pa += astep;
        } else if (what == 2) {
            rb = lb.rsrc(pb, nrows, kload);
            ob = lb.place(kload);
            pb += bstep;
        } else if (DUAL) {
            rc = lb.rsrc(pc, nrows, kload);
            pc += bstep;
        }
    };
    // The tiles behind the one whose loads are under way are asked for a tile early, so that the loads find them in L2: the blocks that
    // share rows (columns) of an operand take a quarter of its lines each, a dword a line, into a corner that nobody reads.  8 workers,
    // 2048 x 1024 x 4096, operands not in any cache: 126 us without, 108 with; two or four tiles early 108, 110.
    const uint32_t line_a = la.line(tile.n & 3, wave, lane, la.ld), line_b = lb.line(tile.m & 3, wave, lane, lb.ld);
    constexpr int FETCHES = DUAL ? 3 : 2;
    auto fetch = [&](int what) {
        const int left = todo > 0 ? kload - GRAWA_BK : 0; // of this segment: its end is not looked beyond
        if (what == 0)
            la.fetch(unread + wave * 256, la.rsrc(pa, mrows, left), line_a);
        else if (what == 1)
            lb.fetch(unread + wave * 256, lb.rsrc(pb, nrows, left), line_b);
        else
            lb.fetch(unread + wave * 256, lb.rsrc(pc, nrows, left), line_b);
    };
    constexpr int LA = GrawaTileLoad<AT, BM, NW>::LOADS, LB = GrawaTileLoad<BT, BR, NW>::LOADS, LOADS = LA + LB * (DUAL ? 2 : 1);
    auto load = [&](char *buf, int i) {
        if (i < LA)
            la.go(i, buf, wave, ra, oa);
        else if (i < LA + LB)
            lb.template go<PAST ? 2 : 0>(i - LA, buf + ABYTES, wave, rb, ob);
        else
            lb.template go<PAST ? 2 : 0>(i - LA - LB, buf + ABYTES + BR * 128, wave, rc, ob);
    };
    grawa_f32x4 acc[MI][NI] = {};
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) asm volatile("" : "+v"(acc[i][j])); // zero from here on, two instructions at least before the first use
    constexpr int MH = MI / 2;
    grawa_bf16x8 a0[MH], a1[MH], b0[NI], b1[NI];
    // A group: MH rows of NI matrix instructions, and between them, evenly, n other things to do.
    auto group = [&](int mh, const grawa_bf16x8 (&a)[MH], const grawa_bf16x8 (&b)[NI], int n, const auto &item) {
        constexpr int PAIRS = MH * NI / 2;
#pragma unroll
        for (int p = 0; p < PAIRS; ++p) {
            const int i = 2 * p / NI, j = 2 * p % NI;
            __builtin_amdgcn_sched_barrier(0);
            mfma_in_place(acc[mh * MH + i][j], b[j], a[i]);
            mfma_in_place(acc[mh * MH + i][j + 1], b[j + 1], a[i]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = p * n / PAIRS; x < (p + 1) * n / PAIRS; ++x) item(x);
        }
    };
    auto read_b = [&](const char *buf, int j, int ks) { return fb.get(buf + ABYTES + (j >= NG ? BR * 128 : 0), j % NG, ks); };
    // One tile of 64 k, two instructions deep (ks), the upper half of the wave's rows (mh = 0) before the lower.  The fragments of its
    // first 32 k, upper half, have been read; every other fragment is read a group before its use.  The buffer is free when every wave
    // has read all of it, a quarter of the tile before its end: then the tile after the next goes there.  Its loads are spread over
    // two groups, since 64 of them keep the path into LDS busy for half a tile's time and a wave that finds it full cannot issue
    // anything else; the half tile that is left is their time to arrive.  8 workers, 2048 x 1024 x 4096: all loads in one group
    // 106 us, in two 100 to 102, in three 104.
    constexpr int LEAD = LOADS / 2; // loads in the first of the groups
    // n reads and the loads from l0 to l1, evenly mixed
    auto mixed = [&](int x, int n, int l0, int l1, char *buf, const auto &read) {
        const int m = l1 - l0, t = n + m, before = x * m / t;
        if ((x + 1) * m / t > before)
            load(buf, l0 + before);
        else
            read(x - before);
    };
    auto step = [&](char *cur, char *next) {
        group(0, a0, b0, MH + NI + LOADS - LEAD, [&](int x) {
            mixed(x, MH + NI, LEAD, LOADS, next, [&](int r) {
                if (r < MH)
                    a1[r] = fa.get(cur, MH + r, 0);
                else
                    b1[r - MH] = read_b(cur, r - MH, 1);
            });
        });
        group(1, a1, b0, 2 * MH + FETCHES, [&](int r) {
            if (r < MH)
                a0[r] = fa.get(cur, r, 1);
            else if (r < MH + FETCHES)
                fetch(r - MH);
            else
                a1[r - MH - FETCHES] = fa.get(cur, r - FETCHES, 1);
        });
        group(0, a0, b1, 4, [&](int x) { prepare(x); });
        grawa_landed<FETCHES>();
        group(1, a1, b1, MH + NI + LEAD, [&](int x) {
            mixed(x, MH + NI, 0, LEAD, cur, [&](int r) {
                if (r < MH)
                    a0[r] = fa.get(next, r, 0);
                else
                    b0[r - MH] = read_b(next, r - MH, 0);
            });
        });
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int what = 0; what < 4; ++what) prepare(what);
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
            if (t == 0 || j < LEAD) load(t ? buf1 : buf0, j);
    }
#pragma unroll
    for (int what = 0; what < FETCHES; ++what) fetch(what);
    grawa_landed<LEAD + FETCHES>();
#pragma unroll
    for (int i = 0; i < MH; ++i) a0[i] = fa.get(buf0, i, 0);
#pragma unroll
    for (int j = 0; j < NI; ++j) b0[j] = read_b(buf0, j, 0);
    for (int t = 0;;) { // tiles that are not there are loaded as zeros
        step(buf0, buf1);
        if (++t >= tiles) break;
        step(buf1, buf0);
        if (++t >= tiles) break;
    }
    grawa_landed<0>(); // nothing may be on its way into LDS when the block ends
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); // the last sums are written: the compiler does not see which instructions write them

    epi.tile(tile.k, tile.split);
    constexpr int NJ = DUAL ? NI / 2 : NI, COLS = NJ * 16;
    static_assert(NW * Epi::OUTS * 16 * COLS * 4 <= ABYTES + BBYTES, "the corners fit a buffer");
    constexpr int DEEP = sizeof(typename Epi::Ahead) <= 24 ? 2 : 1; // rows of fragments that are asked for ahead of their turn
    typename Epi::Ahead r[DEEP + 1][NJ];
#pragma unroll
    for (int i = 0; i < DEEP; ++i) grawa_ahead<NJ>(epi, m0 + wm * TM + i * 16, n0 + wn * COLS, lane, g.M, g.N, r[i]);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int m1 = m0 + wm * TM + i * 16;
        if (m1 >= g.M) break;
        if (i + DEEP < MI) grawa_ahead<NJ>(epi, m1 + DEEP * 16, n0 + wn * COLS, lane, g.M, g.N, r[(i + DEEP) % (DEEP + 1)]);
        grawa_f32x4 v[NJ], u[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            v[j] = acc[i][j];
            u[j] = DUAL ? acc[i][j + NI - NJ] : grawa_f32x4{};
        }
        grawa_finish<NJ>(epi, (float *)buf0 + wave * (Epi::OUTS * 16 * COLS), m1, n0 + wn * COLS, lane, g.M, g.N, r[i % (DEEP + 1)], v, u);
    }
#endif
}

// Where a sum over k is split: the parts as fragments, [split][worker][product][fragments].
struct GrawaParts {
    float *p;
    int64_t blocks; // fragments of a product of a worker, elements
    int K, products, nb;
    __device__ __forceinline__ const float *at(int k, int split, int product) const { return p + (((int64_t)split * K + k) * products + product) * blocks; }
};

__device__ __forceinline__ int64_t grawa_fragment_at(int mb, int nb, int nblocks, int lane) { return (((int64_t)mb * nblocks + nb) * 64 + lane) * 4; }

struct EpiParts {
    static constexpr int OUTS = 0, VEC = 4;
    GrawaParts parts;
    float *v0, *u0;
    __device__ __forceinline__ void tile(int k, int split)
    {
        v0 = const_cast<float *>(parts.at(k, split, 0));
        u0 = const_cast<float *>(parts.at(k, split, parts.products - 1));
    }
    typedef GrawaNothing Ahead;
    __device__ __forceinline__ void ahead(int, int, int, Ahead &) const {}
    __device__ __forceinline__ void fragment(int mb, int nb, int lane, const Ahead &, grawa_f32x4 &v, grawa_f32x4 &u) const
    {
        const int64_t at = grawa_fragment_at(mb, nb, parts.nb, lane);
        *(grawa_f32x4 *)(v0 + at) = v;
        if (parts.products > 1) *(grawa_f32x4 *)(u0 + at) = u;
    }
    __device__ __forceinline__ void put(int, int, int, float *) const {}
};

// The parts added, in order, and the product's own epilogue.  A wave makes sixteen rows of 32 columns; where that gives few waves, SHARED,
// the four waves of a block do so together, a quarter of the parts each: 48 x 4096 in sixteen parts 10.3 us by one wave, 4.8 by four.
template <bool DUAL, bool SHARED, class Epi> __global__ __launch_bounds__(256) void k_join(GrawaParts parts, int splits, int M, int N, Epi epi)
{
    constexpr int NJ = 2;
    __shared__ __attribute__((aligned(16))) float corners[4][Epi::OUTS * 16 * NJ * 16];
    __shared__ __attribute__((aligned(16))) float sums[SHARED ? 4 : 1][2 * NJ][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = blockIdx.z;
    const int m1 = blockIdx.y * 16, n1 = (SHARED ? blockIdx.x : blockIdx.x * 4 + wave) * NJ * 16;
    if (n1 >= N) return; // the whole block where it is shared
    epi.tile(k, 0);
    typename Epi::Ahead r[NJ];
    if (!SHARED || !wave) grawa_ahead<NJ>(epi, m1, n1, lane, M, N, r);
    grawa_f32x4 v[NJ] = {}, u[NJ] = {};
    const int s0 = SHARED ? splits * wave / 4 : 0, s1 = SHARED ? splits * (wave + 1) / 4 : splits;
#pragma unroll 4
    for (int s = s0; s < s1; ++s)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            if (n1 + j * 16 < N) {
                const int64_t at = grawa_fragment_at(m1 >> 4, (n1 >> 4) + j, parts.nb, lane);
                v[j] += *(const grawa_f32x4 *)(parts.at(k, s, 0) + at);
                if (DUAL) u[j] += *(const grawa_f32x4 *)(parts.at(k, s, 1) + at);
            }
    if constexpr (SHARED) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            *(grawa_f32x4 *)&sums[wave][j][lane * 4] = v[j];
            *(grawa_f32x4 *)&sums[wave][NJ + j][lane * 4] = u[j];
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < 4; ++w)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                v[j] += *(const grawa_f32x4 *)&sums[w][j][lane * 4];
                u[j] += *(const grawa_f32x4 *)&sums[w][NJ + j][lane * 4];
            }
    }
    grawa_finish<NJ>(epi, corners[wave], m1, n1, lane, M, N, r, v, u);
}

} // namespace
