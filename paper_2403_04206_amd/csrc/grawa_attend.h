// Tiles of heads in LDS and their fragments for the matrix instructions of 32 x 32, in bfloat16 or float32 (device side of the attention).
//
// A tile is ROWS tokens (keys or queries) of one head, DP elements each, zeros where the head has fewer elements or the sequence no
// more tokens.  It goes from memory straight into LDS, 16 bytes a lane, bounded by its buffer descriptor.  The 16-byte piece c of row r
// stands at place c ^ key(r).  LDS has 64 banks, a load of 16 bytes a lane takes sixteen lanes at a time and the transposing load of 8
// bytes thirty-two: the sixteen rows of the one, the four rows and four pieces of the other (float32 by columns: two rows four apart and
// eight pieces) fall on different banks.  Keys that only told eight rows apart cost four cycles more a load.
//
// A fragment is 32 x 16: the lane has line lane % 32 and eight k of it.  By rows those are k = 8 (lane / 32) + j.  By columns the lines
// are elements of the head and k runs over tokens in the order in which a product's sums stand in registers: for sums of 32 x 32 the
// lane has column lane % 32 and rows j % 4 + 8 (j / 4) + 4 (lane / 32) in register j, so registers 8 t ... 8 t + 7 are, without any
// exchange, the second operand of a product over tokens 16 t + 4 (lane / 32) + j % 4 + 8 (j / 4).
// float32 goes through the same fragments by eight instructions of 32 x 32 x 2, each of which takes register j of both halves.
#pragma once
#include "grawa_attention.h"
#include "grawa_elements.h"

typedef float grawa_f32x16 __attribute__((ext_vector_type(16)));
typedef float grawa_f32x8 __attribute__((ext_vector_type(8)));
typedef float grawa_f32x4v __attribute__((ext_vector_type(4)));
typedef short grawa_s16x4v __attribute__((ext_vector_type(4)));
typedef short grawa_s16x8v __attribute__((ext_vector_type(8)));

#define GRAWA_LDS_AT __attribute__((address_space(3)))

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// Where scores in units of log2 are so large that the roundings of what their exponentials are taken against would show: of the maximum,
// which is a factor of all exponentials, or of the logarithm of their sum.
constexpr float LARGE = 0x1p20f;

template <bool BF16> struct Frag;
template <> struct Frag<true> {
    typedef grawa_bf16x8 V;
};
template <> struct Frag<false> {
    typedef grawa_f32x8 V;
};

// Which pieces of a tile the lanes load and where: NW waves, 64 lanes of 16 bytes each a load.
template <bool BF16, int DP, int ROWS, int NW> struct TilePieces {
    static constexpr int ES = BF16 ? 2 : 4, RB = DP * ES, PPR = RB / 16, BYTES = ROWS * RB, LOADS = BYTES / 1024 / NW;
    static constexpr int RPL = NW * 64 / PPR, TURNS = RPL < 16 ? 16 / RPL : 1; // rows that the waves load at a time; loads until the keys repeat
    static_assert(LOADS * NW * 1024 == BYTES && LOADS % TURNS == 0, "whole loads of whole groups of rows");

    static __host__ __device__ __forceinline__ int key(int row)
    {
        if constexpr (!BF16) return (((row >> 2) & 1) << 3) | ((row & 3) << 1) | ((row >> 3) & 1);
        if constexpr (DP == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
        return (((row >> 1) & 1) << 2) | ((row >> 2) & 1) | (((row >> 3) & 1) << 1); // rows of 128 bytes: their lowest bit is a bank's
    }
    // Offsets of rows of below 2^24 bytes each.  Pieces that the head does not have are beyond every descriptor of the tile in all its loads: up to
    // 128 rows end below 2^31, where such pieces begin, and with them end below 2^32; more rows leave no room to go on in, and such pieces stay.
    static constexpr uint32_t NONE = ROWS <= 128 ? 0x80000000u : 0xffffff00u;
    static __host__ __device__ __forceinline__ uint32_t first_of(int id, int turn, uint32_t token, int D)
    {
        const int row = id / PPR + turn * RPL, c = (id % PPR) ^ key(row);
        return c * 16 < D * ES ? (uint32_t)row * token + (uint32_t)c * 16 : NONE;
    }
    static __host__ __device__ __forceinline__ uint32_t later(uint32_t first, uint32_t by) { return ROWS > 128 && first == NONE ? NONE : first + by; }
};

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ grawa_f32x16 mfma(const grawa_bf16x8 &a, const grawa_bf16x8 &b, const grawa_f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ grawa_f32x16 mfma(const grawa_f32x8 &a, const grawa_f32x8 &b, grawa_f32x16 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// Registers 8 t ... 8 t + 7 of sums as an operand.
__device__ __forceinline__ void as_operand(const grawa_f32x16 &s, int t, grawa_bf16x8 &f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (__bf16)s[8 * t + j];
}
__device__ __forceinline__ void as_operand(const grawa_f32x16 &s, int t, grawa_f32x8 &f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = s[8 * t + j];
}

// What the other half of the wave has.
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

template <bool BF16, int DP, int ROWS, int NW> struct HeadTile : TilePieces<BF16, DP, ROWS, NW> {
    typedef typename Frag<BF16>::V V;
    typedef TilePieces<BF16, DP, ROWS, NW> Pieces;
    using Pieces::ES, Pieces::RB, Pieces::BYTES, Pieces::LOADS, Pieces::RPL, Pieces::TURNS, Pieces::key;

    // Loads: the lane's offset in the wave's first ones, until the keys repeat.
    uint32_t first[TURNS], step;
    __device__ __forceinline__ void init(int wave, int lane, uint32_t token, int D)
    {
#pragma unroll
        for (int i = 0; i < TURNS; ++i) first[i] = Pieces::first_of(wave * 64 + lane, i, token, D);
        step = RPL * TURNS * token;
    }
    // rows: what the sequence has from the tile's first token on; none: nothing is read and all comes as zeros.
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const char *p, int rows, uint32_t token, int D)
    {
        const int n = rows < ROWS ? rows : ROWS;
        return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, n > 0 ? (uint32_t)(n - 1) * token + (uint32_t)(D * ES) : 0, 0x00020000);
    }
    __device__ __forceinline__ void load(char *lds, int wave, __amdgpu_buffer_rsrc_t r) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (GRAWA_LDS_AT void *)(lds + (wave + NW * i) * 1024), 16, Pieces::later(first[i % TURNS], (uint32_t)(i / TURNS) * step), 0, 0, 0);
    }

    // Fragments: an offset of the lane's that all of a tile's share, of which a fragment's differs by some of its low bits and by a constant.
    // Tiles are arrays by themselves and a fragment is read from its array: the compiler then knows that loads on their way into another
    // one need not land first.
    static __device__ __forceinline__ uint32_t rows_of(int lane)
    {
        const int row = lane & 31, half = lane >> 5;
        return row * RB + (((BF16 ? half : 2 * half) ^ key(row)) << 4);
    }
    static __device__ __forceinline__ uint32_t columns_of(int lane)
    {
        const int half = lane >> 5, s = lane & 15, row = 4 * half + (s >> 2), m = lane & 31;
        if constexpr (BF16) return row * RB + (((2 * ((lane >> 4) & 1) + ((s & 3) >> 1)) ^ key(row)) << 4) + (s & 1) * 8;
        return 4 * half * RB + (((m >> 2) ^ key(4 * half)) << 4) + (m & 3) * 4;
    }

    // Lines row0 ... row0 + 31 (a multiple of 32), elements 16 ks ... of the head.
    static __device__ __forceinline__ V by_rows(const char *tile, uint32_t at, int row0, int ks)
    {
        if constexpr (BF16) {
            return *(const V *)(tile + row0 * RB + (at ^ (ks << 5)));
        } else {
            const grawa_f32x4v a = *(const grawa_f32x4v *)(tile + row0 * RB + (at ^ (ks << 6))), b = *(const grawa_f32x4v *)(tile + row0 * RB + (at ^ (ks << 6) ^ 16));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // Lines: elements 32 dt ... of the head, k: tokens row0 ... row0 + 15 (a multiple of 16) in the order of a product's registers.
    static __device__ __forceinline__ V by_columns(const char *tile, uint32_t at, int row0, int dt)
    {
        if constexpr (BF16) {
            const uint32_t lower = at ^ (dt << 6), upper = lower ^ 32; // eight rows on, the key's second bit is another
            const grawa_s16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GRAWA_LDS_AT grawa_s16x4v *)(tile + row0 * RB + lower));
            const grawa_s16x4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GRAWA_LDS_AT grawa_s16x4v *)(tile + (row0 + 8) * RB + upper));
            return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            V v;
#pragma unroll
            for (int j = 0; j < 8; ++j) { // rows 4 (lane / 32) + j % 4 + 8 (j / 4): what their keys differ in
                const int row = (j & 3) + 8 * (j >> 2);
                v[j] = *(const float *)(tile + (row0 + row) * RB + (at ^ (dt << 7) ^ (key(row) << 4)));
            }
            return v;
        }
    }
};

// Where the tiles of keys and values of a head are read from, one after the other: first those with first tokens, then those of the window.
template <class Tile, int BK> struct Tiles {
    const char *k, *v;           // the next one's
    int64_t k_step, v_step;
    uint32_t k_token, v_token, bytes;
    int left;                    // tokens from the next one on
    int jump, gap;               // where the window's tiles do not follow the first tokens': behind `jump` tiles, by `gap`

    __device__ __forceinline__ void init(const char *k0, const char *v0, uint32_t kt, uint32_t vt, int length, int D, int from, int first_tiles, int t0)
    {
        const int j0 = (from < first_tiles ? from : from - first_tiles + t0) * BK;
        k_token = kt, v_token = vt, bytes = D * Tile::ES;
        k_step = (int64_t)kt * BK, v_step = (int64_t)vt * BK;
        k = k0 + (int64_t)j0 * kt, v = v0 + (int64_t)j0 * vt;
        left = length - j0;
        jump = from < first_tiles ? first_tiles - from : -1;
        gap = t0 - first_tiles;
    }
    __device__ __forceinline__ void load(const Tile &lk, const Tile &lv, char *buf, int wave)
    {
        const uint32_t n = left < BK ? left : BK; // more than 0: tiles beyond the length are not asked for
        lk.load(buf, wave, __builtin_amdgcn_make_buffer_rsrc((void *)k, 0, (n - 1) * k_token + bytes, 0x00020000));
        lv.load(buf + Tile::BYTES, wave, __builtin_amdgcn_make_buffer_rsrc((void *)v, 0, (n - 1) * v_token + bytes, 0x00020000));
        k += k_step, v += v_step, left -= BK;
        if (--jump == 0) k += gap * k_step, v += gap * v_step, left -= gap * BK;
    }
};

// Keeps what an offset differs in from being formed ahead for all fragments and held in registers.
__device__ __forceinline__ uint32_t here(uint32_t at)
{
    asm volatile("" : "+v"(at));
    return at;
}

// All loads into LDS have landed and all reads from it are done, the wave's own and then the other waves'.
__device__ __forceinline__ void landed()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A run of N matrix instructions whose fragments from LDS are asked for AHEAD before they are used; f holds the first ones (asked for
// by `ask`, early).  Nothing is moved across: left to itself the compiler reads a fragment, waits, uses it and reads the next one as
// soon as registers are few.
template <int AHEAD, class V, class L> __device__ __forceinline__ void ask(V (&f)[AHEAD], L &&load)
{
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = load(i);
    __builtin_amdgcn_sched_barrier(0);
}
template <int N, int AHEAD, class V, class L, class U> __device__ __forceinline__ void flow(V (&f)[AHEAD], L &&load, U &&use)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        use(i, f[i % AHEAD]);
        if (i + AHEAD < N) f[i % AHEAD] = load(i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// What the wave's lanes have written to LDS, its other lanes read from here on.
__device__ __forceinline__ void wave_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// sums += a w for a tile of which only some pairs count: a pair that does not count has w = 0, but an infinity or no number in its line
// of a must not reach the sum.  `counts` has 1 for pairs that count; what they bring that is not finite makes the sum no number.  One
// at a time: this is not where speed counts, and registers are few.
template <class V> __device__ __forceinline__ void product_of_some(grawa_f32x16 &sums, V a, const V &w, const V &counts)
{
    V odd;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float f = (float)a[j];
        const bool finite = fabsf(f) < __builtin_inff();
        odd[j] = finite ? 0.f : 1.f;
        a[j] = finite ? f : 0.f;
    }
    __builtin_amdgcn_sched_barrier(0);
    sums = mfma(a, w, sums);
    __builtin_amdgcn_sched_barrier(0);
    grawa_f32x16 n = {};
    n = mfma(odd, counts, n);
#pragma unroll
    for (int j = 0; j < 16; ++j) sums[j] = n[j] > 0.f ? __builtin_nanf("") : sums[j];
    __builtin_amdgcn_sched_barrier(0);
}

template <bool B> struct Is {
    static constexpr bool value = B;
};

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Which tokens a sequence has and where its new ones begin; whatever the caller's numbers are, positions stay far from 32 bits.
struct Place {
    int start, length;
};
__device__ __forceinline__ Place place_of(const GrawaAttend &a, int kn)
{
    Place p;
    p.start = a.starts ? clamp_int(a.starts[kn], -(1 << 29), 1 << 29) : a.Sk - a.Sq;
    p.length = a.lengths ? clamp_int(a.lengths[kn], 0, a.Sk) : a.Sk;
    return p;
}

// One column of queries: its 32 x 16 fragments straight from memory, zeros where there is nothing.
template <bool BF16> __device__ __forceinline__ typename Frag<BF16>::V load_line(const char *row, int e, int D, bool there)
{
    typedef typename Frag<BF16>::V V;
    V v = {};
    if (there && e < D) {
        if constexpr (BF16) {
            v = *(const V *)(row + e * 2);
        } else {
            const grawa_f32x4v a = *(const grawa_f32x4v *)(row + e * 4), b = *(const grawa_f32x4v *)(row + e * 4 + 16);
            v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    return v;
}

// Sixteen sums of a column, elements 32 dt + 8 q + 4 (lane / 32) ... of the head, to memory.
template <bool BF16> __device__ __forceinline__ void store_column(char *row, int lane, int dt, int D, const grawa_f32x16 &s, float f)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = 32 * dt + 8 * q + 4 * (lane >> 5);
        if (e >= D) continue;
        if constexpr (BF16) {
            typedef __bf16 B4 __attribute__((ext_vector_type(4)));
            B4 b;
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = (__bf16)(s[4 * q + j] * f);
            *(B4 *)(row + e * 2) = b;
        } else {
            grawa_f32x4v b;
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = s[4 * q + j] * f;
            *(grawa_f32x4v *)(row + e * 4) = b;
        }
    }
}

__device__ __forceinline__ bool sees(const GrawaAttend &a, int pos, int j)
{
    const int d = pos - j;
    return d >= 0 && (d < a.window || j < a.sinks);
}

// A bias in units of log2.  The type's lowest number hides a key as minus infinity does: a row that sees nothing else would have a sum of
// exponentials whose logarithm float32 cannot tell from its neighbours'.
template <bool BF16> __device__ __forceinline__ float bias_of(const char *p)
{
    const float b = load_one<BF16>(p);
    return b < -0x1p100f ? -__builtin_inff() : b * LOG2E;
}

// Marks of the tokens j0 + ... that a column sees, in the order of an operand.
template <class V> __device__ __forceinline__ V marks(const GrawaAttend &a, int pos, int j0, int half)
{
    V v;
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? 1.f : 0.f;
    return v;
}

#endif // __HIP_DEVICE_COMPILE__

// Which head and which of its blocks a workgroup has.  Workgroups go round the eight XCDs.  The `share` heads that read the same keys stay
// on one, so that their blocks share its L2, and such groups are dealt out one by one, so that long sequences are spread.  An XCD takes the
// first block of all its heads, then the second: blocks are numbered from the longest on, and the short ones fill the end.  Few groups that
// eight does not divide are dealt out head by head.
struct Turn {
    int head, block;
};
__host__ __device__ inline Turn turn_of(uint32_t id, uint32_t groups, uint32_t share, int by_xcd)
{
    const uint32_t heads = groups * share;
    if (!by_xcd) return Turn{(int)(id % heads), (int)(id / heads)};
    const uint32_t each = (groups + 7) / 8 * share, r = id / 8, h = r % each;
    // Eight groups after the other start one XCD further on, so that the groups of one sequence, four of eight, do not always fall to the
    // same: 4 workers' 3 sequences of up to 600 tokens, float32, 77 us, and 84 without.
    const uint32_t group = h / share * 8 + (id + h / share) % 8;
    return Turn{(int)(group * share + h % share), (int)(r / each)};
}

// The grid for turn_of; heads that are not there have workgroups that end at once.
inline uint32_t grid_of(int64_t groups, int64_t share, int64_t blocks, int &by_xcd)
{
    by_xcd = groups % 8 == 0 || groups >= 64;
    return (uint32_t)((by_xcd ? (groups + 7) / 8 * 8 : groups) * share * blocks);
}

} // namespace
