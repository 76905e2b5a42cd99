// The gated feed-forward block of K workers, forward and backward:
//   G = x Wg^T;  U = x Wu^T;  H = act(G) U;  y = H Wd^T [dropped, plus a residual]
//   dH = dy Wd;  dU = dH act(G);  dG = dH U act'(G);  dx = dG Wg + dU Wu;  dWg = dG^T x;  dWu = dU^T x;  dWd = dy^T H
// Three kinds of product in the forward pass and six in the backward, 18 K T d f operations together: bound by the matrix cores but
// for a few tokens.  Gate and up come from one kernel, whose epilogue has both in registers and leaves H; the backward's first
// kernel makes dH and from it dG and dU in its epilogue, so that no pass over [T][f] arrays stands between the products.
//
// Roundings.  bfloat16: H, dG and dU are rounded to bfloat16, as the matrix instructions take them; G and U are kept for the
// backward pass with eight bits more than that (a rounding of theirs would be a third one on the way to dWg, dWu and dx).  float32: every matrix
// element is split exactly into three bfloat16 terms and the six largest of the nine products of terms are summed in float32;
// what is left out is at most 2^-24 of a product.  (An infinity times a number that is exactly a bfloat16 gives NaN there.)
#include "grawa_few.h"
#include "grawa_gemm.h"

namespace {

// The three terms, each what the terms before it left, rounded to nearest; the last takes all that is left.  Rounded, and not cut off: the second
// and the third term are then at most 2^-8 and 2^-17 of the number's leading bit, and of either sign.  Cut off, they reach 2^-7 and 2^-15 and have
// the number's own sign, so that what a sum of products leaves out is up to 2^-21 of it and always on one side.  A number that
// would round to infinity is cut off.
__device__ __forceinline__ void split3(float v, uint16_t t[3])
{
    const uint32_t u = __float_as_uint(v);
    t[0] = __builtin_bit_cast(uint16_t, (__bf16)v);
    if ((t[0] & 0x7fff) == 0x7f80) t[0] = (uint16_t)(u >> 16);
    const float r = (u & 0x7f800000u) == 0x7f800000u ? 0.f : v - bf16_one(t[0]);
    t[1] = __builtin_bit_cast(uint16_t, (__bf16)r);
    t[2] = __builtin_bit_cast(uint16_t, (__bf16)(r - bf16_one(t[1])));
}

// Eight numbers to the planes at p, p + plane, p + 2 plane (bytes): 16 bytes each.
template <int PLANES> __device__ __forceinline__ void store_planes8(char *p, int64_t plane, const float *v)
{
    if constexpr (PLANES == 1) {
        store_piece<true>(p, 8, v);
    } else {
        uint16_t t[8][3];
#pragma unroll
        for (int j = 0; j < 8; ++j) split3(v[j], t[j]);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = t[2 * j][q] | ((uint32_t)t[2 * j + 1][q] << 16);
            *(uint4 *)(p + q * plane) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// Copies of matrices and activations whose rows are not on 16-byte boundaries, and of all in float32: [K][R][C] elements into planes of
// pitch Cp with zeros behind C to the next multiple of 8.  Up to five in a launch; eight elements a thread, read at any alignment.  Bound by
// memory: two workers' 1000 x 2731 in bfloat16, 66 MB, 12.3 us; four workers' 1024 x 4096 in float32, 540 MB, 80 us.
struct CopyJob {
    const char *src;
    char *dst;
    int64_t worker, row, plane; // src in elements; dst in bytes
    uint32_t R, C, Cp;
};

struct CopyJobs {
    CopyJob job[5];
    int n;
};

template <bool BF16> __global__ __launch_bounds__(256) void k_planes(CopyJobs jobs)
{
    constexpr int S = BF16 ? 2 : 4;
    const CopyJob &j = jobs.job[blockIdx.z];
    const uint32_t groups = (j.C + 7) / 8, k = blockIdx.y;
    const uint64_t total = (uint64_t)j.R * groups;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
        const uint32_t r = total >> 32 ? (uint32_t)(i / groups) : (uint32_t)i / groups, c = (uint32_t)(i - (uint64_t)r * groups) * 8;
        const char *p = j.src + ((int64_t)k * j.worker + (int64_t)r * j.row + c) * S;
        float v[8] = {};
        if (c + 8 <= j.C) {
            const GrawaAny16 a = *(const GrawaAny16 *)p, b = BF16 ? a : *(const GrawaAny16 *)(p + 16);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (BF16) {
                    v[2 * q] = bf16_lo(a[q]);
                    v[2 * q + 1] = bf16_hi(a[q]);
                } else {
                    v[q] = __uint_as_float(a[q]);
                    v[4 + q] = __uint_as_float(b[q]);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < j.C) v[q] = load_one<BF16>(p + q * S);
        }
        store_planes8<BF16 ? 1 : 3>(j.dst + (((int64_t)k * j.R + r) * j.Cp + c) * 2, j.plane, v);
    }
}

// The activation and its derivative.  Float32 calls the mathematical functions, but for the error function.  For results that are rounded to bfloat16 the hardware's
// 2^z and 1/z (an ulp each) do, and for the error function a formula of the form of 7.1.26 in Abramowitz and Stegun, "Handbook of
// Mathematical Functions" (1964), erfc(x) = e^(-x^2) t P(t) with t = 1 / (1 + 0.411 x), whose P is fitted to erfc for this: evaluated in
// float32, the smaller tail is off by at most 2e-7 and by at most 9e-5 of itself as far as float32 has it (z = -13); theirs, with a
// term less, by 1.6e-3 of itself at -5 and 1e-2 at -8, more than bfloat16 rounds.  With division, expf and erff the kernel of dH
// took 266 us for 8 x 2048 tokens, 1024 x 4096, by such formulas 252.
template <int PLANES> __device__ __forceinline__ float sigmoid_of(float z)
{
    if constexpr (PLANES == 3) return 1.f / (1.f + expf(-z));
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
}

// The normal distribution's cumulative function at z and its density.  For float32 the formula with nine terms and the reciprocal corrected
// once: the smaller tail is off by 3.1e-7 of itself at most, besides what a rounding of z^2 makes of e^(-z^2/2).  (1 + erff has an error of
// 6e-8 in all and so nothing of the tail below -5.4; erfcf takes so many registers that the kernel of dH keeps sums in memory.)
template <int PLANES> __device__ __forceinline__ void normal_of(float z, float &cdf, float &density)
{
    float half, e;
    if constexpr (PLANES == 3) {
        const float x = fabsf(z) * 0.70710678118654752f, q = fmaf(x, 0.5f, 1.f);
        float t = __builtin_amdgcn_rcpf(q);
        t = q < INFINITY ? fmaf(t, fmaf(-q, t, 1.f), t) : 0.f;
        float p = -0.0589314164f;
        constexpr float terms[8] = {0.28390128f, -0.485798848f, 0.276456327f, -0.0255096898f, 0.202211608f, 0.243224785f, 0.282358527f, 0.282087384f};
#pragma unroll
        for (int i = 0; i < 8; ++i) p = fmaf(p, t, terms[i]);
        e = expf(-0.5f * z * z);
        half = 0.5f * e * (t * p);
    } else {
        const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.f + 0.411f * x);
        e = __builtin_amdgcn_exp2f(x * x * -1.4426950408889634f);
        half = e * (t * (0.117116504f + t * (0.101114006f + t * (0.178743041f + t * (-0.0907627439f + t * (0.282544145f + t * -0.0887550025f)))))); // P / 2
    }
    cdf = z < 0.f ? half : 1.f - half;
    density = e * 0.39894228040143268f;
}

// a = act(z) and back = v act'(z).  What relu closes is 0 whatever stands beside it: a gate of -infinity, an infinite v; a NaN stays one.
template <int PLANES, int ACT> __device__ __forceinline__ void act_both(float z, float v, float &a, float &back)
{
    float da;
    if constexpr (ACT == GRAWA_ACT_SILU) {
        const float s = sigmoid_of<PLANES>(z);
        a = z * s;
        da = s + a * (1.f - s);
    } else if constexpr (ACT == GRAWA_ACT_GELU) {
        float cdf, density;
        normal_of<PLANES>(z, cdf, density);
        a = z * cdf;
        da = cdf + z * density;
    } else {
        a = z <= 0.f ? 0.f : z;
        back = z > 0.f ? v : 0.f;
        return;
    }
    back = v * da;
}

template <int PLANES, int ACT> __device__ __forceinline__ float act_of(float z)
{
    float a, back;
    act_both<PLANES, ACT>(z, 0.f, a, back);
    return a;
}

// Gate and up before the activation are kept for the backward pass as the fragments of the matrix instruction, blocks of 16 x 16 by 64
// lanes, so that both kernels move them by whole KiB straight from and to the registers.  Float32 keeps them whole: a plane of G, a
// plane of U.  Bfloat16 keeps 24 bits, rounded to nearest (a sign, 8 and 15: 2^-16 of a value, dG and dU are rounded by 2^-8):
// a plane of 16 bytes a lane with the upper halves of four G and four U, then one of 8 bytes with the next byte of each.  The forward
// and the backward kernel of 8 x 2048 tokens, 1024 x 4096, move 270 MB less for it.  Both go past the caches, where they would take the
// place of the tiles: training 1223 us by cached loads and stores, so 1193.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int PLANES> struct KeptGateUp {
    char *p;          // null: not kept
    int64_t all;      // fragments of all workers, elements of one plane
    __device__ __forceinline__ void put(int64_t at, const grawa_f32x4 &g, const grawa_f32x4 &u) const
    {
        if constexpr (PLANES == 3) {
            __builtin_nontemporal_store(g, (grawa_f32x4 *)(p + at * 4));
            __builtin_nontemporal_store(u, (grawa_f32x4 *)(p + (all + at) * 4));
        } else {
            uint32_t a[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(g[j]) + 0x80, a[4 + j] = __float_as_uint(u[j]) + 0x80; // half of what the last byte counts; a NaN, whose low bits are 0, stays one
            uint32_t hi[4], lo[2];
#pragma unroll
            for (int j = 0; j < 4; ++j) hi[j] = __builtin_amdgcn_perm(a[2 * j + 1], a[2 * j], 0x07060302);
#pragma unroll
            for (int j = 0; j < 2; ++j) lo[j] = __builtin_amdgcn_perm(a[4 * j + 1], a[4 * j], 0x0c0c0501) | __builtin_amdgcn_perm(a[4 * j + 3], a[4 * j + 2], 0x05010c0c);
            __builtin_nontemporal_store(u32x4{hi[0], hi[1], hi[2], hi[3]}, (u32x4 *)(p + at * 4));
            __builtin_nontemporal_store(u32x2{lo[0], lo[1]}, (u32x2 *)(p + all * 4 + at * 2));
        }
    }
    struct Raw {
        uint32_t w[PLANES == 3 ? 8 : 6];
    };
    __device__ __forceinline__ void get(int64_t at, Raw &r) const
    {
        const u32x4 a = __builtin_nontemporal_load((const u32x4 *)(p + at * 4));
        r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
        if constexpr (PLANES == 3) {
            const u32x4 b = __builtin_nontemporal_load((const u32x4 *)(p + (all + at) * 4));
            r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
        } else {
            const u32x2 b = __builtin_nontemporal_load((const u32x2 *)(p + all * 4 + at * 2));
            r.w[4] = b.x, r.w[5] = b.y;
        }
    }
    static __device__ __forceinline__ void values(const Raw &r, grawa_f32x4 &g, grawa_f32x4 &u)
    {
        constexpr uint32_t which[4] = {0x0504000c, 0x0706010c, 0x0504020c, 0x0706030c};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] = __uint_as_float(PLANES == 3 ? r.w[j] : __builtin_amdgcn_perm(r.w[j / 2], r.w[4], which[j]));
            u[j] = __uint_as_float(PLANES == 3 ? r.w[4 + j] : __builtin_amdgcn_perm(r.w[2 + j / 2], r.w[5], which[j]));
        }
    }
};

// Epilogue of gate and up: H, and for a backward pass G and U.
template <int PLANES, int ACT> struct EpiGateUp {
    static constexpr int OUTS = 1, VEC = 8;
    char *h;            // [PLANES][K][M][pitch]
    KeptGateUp<PLANES> kept;
    int64_t plane;      // bytes between the planes of h
    int64_t worker;     // elements of a worker's h
    int64_t blocks;     // fragments of a worker, elements
    int N, pitch;
    int64_t at0;
    __device__ __forceinline__ void tile(int k, int)
    {
        h += k * worker * 2;
        at0 = k * blocks;
    }
    typedef GrawaNothing Ahead;
    __device__ __forceinline__ void ahead(int, int, int, Ahead &) const {}
    __device__ __forceinline__ void fragment(int mb, int nb, int lane, const Ahead &, grawa_f32x4 &g, grawa_f32x4 &u) const
    {
        if (kept.p) kept.put(at0 + grawa_fragment_at(mb, nb, (N + 15) >> 4, lane), g, u);
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] = act_of<PLANES, ACT>(g[j]) * u[j];
    }
    __device__ __forceinline__ void put(int, int m, int n, float *v) const
    {
        if (n + 8 > N)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (n + j >= N) v[j] = 0.f;
        store_planes8<PLANES>(h + ((int64_t)m * pitch + n) * 2, plane, v);
    }
};

// Epilogue of dH: dG and dU.
template <int PLANES, int ACT> struct EpiBack {
    static constexpr int OUTS = 2, VEC = 8;
    KeptGateUp<PLANES> kept;
    char *dg, *du;
    int64_t plane, worker, blocks;
    int N, pitch;
    int64_t at0;
    __device__ __forceinline__ void tile(int k, int)
    {
        at0 = k * blocks;
        dg += k * worker * 2;
        du += k * worker * 2;
    }
    typedef typename KeptGateUp<PLANES>::Raw Ahead;
    __device__ __forceinline__ void ahead(int mb, int nb, int lane, Ahead &r) const { kept.get(at0 + grawa_fragment_at(mb, nb, (N + 15) >> 4, lane), r); }
    __device__ __forceinline__ void fragment(int, int, int, const Ahead &r, grawa_f32x4 &dh, grawa_f32x4 &out) const
    {
        grawa_f32x4 g, u;
        kept.values(r, g, u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a, back;
            act_both<PLANES, ACT>(g[j], dh[j] * u[j], a, back);
            out[j] = dh[j] * a;
            dh[j] = back;
        }
    }
    __device__ __forceinline__ void put(int o, int m, int n, float *v) const
    {
        if (n + 8 > N)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (n + j >= N) v[j] = 0.f;
        store_planes8<PLANES>((o ? du : dg) + ((int64_t)m * pitch + n) * 2, plane, v);
    }
};

// Epilogue of everything else: to an array of the caller's, rounded once, added to what is there (accumulate) or dropped and added to a
// residual (OUT).
template <bool BF16, bool OUT> struct EpiStore {
    static constexpr int OUTS = 1, VEC = BF16 ? 8 : 4;
    GrawaRows y, res;   // OUT: res.p may be null
    GrawaDrop drop;     // OUT
    int N, T, accumulate;
    uint32_t row0;      // of the worker, for the dropout
    GrawaMat second;    // !OUT: what the workers from `one` on, a second product's, write to
    int one;
    __device__ __forceinline__ void tile(int k, int)
    {
        constexpr int S = BF16 ? 2 : 4;
        if (!OUT && k >= one) {
            k -= one;
            y.p = second.p;
            y.worker = second.worker;
        }
        y.p += (int64_t)k * y.worker * S;
        if (OUT && res.p) res.p += (int64_t)k * res.worker * S;
        row0 = (uint32_t)k * (uint32_t)T;
    }
    typedef GrawaNothing Ahead;
    __device__ __forceinline__ void ahead(int, int, int, Ahead &) const {}
    __device__ __forceinline__ void fragment(int, int, int, const Ahead &, grawa_f32x4 &, grawa_f32x4 &) const {}
    __device__ __forceinline__ void put(int, int m, int n, float *v) const
    {
        constexpr int S = BF16 ? 2 : 4;
        if (OUT && drop.threshold) {
            const GrawaDropKey key = grawa_drop_key(drop);
#pragma unroll
            for (int q = 0; q < VEC / 4; ++q) grawa_drop4(drop, key, row0 + (uint32_t)m, (uint32_t)n / 4 + q, v + 4 * q);
        }
        char *p = y.p + ((int64_t)m * y.row + n) * S;
        const char *from = OUT ? (res.p ? res.p + ((int64_t)m * res.row + n) * S : nullptr) : accumulate ? p : nullptr;
        if (from) {
            GrawaPiece<BF16> r;
            r.load(from, N - n);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] += r[j];
        }
        store_piece<BF16, true>(p, N - n, v);
    }
};

// A matrix operand as the products read it.
struct Operand {
    const char *p;
    int64_t worker, plane; // bytes
    int64_t ld;
};

constexpr int64_t MAX_LD = ((int64_t)1 << 31) / 256 - 128; // bytes; a tile's offsets have 31 bits

// How a product is cut: its tiles, and the parts that its sum over k is split into.
struct Cut {
    int kind; // 0: 256 x 256, 1: 128 x 128, 2: 64 x 128
    int splits;
    int64_t tiles;
};

constexpr int64_t PART_FLOATS = (int64_t)512 * 256 * 256; // most that the parts of a product take
constexpr int MAX_SPLITS = 16;

// The cut with the least time by what was measured (us): a tile of 64 k takes 1.6 in a block of 256 x 256, of which a CU holds one; in
// one of 128 x 128 it takes 1.3 where a CU holds two and 0.8 where it has one; in one of 64 x 128, for products of no more rows than
// that, 1.2 where a CU holds three, 0.9 with two, 0.7 with one; a block costs about three such tiles more; parts are written and read at 4 TB/s by a
// launch more.
Cut cut_of(int64_t K, int64_t M, int64_t N, int64_t ktiles, bool dual, bool short_rows, int64_t part_floats)
{
    static const struct { int bm, bn, slots; double us[3]; } kinds[3] = {{256, 256, 256, {1.6, 1.6, 1.6}}, {128, 128, 512, {0.8, 1.3, 1.3}}, {64, 128, 768, {0.7, 0.9, 1.2}}};
    Cut best{};
    double least = 0;
    const int64_t padded = K * grawa_round16(M) * grawa_round16(N) * (dual ? 2 : 1);
    for (int kind = short_rows && M <= 64 ? 2 : 0; kind < (short_rows && M <= 64 ? 3 : 2); ++kind) {
        const auto &c = kinds[kind];
        const int64_t bn = dual ? c.bn / 2 : c.bn, tiles = K * ((M + c.bm - 1) / c.bm) * ((N + bn - 1) / bn);
        for (int s = 1; s <= MAX_SPLITS; ++s) {
            if (s > 1 && (s * padded > part_floats || ktiles / s < 4 || s * tiles > 2 * c.slots)) break;
            const int64_t full = s * tiles / c.slots, rest = s * tiles - full * c.slots;
            const double tile_us = (double)full * c.us[2] + (rest ? c.us[(rest - 1) / 256] : 0);
            double us = tile_us * ((double)((ktiles + s - 1) / s) + 3);
            if (s > 1) us += 5 + 8e-6 * (double)(s * padded) / 4;
            if (!best.splits || us < least) {
                best = Cut{kind, s, tiles};
                least = us;
            }
        }
    }
    return best;
}

// A product of one row of tiles reads its matrix once.  If the block's three matrices are more than the last-level cache holds, nothing of
// them is there at the next call, and they are read past it: 48 tokens, 4096 x 11264 (277 MB), 79.6 us by cached loads, 69.3 so, but
// four workers' 1024 x 4096 (101 MB) 28.6 us again and again by cached loads and 35.8 past them.
constexpr int64_t CACHED = (int64_t)256 << 20;

// SHORT: products of no more rows than the lowest tile has come here at all.
template <bool AT, bool BT, bool DUAL, bool SHORT, class Epi> void launch_tiles(const grawa_sublayer *s, const GrawaGemm &g, const Cut &cut, const Epi &epi, hipStream_t st)
{
    const dim3 grid((unsigned)(cut.tiles * cut.splits));
    if (cut.kind == 0)
        k_gemm<256, 256, 2, 4, false, AT, BT, DUAL, Epi><<<grid, 512, 0, st>>>(g, epi);
    else if (cut.kind == 1)
        k_gemm<128, 128, 2, 2, false, AT, BT, DUAL, Epi><<<grid, 256, 0, st>>>(g, epi);
    else if constexpr (SHORT) {
        if (6 * s->planes * (int64_t)s->K * s->d * s->f > CACHED)
            k_gemm<64, 128, 1, 4, true, AT, BT, DUAL, Epi><<<grid, 256, 0, st>>>(g, epi);
        else
            k_gemm<64, 128, 1, 4, false, AT, BT, DUAL, Epi><<<grid, 256, 0, st>>>(g, epi);
    }
}

template <bool AT, bool BT, bool DUAL, bool SHORT, class Epi> hipError_t launch_gemm(const grawa_sublayer *s, GrawaGemm g, const Epi &epi, hipStream_t st)
{
    const Cut cut = cut_of(g.K, g.M, g.N, (int64_t)((g.len + GRAWA_BK - 1) / GRAWA_BK) * g.nseg, DUAL, SHORT, s->part_floats);
    g.splits = cut.splits;
    if (cut.splits == 1) {
        launch_tiles<AT, BT, DUAL, SHORT>(s, g, cut, epi, st);
    } else {
        const int64_t blocks = grawa_round16(g.M) * grawa_round16(g.N);
        const GrawaParts parts{s->part, blocks, g.K, DUAL ? 2 : 1, (g.N + 15) >> 4};
        launch_tiles<AT, BT, DUAL, SHORT>(s, g, cut, EpiParts{parts, nullptr, nullptr}, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const unsigned rows = (unsigned)((g.M + 15) / 16);
        if (cut.splits >= 4 && (int64_t)((g.N + 127) / 128) * rows * g.K < 512)
            k_join<DUAL, true, Epi><<<dim3((unsigned)((g.N + 31) / 32), rows, (unsigned)g.K), 256, 0, st>>>(parts, cut.splits, g.M, g.N, epi);
        else
            k_join<DUAL, false, Epi><<<dim3((unsigned)((g.N + 127) / 128), rows, (unsigned)g.K), 256, 0, st>>>(parts, cut.splits, g.M, g.N, epi);
    }
    return hipGetLastError();
}

// Segments of A B, small products first.  A product has one pitch for all its A and one for all its B: operands that do not agree are refused.
hipError_t add_segments(GrawaGemm &g, int planes, const Operand &a, const Operand &b, const Operand *b2)
{
    if ((b2 && b2->ld != b.ld) || (g.nseg && (g.lda != a.ld || g.ldb != b.ld))) return hipErrorInvalidValue;
    static const int pairs[6][2] = {{0, 2}, {2, 0}, {1, 1}, {0, 1}, {1, 0}, {0, 0}};
    const int n = planes == 1 ? 1 : 6;
    for (int i = 0; i < n; ++i) {
        const int *q = planes == 1 ? pairs[5] : pairs[i];
        g.a[g.nseg] = GrawaSeg{a.p + q[0] * a.plane, a.worker};
        g.b[g.nseg] = GrawaSeg{b.p + q[1] * b.plane, b.worker};
        if (b2) g.b[n + i] = GrawaSeg{b2->p + q[1] * b2->plane, b2->worker};
        ++g.nseg;
    }
    g.lda = a.ld;
    g.ldb = b.ld;
    return hipSuccess;
}

struct Sublayer { // one call
    const grawa_sublayer *s;
    int64_t T;
    hipStream_t st;
    hipError_t err = hipSuccess;

    int S() const { return s->dtype == GRAWA_BF16 ? 2 : 4; }
    CopyJobs copies{};
    int64_t most = 0; // groups of eight of the largest copy

    // An operand read in place where it can be, else a copy in `room`, which copy_all() makes.
    bool in_place(const char *p, int64_t worker, int64_t row, int64_t C) const
    {
        return s->planes == 1 && C % 8 == 0 && !(((uintptr_t)p | (uint64_t)worker * 2 | (uint64_t)row * 2) & 15) && row >= C && row * 2 <= MAX_LD;
    }
    Operand operand(const char *p, int64_t worker, int64_t row, int64_t R, int64_t C, int64_t Cp, char *room, bool here)
    {
        if (here) return Operand{p, worker * 2, 0, row * 2};
        const Operand o{room, R * Cp * 2, (int64_t)s->K * R * Cp * 2, Cp * 2};
        copies.job[copies.n++] = CopyJob{p, room, worker, row, o.plane, (uint32_t)R, (uint32_t)C, (uint32_t)Cp};
        most = most > R * ((C + 7) / 8) ? most : R * ((C + 7) / 8);
        return o;
    }
    void copy_all()
    {
        if (!copies.n) return;
        const int64_t blocks = (most + 255) / 256;
        const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), (unsigned)s->K, (unsigned)copies.n);
        run([&] {
            if (s->planes == 1)
                k_planes<true><<<grid, 256, 0, st>>>(copies);
            else
                k_planes<false><<<grid, 256, 0, st>>>(copies);
            return hipGetLastError();
        });
    }
    // The same of what a forward pass left in `room`.
    Operand kept(int64_t R, int64_t Cp, char *room) const { return Operand{room, R * Cp * 2, (int64_t)s->K * R * Cp * 2, Cp * 2}; }
    Operand tokens(const GrawaRows &x, char *room) { return operand(x.p, x.worker, x.row, T, s->d, s->dp, room, in_place(x.p, x.worker, x.row, s->d)); }
    // Wg and Wu are operands of one product, which has one pitch: both are read in place, or both are copied.
    void up_matrices(const GrawaMat &wg, const GrawaMat &wu, char *room_g, char *room_u, Operand &g, Operand &u)
    {
        const bool here = in_place(wg.p, wg.worker, s->d, s->d) && in_place(wu.p, wu.worker, s->d, s->d);
        g = operand(wg.p, wg.worker, s->d, s->f, s->d, s->dp, room_g, here);
        u = operand(wu.p, wu.worker, s->d, s->f, s->d, s->dp, room_u, here);
    }
    Operand down_matrix(const GrawaMat &w, char *room) { return operand(w.p, w.worker, s->f, s->d, s->f, s->fp, room, in_place(w.p, w.worker, s->f, s->f)); }
    Operand inner(char *p) const { return Operand{p, T * s->fp * 2, s->K * T * s->fp * 2, s->fp * 2}; }
    GrawaGemm product(int64_t M, int64_t N, int64_t len) const
    {
        GrawaGemm g{};
        g.K = g.one = s->K;
        g.M = (int)M;
        g.N = (int)N;
        g.len = (int)len;
        return g;
    }
    template <class F> void run(const F &f)
    {
        if (err == hipSuccess) err = f();
    }
};

// Where the copies of x and of the matrices go: with float32 and more than a few tokens into the buffer that the backward pass gets (it
// would make the same ones again: 85 of 1150 us with 4 x 512 tokens, 1024 x 4096), else into the workspace.
struct Kept {
    char *x, *wg, *wu, *wd;
};

Kept kept_in(const grawa_sublayer *s, int64_t T, char *save)
{
    if (!save || !grawa_keeps_copies(s, T)) return Kept{s->x, s->wg, s->wu, s->wd};
    const int64_t tokens = 6 * s->K * T * s->dp, up = 6 * s->K * s->f * s->dp;
    char *p = save + grawa_save_bytes_own(s, T);
    return Kept{p, p + tokens, p + tokens + up, p + tokens + 2 * up};
}

// A product of at most GRAWA_FEW tokens.
template <bool BF16, bool DUAL, bool PLANES, class Epi> hipError_t launch_few(const GrawaFew &g, int K, const Epi &epi, hipStream_t st)
{
    const int mt = (g.M + 15) / 16, columns = few_columns(mt, DUAL);
    const dim3 grid((unsigned)((g.N + columns - 1) / columns), (unsigned)K);
    // Eight waves share k where the columns alone give few waves.
    const unsigned threads = (int64_t)grid.x * K < 1024 ? 512 : 256;
    if (mt == 1) k_few<BF16, 1, DUAL, PLANES, Epi><<<grid, threads, 0, st>>>(g, epi);
    else if (mt == 2) k_few<BF16, 2, DUAL, PLANES, Epi><<<grid, threads, 0, st>>>(g, epi);
    else if constexpr (BF16) return hipErrorInvalidValue; // more than 32 tokens do not come here
    else if (mt == 3) k_few<BF16, 3, DUAL, PLANES, Epi><<<grid, threads, 0, st>>>(g, epi);
    else k_few<BF16, 4, DUAL, PLANES, Epi><<<grid, threads, 0, st>>>(g, epi);
    return hipGetLastError();
}

template <int PLANES, int ACT> hipError_t forward(Sublayer c, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd, GrawaRows residual, GrawaDrop drop, GrawaRows y, char *save)
{
    const grawa_sublayer *s = c.s;
    const int64_t n = c.T * s->fp;
    const int64_t blocks = grawa_round16(c.T) * grawa_round16(s->f);
    char *h = save ? save + s->K * blocks * grawa_kept_bytes(s) : s->h;
    const EpiGateUp<PLANES, ACT> inner{h, {save, s->K * blocks}, s->K * n * 2, n, blocks, (int)s->f, (int)s->fp, 0};
    const EpiStore<PLANES == 1, true> outer{y, residual, drop, (int)s->d, (int)c.T, 0, 0, GrawaMat{}, s->K};
    // Few tokens: see grawa_few.h.  To the end in float32, which tiles multiply six times: 4 workers, 1024 x 4096, 64 tokens 189 us, by tiles
    // 240.  In bfloat16 up to 16 tokens, and up to 32 while no axis is long (one block then goes along it by itself) and the matrices are small.  us
    // by k_few and by tiles, the matrices in no cache, K x (d x f).  16 tokens: 4 x (1024 x 4096) 25.6 and 35.2, 1 x (4096 x 11264) 61.3 and 58.1, 1 x (1024 x
    // 16384) 45.3 and 40.8.  17 and 32 tokens: 1 x (4096 x 4096) 32.7, 36.9 and 36.1, 36.1; 4 x (1024 x 4096) 32.0, 37.8 and 36.5, 36.7; 4 x (2048 x
    // 2048) 27.8, 31.9 and 36.0, 36.4; 256 x (256 x 256) 35.7, 39.7 and 32.3, 33.2; beyond: 8 x (1024 x 4096) 48.5, 56.3 and 50.4, 51.0; 1 x (1536
    // x 6144) 34.9, 40.4 and 30.2, 29.8; 1 x (8192 x 1024) 33.4, 38.8 and 29.6, 29.6; 1 x (1024 x 16384) 66.7, 78.2 and 41.1, 41.3.  With the matrices
    // in a cache tiles gain up to 8 us on these figures, k_few 2.
    constexpr bool BF16 = PLANES == 1;
    const bool small = s->d <= 4096 && s->f <= 4096 && s->K * s->d * s->f <= (int64_t)1 << 24;
    if (c.T <= (!BF16 ? GRAWA_FEW : small ? 32 : 16)) {
        constexpr int S = BF16 ? 2 : 4;
        GrawaFew g{(int)c.T, (int)s->f, (int)s->d, {wg.p, wg.worker * S}, {wu.p, wu.worker * S}, x.p, x.worker * S, x.row * S, 0};
        c.run([&] { return launch_few<BF16, true, false>(g, s->K, inner, c.st); });
        g = GrawaFew{(int)c.T, (int)s->d, (int)s->f, {wd.p, wd.worker * S}, {}, h, n * 2, s->fp * 2, s->K * n * 2};
        c.run([&] { return launch_few<BF16, false, !BF16>(g, s->K, outer, c.st); });
        return c.err;
    }
    // The split copies of float32 go to where the backward pass finds them, if one follows.
    const Kept at = kept_in(s, c.T, save);
    const Operand ox = c.tokens(x, at.x), od = c.down_matrix(wd, at.wd);
    Operand og, ou;
    c.up_matrices(wg, wu, at.wg, at.wu, og, ou);
    c.copy_all();
    {
        GrawaGemm g = c.product(c.T, s->f, s->d);
        c.run([&] { return add_segments(g, PLANES, ox, og, &ou); });
        c.run([&] { return launch_gemm<false, false, true, BF16>(s, g, inner, c.st); });
    }
    {
        GrawaGemm g = c.product(c.T, s->d, s->f);
        c.run([&] { return add_segments(g, PLANES, c.inner(h), od, nullptr); });
        c.run([&] { return launch_gemm<false, false, false, BF16>(s, g, outer, c.st); });
    }
    return c.err;
}

template <int PLANES, int ACT>
hipError_t backward(Sublayer c, GrawaRows dy, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd, const char *save, GrawaRows dx, GrawaMat dwg, GrawaMat dwu, GrawaMat dwd, int accumulate)
{
    const grawa_sublayer *s = c.s;
    const bool have = grawa_keeps_copies(s, c.T);
    const Kept at = kept_in(s, c.T, (char *)save);
    const Operand ody = c.tokens(dy, s->dy), ox = have ? c.kept(c.T, s->dp, at.x) : c.tokens(x, at.x);
    Operand og = c.kept(s->f, s->dp, at.wg), ou = c.kept(s->f, s->dp, at.wu);
    if (!have) c.up_matrices(wg, wu, at.wg, at.wu, og, ou);
    const Operand od = have ? c.kept(s->d, s->fp, at.wd) : c.down_matrix(wd, at.wd);
    c.copy_all();
    const int64_t n = c.T * s->fp;
    const int64_t blocks = grawa_round16(c.T) * grawa_round16(s->f);
    const Operand oh = c.inner((char *)save + s->K * blocks * grawa_kept_bytes(s)), odg = c.inner(s->dg), odu = c.inner(s->du);
    typedef EpiStore<PLANES == 1, false> Store;
    auto weight_product = [&](const Operand &a, const Operand &b, int64_t M, int64_t N) {
        GrawaGemm g = c.product(M, N, c.T);
        c.run([&] { return add_segments(g, PLANES, a, b, nullptr); });
        return g;
    };
    auto weight_store = [&](GrawaMat w, int64_t N, GrawaMat second) { return Store{GrawaRows{w.p, w.worker, N}, GrawaRows{}, GrawaDrop{}, (int)N, 0, accumulate, 0, second, s->K}; };
    {
        GrawaGemm g = c.product(c.T, s->f, s->d);
        c.run([&] { return add_segments(g, PLANES, ody, od, nullptr); });
        const EpiBack<PLANES, ACT> epi{{(char *)save, s->K * blocks}, s->dg, s->du, s->K * n * 2, n, blocks, (int)s->f, (int)s->fp, 0};
        c.run([&] { return launch_gemm<false, true, false, true>(s, g, epi, c.st); });
    }
    // dWg and dWu: in one launch while one of them gives a CU no more than a tile: 2 x 54 tokens, 192 x 64, 48 -> 42 us for a whole
    // training pass.  One after the other beyond: 8192 tokens, 4096 x 11264, 5225 us, side by side 5275.
    GrawaGemm gate = weight_product(odg, ox, s->f, s->d);
    const GrawaGemm up = weight_product(odu, ox, s->f, s->d);
    if (s->K * ((s->f + 255) / 256) * ((s->d + 255) / 256) <= 256) {
        for (int i = 0; i < up.nseg; ++i) gate.a[gate.nseg + i] = up.a[i];
        gate.K = 2 * s->K;
        c.run([&] { return launch_gemm<true, true, false, false>(s, gate, weight_store(dwg, s->d, dwu), c.st); });
    } else {
        c.run([&] { return launch_gemm<true, true, false, false>(s, gate, weight_store(dwg, s->d, GrawaMat{}), c.st); });
        c.run([&] { return launch_gemm<true, true, false, false>(s, up, weight_store(dwu, s->d, GrawaMat{}), c.st); });
    }
    const GrawaGemm down = weight_product(ody, oh, s->d, s->f);
    c.run([&] { return launch_gemm<true, true, false, false>(s, down, weight_store(dwd, s->f, GrawaMat{}), c.st); });
    {
        GrawaGemm g = c.product(c.T, s->d, s->f);
        c.run([&] { return add_segments(g, PLANES, odg, og, nullptr); });
        c.run([&] { return add_segments(g, PLANES, odu, ou, nullptr); });
        const Store epi{dx, GrawaRows{}, GrawaDrop{}, (int)s->d, 0, 0, 0, GrawaMat{}, s->K};
        c.run([&] { return launch_gemm<false, true, false, true>(s, g, epi, c.st); });
    }
    return c.err;
}

// Gradients of no tokens.
template <bool BF16> __global__ __launch_bounds__(256) void k_zero(GrawaMat w, int64_t n)
{
    constexpr int S = BF16 ? 2 : 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
        store_one<BF16>(w.p + ((int64_t)blockIdx.y * w.worker + i) * S, 0.f);
}

#define GRAWA_FFN_FORMS(GO)                                                                                        \
    do {                                                                                                           \
        if (s->planes == 1) {                                                                                      \
            if (s->act == GRAWA_ACT_SILU) return GO(1, GRAWA_ACT_SILU);                                            \
            return s->act == GRAWA_ACT_GELU ? GO(1, GRAWA_ACT_GELU) : GO(1, GRAWA_ACT_RELU);                       \
        }                                                                                                          \
        if (s->act == GRAWA_ACT_SILU) return GO(3, GRAWA_ACT_SILU);                                                \
        return s->act == GRAWA_ACT_GELU ? GO(3, GRAWA_ACT_GELU) : GO(3, GRAWA_ACT_RELU);                           \
    } while (0)

} // namespace

// Enough for every product of a call of at most T tokens: MAX_SPLITS parts of the largest one, but no more than a product's parts may
// take.
int64_t grawa_ffn_part_floats(const grawa_sublayer *s)
{
    const int64_t t = grawa_round16(s->T), d = grawa_round16(s->d), f = grawa_round16(s->f);
    int64_t most = 2 * t * f;
    for (const int64_t n : {t * d, d * f}) most = most > n ? most : n;
    most *= s->K * MAX_SPLITS;
    return most < PART_FLOATS ? most : PART_FLOATS;
}

hipError_t grawa_launch_ffn(const grawa_sublayer *s, int64_t T, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd, GrawaRows residual,
                            GrawaDrop drop, GrawaRows y, char *save, hipStream_t st)
{
    if (!T) return hipSuccess;
    const Sublayer c{s, T, st};
#define GO(P, A) forward<P, A>(c, x, wg, wu, wd, residual, drop, y, save)
    GRAWA_FFN_FORMS(GO);
#undef GO
}

hipError_t grawa_launch_ffn_backward(const grawa_sublayer *s, int64_t T, GrawaRows dy, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd,
                                     const char *save, GrawaRows dx, GrawaMat dwg, GrawaMat dwu, GrawaMat dwd, int accumulate,
                                     hipStream_t st)
{
    if (!T) {
        if (accumulate) return hipSuccess;
        const dim3 grid(256, (unsigned)s->K);
        for (const GrawaMat &w : {dwg, dwu, dwd}) {
            if (s->dtype == GRAWA_BF16)
                k_zero<true><<<grid, 256, 0, st>>>(w, s->d * s->f);
            else
                k_zero<false><<<grid, 256, 0, st>>>(w, s->d * s->f);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const Sublayer c{s, T, st};
#define GO(P, A) backward<P, A>(c, dy, x, wg, wu, wd, save, dx, dwg, dwu, dwd, accumulate)
    GRAWA_FFN_FORMS(GO);
#undef GO
}
