// Products of a few tokens with a whole matrix: C[m][n] = sum over k of A[m][k] B[n][k] for at most 64 rows m.  They are bound by reading B
// once.  A wave takes some columns (of each of two matrices, DUAL; more of them where there are more rows, so that the rows, which come
// from L2 again for every wave, do not outweigh B), goes straight from memory to the matrix instructions, and asks for the next
// piece of each row before it works on the one it has; the waves of a block share k and add their sums in LDS, in order.
// Elements are read where they are, at any alignment: no copy of a matrix is made, and float32 is multiplied as float32.
// One token of each of four workers, 1024 x 4096 in bfloat16, 101 MB of matrices: 12.3 and 8.4 us, 5.4 and 4.0 TB/s.  Loads past the caches
// make it 22.9 us instead of 20.9 as a whole, and are no faster where other data has passed through the caches in between (26.4, 24.6).
#pragma once
#include "grawa_gemm.h"

constexpr int GRAWA_FEW_WAVES = 8; // most waves of a block

struct GrawaFew {
    int M, N, len;
    GrawaSeg b, b2;       // matrices, len elements a row
    const char *a;        // rows, bytes apart
    int64_t a_worker, a_row, a_plane; // a_plane: not 0 where A is three planes of bfloat16 for a float32
};

namespace {

// What a lane holds of a step of 64 bytes of k (of float32 16 k, of bfloat16 32): 16 bytes, k = 16 / S (lane / 16) ... of row lane % 16.
struct GrawaStep {
    uint32_t w[4];
};

template <bool BF16> __device__ __forceinline__ GrawaStep few_load(const char *p)
{
    const GrawaAny16 v = *(const GrawaAny16 *)p;
    return GrawaStep{{v.x, v.y, v.z, v.w}};
}

// The same where only `n` elements of the row are left.
template <bool BF16> __device__ __forceinline__ GrawaStep few_load_end(const char *p, int n)
{
    GrawaStep s{};
    if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) s.w[j / 2] |= (uint32_t)((const uint16_t *)p)[j] << (j % 2 * 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) s.w[j] = ((const uint32_t *)p)[j];
    }
    return s;
}

// Float32 from its three planes, which add up to it exactly; the row holds zeros behind its end.
__device__ __forceinline__ GrawaStep few_load_planes(const char *p, int64_t plane)
{
    GrawaStep s;
    const GrawaAny8 a = *(const GrawaAny8 *)p, b = *(const GrawaAny8 *)(p + plane), c = *(const GrawaAny8 *)(p + 2 * plane);
    const uint32_t x[2] = {a.x, a.y}, y[2] = {b.x, b.y}, z[2] = {c.x, c.y};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t u = j % 2 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16, v = j % 2 ? y[j / 2] & 0xffff0000u : y[j / 2] << 16,
                       w = j % 2 ? z[j / 2] & 0xffff0000u : z[j / 2] << 16;
        s.w[j] = __float_as_uint(__uint_as_float(u) + (__uint_as_float(v) + __uint_as_float(w)));
    }
    return s;
}

template <bool BF16> __device__ __forceinline__ void few_mfma(grawa_f32x4 &c, const GrawaStep &b, const GrawaStep &a)
{
    if constexpr (BF16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(grawa_bf16x8, b), __builtin_bit_cast(grawa_bf16x8, a), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.w[j]), __uint_as_float(a.w[j]), c, 0, 0, 0);
    }
}

// Columns of a product that a wave takes, and steps that it has in flight twice: up to sixteen rows, and of two matrices, one fragment of each
// matrix, else two; 256 bytes of each row up to 32 rows, 128 above.
constexpr int few_columns(int mt, bool dual) { return mt == 1 || dual ? 16 : 32; }
constexpr int few_chunk(int mt) { return mt <= 2 ? 4 : 2; }

template <bool BF16, int MT, bool DUAL, bool PLANES, class Epi>
__global__ __launch_bounds__(GRAWA_FEW_WAVES * 64, 1) void k_few(GrawaFew g, Epi epi)
{
    constexpr int S = BF16 ? 2 : 4, KS = 64 / S, CHUNK = few_chunk(MT); // k of a step, steps of a chunk
    constexpr int NF = few_columns(MT, DUAL) / 16, NB = DUAL ? 2 * NF : NF; // fragments of a product and of B a step
    __shared__ __attribute__((aligned(16))) float sums[GRAWA_FEW_WAVES][MT * NB][256];
    static_assert(MT * NB <= 8, "64 KiB at most");
    __shared__ __attribute__((aligned(16))) float corners[GRAWA_FEW_WAVES][Epi::OUTS * 256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, k = blockIdx.y;
    const int q = lane >> 4, n0 = blockIdx.x * (16 * NF);
    const char *pb[NB], *pa[MT];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const GrawaSeg &s = j >= NF ? g.b2 : g.b;
        const int n = n0 + j % NF * 16 + (lane & 15);
        pb[j] = s.p + k * s.worker + (int64_t)(n < g.N ? n : g.N - 1) * g.len * S + q * 16; // rows that are not there: their sums are not used
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = i * 16 + (lane & 15);
        pa[i] = g.a + k * g.a_worker + (int64_t)(m < g.M ? m : g.M - 1) * g.a_row + q * (PLANES ? 8 : 16);
    }
    auto load_a = [&](int i, int64_t step) { return PLANES ? few_load_planes(pa[i] + step * 32, g.a_plane) : few_load<BF16>(pa[i] + step * 64); };
    grawa_f32x4 acc[MT][NB] = {};
    const int steps = g.len / KS, chunks = steps / CHUNK;
    GrawaStep b[2][CHUNK][NB], a[2][CHUNK][MT];
    auto load = [&](int to, int c) {
#pragma unroll
        for (int s = 0; s < CHUNK; ++s) {
#pragma unroll
            for (int j = 0; j < NB; ++j) b[to][s][j] = few_load<BF16>(pb[j] + ((int64_t)c * CHUNK + s) * 64);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[to][s][i] = load_a(i, (int64_t)c * CHUNK + s);
        }
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int s = 0; s < CHUNK; ++s)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) few_mfma<BF16>(acc[i][j], b[from][s][j], a[from][s][i]);
    };
    if (wave < chunks) load(0, wave);
    for (int c = wave; c < chunks; c += 2 * waves) {
        if (c + waves < chunks) load(1, c + waves);
        multiply(0);
        if (c + waves >= chunks) break;
        if (c + 2 * waves < chunks) load(0, c + 2 * waves);
        multiply(1);
    }
    // What is left: fewer steps than a chunk, and fewer k than a step.
    for (int step = chunks * CHUNK + wave; step * KS < g.len; step += waves) {
        const int left = g.len - step * KS - q * (16 / S); // elements from the lane's own on
        GrawaStep a[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (step < steps)
                a[i] = load_a(i, step);
            else if (PLANES)
                a[i] = left > 0 ? load_a(i, step) : GrawaStep{};
            else
                a[i] = few_load_end<BF16>(pa[i] + (int64_t)step * 64, left);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const GrawaStep t = step < steps ? few_load<BF16>(pb[j] + (int64_t)step * 64) : few_load_end<BF16>(pb[j] + (int64_t)step * 64, left);
#pragma unroll
            for (int i = 0; i < MT; ++i) few_mfma<BF16>(acc[i][j], t, a[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *(grawa_f32x4 *)&sums[wave][i * NB + j][lane * 4] = acc[i][j];
    __syncthreads();
    epi.tile(k, 0);
    for (int t = wave; t < MT * NF; t += waves) {
        const int i = t / NF, j = t % NF;
        grawa_f32x4 v[1] = {}, u[1] = {};
        for (int w = 0; w < waves; ++w) {
            v[0] += *(const grawa_f32x4 *)&sums[w][i * NB + j][lane * 4];
            if (DUAL) u[0] += *(const grawa_f32x4 *)&sums[w][i * NB + NF + j][lane * 4];
        }
        typename Epi::Ahead r[1]; // the epilogues of these products read nothing
        if (i * 16 < g.M && n0 + j * 16 < g.N) grawa_finish<1>(epi, corners[wave], i * 16, n0 + j * 16, lane, g.M, g.N, r, v, u);
    }
}

} // namespace
