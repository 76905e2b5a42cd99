// Norms of the heads of queries and keys with the position rotation, forward and backward, each worker with its own weights:
//   r = (sum x^2 / D + eps)^(-1/2);  n = x r w;  y = n turned by position * frequency in R / 2 pairs, (e, e + R / 2) or (2 e, 2 e + 1)
//   dn = dy turned back;  a = dn w;  dx = r (a - x r mean(a x r));  dw = sum over tokens and heads of dn x r
// An angle is formed in turns, position times turns a position in 64 bits, of which the whole turns are dropped before the rest is
// rounded to 32: far positions are as exact as near ones.  The angles of a token serve several of its heads, and a row is read once.
// Sums over tokens are kept in registers, left in a workspace by each block and added in order by a second launch.
#include "grawa_attention.h"
#include "grawa_elements.h"

namespace {

struct HeadNorm {
    GrawaHeads q, k, yq, yk, gq, gk; // forward: x and y; backward: x, dx (in yq, yk) and dy
    GrawaMat wq, wk, dwq, dwk;
    const int *starts;
    const double *turns;
    float *part;
    float eps;
    int N, S, H, G, D, rotary, interleaved;
    int heads; // of an item: so many rows share a token's angles
    int accumulate;
};

#ifdef __HIP_DEVICE_COMPILE__
template <bool BF16> struct Eight {
    float v[8];
    __device__ __forceinline__ void load(const char *p, bool there)
    {
        constexpr int N = GrawaPiece<BF16>::N;
        GrawaPiece<BF16> piece;
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) {
            if (there) {
                piece.load(p + i * 16, N);
#pragma unroll
                for (int j = 0; j < N; ++j) v[i * N + j] = piece[j];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[i * N + j] = 0.f;
            }
        }
    }
    __device__ __forceinline__ void store(char *p) const
    {
        constexpr int N = GrawaPiece<BF16>::N;
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) store_piece<BF16>(p + i * 16, N, v + i * N);
    }
};

template <int LPR> __device__ __forceinline__ float row_total(float v)
{
#pragma unroll
    for (int m = 1; m < LPR; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// Elements e0 ... e0 + 7 of a row and what they are turned with.
struct Turn {
    float cos[8], sin[8]; // sin with the sign that it has in y_e = x_e cos + x_partner sin
    int partner;          // first of the partners, where pairs are halves apart
    bool whole;           // they are read by fours

    __device__ __forceinline__ void init(const HeadNorm &a, int64_t position, int e0)
    {
        const int half = a.rotary / 2;
        partner = e0;
        whole = half % 4 == 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = e0 + j;
            cos[j] = 1.f;
            sin[j] = 0.f;
            if (e >= a.rotary) continue;
            if (a.interleaved && j % 2) {
                cos[j] = cos[j - 1];
                sin[j] = -sin[j - 1];
                continue;
            }
            const bool second = !a.interleaved && e >= half;
            const double turns = (double)position * a.turns[a.interleaved ? e / 2 : second ? e - half : e];
            const float part = (float)(2.0 * (turns - __builtin_rint(turns))); // of half a turn
            float s, c;
            s = sinpif(part);
            c = cospif(part);
            cos[j] = c;
            sin[j] = second ? s : -s;
        }
    }
    static __device__ __forceinline__ int partner_of(const HeadNorm &a, int e)
    {
        const int half = a.rotary / 2;
        return e < half ? e + half : e < a.rotary ? e - half : e;
    }
    // The partners of v; row: the wave's own place in LDS for a row.
    __device__ __forceinline__ void partners(const HeadNorm &a, const float *v, float *row, int e0, float *p) const
    {
        if (a.interleaved || a.rotary == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = v[j ^ 1];
            return;
        }
        *(float4 *)(row + e0) = make_float4(v[0], v[1], v[2], v[3]);
        *(float4 *)(row + e0 + 4) = make_float4(v[4], v[5], v[6], v[7]);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
        if (whole) {
            const float4 x = *(const float4 *)(row + partner_of(a, e0)), y = *(const float4 *)(row + partner_of(a, e0 + 4));
            p[0] = x.x, p[1] = x.y, p[2] = x.z, p[3] = x.w, p[4] = y.x, p[5] = y.y, p[6] = y.z, p[7] = y.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = row[partner_of(a, e0 + j)];
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
    }
};

__device__ __forceinline__ int64_t byte_of(const GrawaHeads &h, int k, int n, int s, int head)
{
    return (int64_t)k * h.worker + (int64_t)n * h.seq + (int64_t)s * h.token + (int64_t)head * h.head;
}
#endif

// LPR lanes have a row of up to 8 LPR elements.  An item is `heads` rows of a token; blocks of a worker take items in turn.
template <bool BF16, int LPR, bool BACK> __global__ __launch_bounds__(256) void k_head_norm([[maybe_unused]] HeadNorm a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int ROWS = 256 / LPR, DP = LPR * 8, ES = BF16 ? 2 : 4, U = BACK ? 2 : 4;
    __shared__ float lds[BACK ? ROWS * 2 * DP : ROWS * DP];
    const int row = threadIdx.x / LPR, e0 = threadIdx.x % LPR * 8, k = blockIdx.y;
    const bool there = e0 < a.D;
    const int all = a.H + a.G, chunks = (all + a.heads - 1) / a.heads;
    const int64_t items = (int64_t)a.N * a.S * chunks;
    Eight<BF16> wq, wk;
    wq.load(a.wq.p + ((int64_t)k * a.wq.worker + e0) * ES, there);
    wk.load(a.wk.p + ((int64_t)k * a.wk.worker + e0) * ES, there);
    float sq[8], sk[8];
    if (BACK)
#pragma unroll
        for (int j = 0; j < 8; ++j) sq[j] = sk[j] = 0.f;
    // all rows of a wave go round alike: what a wave's last items do not have is left out row by row
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < items; base += (int64_t)gridDim.x * ROWS) {
        const int64_t item = base + row;
        const bool live = item < items;
        const int64_t token = live ? item / chunks : 0;
        const int h0 = live ? (int)(item - token * chunks) * a.heads : all, h1 = min(h0 + a.heads, all);
        const int n = (int)(token / a.S), s = (int)(token - (int64_t)n * a.S);
        Turn turn;
        turn.init(a, (a.starts ? (int64_t)a.starts[k * a.N + n] : 0) + s, e0);
        for (int first = 0; first < a.heads; first += U) {
            Eight<BF16> x[U], g[BACK ? U : 1];
#pragma unroll
            for (int u = 0; u < U; ++u) { // all on their way before the first is waited for
                const int h = h0 + first + u;
                const bool has = there && first + u < a.heads && h < h1;
                const bool key = h >= a.H;
                x[u].load((key ? a.k.p + byte_of(a.k, k, n, s, h - a.H) : a.q.p + byte_of(a.q, k, n, s, h)) + e0 * ES, has);
                if constexpr (BACK) g[u].load((key ? a.gk.p + byte_of(a.gk, k, n, s, h - a.H) : a.gq.p + byte_of(a.gq, k, n, s, h)) + e0 * ES, has);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + first + u;
                const bool has = there && first + u < a.heads && h < h1, key = h >= a.H;
                float squares = 0.f, p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) squares += x[u].v[j] * x[u].v[j];
                const float r = 1.f / sqrtf(row_total<LPR>(squares) / (float)a.D + a.eps);
                Eight<BF16> y;
                if constexpr (!BACK) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) y.v[j] = x[u].v[j] * r * (key ? wk.v[j] : wq.v[j]);
                    turn.partners(a, y.v, lds + row * DP, e0, p);
#pragma unroll
                    for (int j = 0; j < 8; ++j) y.v[j] = e0 + j >= a.rotary ? y.v[j] * turn.cos[j] : y.v[j] * turn.cos[j] + p[j] * turn.sin[j];
                } else {
                    turn.partners(a, g[u].v, lds + row * DP, e0, p);
                    float dot = 0.f, c[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float dn = e0 + j >= a.rotary ? g[u].v[j] * turn.cos[j] : g[u].v[j] * turn.cos[j] - p[j] * turn.sin[j];
                        x[u].v[j] *= r;
                        c[j] = dn * x[u].v[j];
                        y.v[j] = dn * (key ? wk.v[j] : wq.v[j]);
                        dot += y.v[j] * x[u].v[j];
                    }
                    dot = row_total<LPR>(dot) / (float)a.D;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        y.v[j] = r * (y.v[j] - x[u].v[j] * dot);
                        if (has && key) sk[j] += c[j];
                        if (has && !key) sq[j] += c[j];
                    }
                }
                if (has) y.store((key ? a.yk.p + byte_of(a.yk, k, n, s, h - a.H) : a.yq.p + byte_of(a.yq, k, n, s, h)) + e0 * ES);
            }
        }
    }
    if constexpr (BACK) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lds[(row * 2) * DP + e0 + j] = sq[j];
            lds[(row * 2 + 1) * DP + e0 + j] = sk[j];
        }
        __syncthreads();
        const int which = threadIdx.x / DP, e = threadIdx.x % DP;
        if (which < 2 && e < a.D) {
            float sum = 0.f;
            for (int i = 0; i < ROWS; ++i) sum += lds[(i * 2 + which) * DP + e];
            a.part[(((int64_t)k * gridDim.x + blockIdx.x) * 2 + which) * a.D + e] = sum;
        }
    }
#endif
}

// Gradients of the weights from the sums of `blocks` blocks, each thread an eighth of them.
template <bool BF16> __global__ __launch_bounds__(1024) void k_head_sums([[maybe_unused]] HeadNorm a, [[maybe_unused]] int blocks)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float lds[8][128];
    const int e = threadIdx.x % 128, part = threadIdx.x / 128, which = blockIdx.x, k = blockIdx.y;
    float sum = 0.f;
    if (e < a.D)
        for (int i = part; i < blocks; i += 8) sum += a.part[(((int64_t)k * blocks + i) * 2 + which) * a.D + e];
    lds[part][e] = sum;
    __syncthreads();
    if (part || e >= a.D) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) sum += lds[i][e];
    const GrawaMat &to = which ? a.dwk : a.dwq;
    char *out = to.p + ((int64_t)k * to.worker + e) * (BF16 ? 2 : 4);
    store_one<BF16>(out, a.accumulate ? load_one<BF16>(out) + sum : sum);
#endif
}

// How many rows share a token's angles: more of them where there are rows enough to fill the card.
int heads_of(const grawa_attention_plan *s, int64_t tokens)
{
    const int64_t rows = (int64_t)s->K * tokens * (s->H + s->G);
    return rows >= 1 << 18 ? 16 : rows >= 1 << 15 ? 8 : 4;
}

template <bool BACK> hipError_t launch(const grawa_attention_plan *s, HeadNorm a, int blocks, hipStream_t st)
{
    const dim3 grid((uint32_t)blocks, (uint32_t)s->K);
    if (s->dtype == GRAWA_BF16) {
        if (s->D <= 64)
            hipLaunchKernelGGL((k_head_norm<true, 8, BACK>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_head_norm<true, 16, BACK>), grid, dim3(256), 0, st, a);
    } else {
        if (s->D <= 64)
            hipLaunchKernelGGL((k_head_norm<false, 8, BACK>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_head_norm<false, 16, BACK>), grid, dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

int64_t blocks_of(const grawa_attention_plan *s, int64_t tokens, int heads, int64_t most)
{
    const int rows = s->D <= 64 ? 32 : 16;
    const int64_t items = tokens * ((s->H + s->G + heads - 1) / heads), b = (items + rows - 1) / rows;
    return b < most ? b : most;
}

} // namespace

int grawa_head_norm_blocks(const grawa_attention_plan *s)
{
    const int64_t most = 2048 / s->K > 1 ? 2048 / s->K : 1, b = blocks_of(s, s->N * s->S, 4, most);
    return b < 1 ? 1 : (int)b;
}

hipError_t grawa_launch_head_norm(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads q, GrawaHeads k, GrawaMat qw, GrawaMat kw, float eps,
                                  const int *starts, GrawaHeads qo, GrawaHeads ko, hipStream_t st)
{
    if (N * S == 0) return hipSuccess;
    HeadNorm a{};
    a.q = q, a.k = k, a.yq = qo, a.yk = ko, a.wq = qw, a.wk = kw, a.starts = starts, a.turns = s->turns, a.eps = eps;
    a.N = (int)N, a.S = (int)S, a.H = s->H, a.G = s->G, a.D = s->D, a.rotary = s->rotary, a.interleaved = s->interleaved;
    a.heads = heads_of(s, N * S);
    return launch<false>(s, a, (int)blocks_of(s, N * S, a.heads, 1 << 20), st);
}

hipError_t grawa_launch_head_norm_backward(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads dqo, GrawaHeads dko, GrawaHeads q, GrawaHeads k,
                                           GrawaMat qw, GrawaMat kw, float eps, const int *starts, GrawaHeads dq, GrawaHeads dk, GrawaMat dqw,
                                           GrawaMat dkw, int accumulate, hipStream_t st)
{
    HeadNorm a{};
    a.q = q, a.k = k, a.yq = dq, a.yk = dk, a.gq = dqo, a.gk = dko, a.wq = qw, a.wk = kw, a.dwq = dqw, a.dwk = dkw;
    a.starts = starts, a.turns = s->turns, a.part = s->norm_part, a.eps = eps, a.accumulate = accumulate;
    a.N = (int)N, a.S = (int)S, a.H = s->H, a.G = s->G, a.D = s->D, a.rotary = s->rotary, a.interleaved = s->interleaved;
    a.heads = heads_of(s, N * S);
    const int blocks = (int)blocks_of(s, N * S, a.heads, s->norm_blocks);
    if (blocks > 0) {
        const hipError_t e = launch<true>(s, a, blocks, st);
        if (e != hipSuccess) return e;
    }
    const dim3 grid(2, (uint32_t)s->K);
    if (s->dtype == GRAWA_BF16)
        hipLaunchKernelGGL((k_head_sums<true>), grid, dim3(1024), 0, st, a, blocks);
    else
        hipLaunchKernelGGL((k_head_sums<false>), grid, dim3(1024), 0, st, a, blocks);
    return hipGetLastError();
}
