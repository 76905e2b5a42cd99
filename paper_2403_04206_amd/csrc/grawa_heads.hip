// Norms of the heads of queries and keys with the position rotation, forward and backward, each worker with its own weights:
//   r = (sum x^2 / D + eps)^(-1/2);  n = x r w;  y = n turned by position * frequency in R / 2 pairs, (e, e + R / 2) or (2 e, 2 e + 1)
//   dn = dy turned back;  a = dn w;  dx = r (a - x r mean(a x r));  dw = sum over tokens and heads of dn x r
// An angle is formed in turns, position times turns a position in 64 bits, of which the whole turns are dropped before the rest is
// rounded to 32: far positions are as exact as near ones.  The angles of a token serve several of its heads, and a row is read once.
// Sums over tokens are kept in registers, left in a workspace by each block and added in order by a second launch.
#include "grawa_attention.h"
#include "grawa_elements.h"

namespace {

// How the elements of a rotation go in pairs.
enum Pairs { HALVES, NEIGHBOURS, APART };

struct HeadNorm {
    GrawaHeads q, k, yq, yk, gq, gk; // forward: x and y; backward: x, dx (in yq, yk) and dy
    GrawaMat wq, wk, dwq, dwk;
    const int *starts;
    const double *turns;
    float *part;
    float eps, least; // rows whose squares are less in all are taken larger first
    int N, S, H, G, D, rotary;
    int heads; // of an item: so many rows share a token's angles
    int accumulate;
};

#ifdef __HIP_DEVICE_COMPILE__
// Eight elements of a row, four from `lo` on and four from `hi` on, at any alignment.
template <bool BF16> struct Eight {
    float v[8];
    __device__ __forceinline__ void load(const char *p, int lo, int hi, bool there)
    {
        if constexpr (BF16) {
            GrawaAny8 x = {0, 0}, y = {0, 0};
            if (there) x = *(const GrawaAny8 *)(p + lo * 2), y = *(const GrawaAny8 *)(p + hi * 2);
            v[0] = bf16_lo(x.x), v[1] = bf16_hi(x.x), v[2] = bf16_lo(x.y), v[3] = bf16_hi(x.y);
            v[4] = bf16_lo(y.x), v[5] = bf16_hi(y.x), v[6] = bf16_lo(y.y), v[7] = bf16_hi(y.y);
        } else {
            GrawaAny16 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
            if (there) x = *(const GrawaAny16 *)(p + lo * 4), y = *(const GrawaAny16 *)(p + hi * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(x[j]), v[4 + j] = __uint_as_float(y[j]);
        }
    }
    __device__ __forceinline__ void store(char *p, int lo, int hi) const
    {
        if constexpr (BF16) {
            typedef __bf16 B4 __attribute__((ext_vector_type(4)));
            const B4 x = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]}, y = {(__bf16)v[4], (__bf16)v[5], (__bf16)v[6], (__bf16)v[7]};
            *(GrawaAny8 *)(p + lo * 2) = __builtin_bit_cast(GrawaAny8, x);
            *(GrawaAny8 *)(p + hi * 2) = __builtin_bit_cast(GrawaAny8, y);
        } else {
            GrawaAny16 x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(v[j]), y[j] = __float_as_uint(v[4 + j]);
            *(GrawaAny16 *)(p + lo * 4) = x;
            *(GrawaAny16 *)(p + hi * 4) = y;
        }
    }
};

template <int CTRL> __device__ __forceinline__ float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum over the 8 or 16 lanes of a row: neighbours, pairs, quads from the other end, eights from the other end.
template <int LPR> __device__ __forceinline__ float row_total(float v)
{
    v += moved<0xb1>(v);
    v += moved<0x4e>(v);
    v += moved<0x141>(v);
    if constexpr (LPR == 16) v += moved<0x140>(v);
    return v;
}

// Sine and cosine of part turns, |part| <= 1/2: quarter turns off, then the series of both up to the tenth power of an angle of at most
// an eighth of a turn, where what is left out is below 2^-28.
__device__ __forceinline__ void sine_cosine(float part, float &s, float &c)
{
    const float quarters = __builtin_rintf(4.f * part), x = (4.f * part - quarters) * 1.57079633f, x2 = x * x;
    const float sx = x * (1.f + x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880)))));
    const float cx = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 - x2 * (1.f / 3628800)))));
    const int q = (int)quarters & 3;
    s = q & 1 ? cx : sx;
    c = q & 1 ? sx : cx;
    s = q & 2 ? -s : s;
    c = (q + 1) & 2 ? -c : c;
}

// What the lane's eight elements are turned with.  Pairs of neighbours are j and j ^ 1; pairs of halves are j and j ^ 4, `lo` and `hi` being
// half the rotated elements apart.  Where that half is no multiple of four the partners are APART and come from LDS.
template <Pairs P> struct Turn {
    float cos[8], sin[8]; // sin with the sign that it has in y_e = x_e cos + x_partner sin

    __device__ __forceinline__ void init(const HeadNorm &a, int64_t position, int lo, int hi)
    {
        const int half = a.rotary / 2;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = j < 4 ? lo + j : hi + j - 4;
            cos[j] = 1.f;
            sin[j] = 0.f;
            if (e >= a.rotary) continue;
            const int before = P == NEIGHBOURS ? j & 6 : P == HALVES ? j & 3 : j; // the pair's first
            if (before != j) {
                cos[j] = cos[before];
                sin[j] = -sin[before];
                continue;
            }
            const bool second = P == APART && e >= half;
            const double turns = (double)position * a.turns[P == NEIGHBOURS ? e / 2 : second ? e - half : e];
            float s;
            sine_cosine((float)(turns - __builtin_rint(turns)), s, cos[j]);
            sin[j] = second ? s : -s;
        }
    }
    // The partners of v; row: the row's own place in LDS.
    __device__ __forceinline__ void partners(const HeadNorm &a, const float *v, float *row, int lo, int hi, float *p) const
    {
        if constexpr (P == APART) {
#pragma unroll
            for (int j = 0; j < 8; ++j) row[j < 4 ? lo + j : hi + j - 4] = v[j];
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
            const int half = a.rotary / 2;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = j < 4 ? lo + j : hi + j - 4;
                p[j] = row[e < half ? e + half : e < a.rotary ? e - half : e];
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = P == NEIGHBOURS ? v[j ^ 1] : v[j ^ 4];
        }
    }
};

template <bool B> struct Is {
    static constexpr bool value = B;
};

__device__ __forceinline__ int64_t byte_of(const GrawaHeads &h, int k, int n, int s)
{
    return (int64_t)k * h.worker + (int64_t)n * h.seq + (int64_t)s * h.token;
}
#endif

// LPR lanes have a row of up to 8 LPR elements.  An item is `heads` rows of a token; blocks of a worker take items in turn.
// Bound by memory forward, and backward by it and the vector unit, which is busy 76 % of both: angles are formed in each, in 64 bits; what they
// take is shared by an item's rows, of which few heads leave many empty, and there is no exchange between lanes but a row's sums.
// 8 workers, 2048 tokens of 2 x 16 heads of 64, bf16: forward 26 us (134 MB, 5.2 TB/s), backward 44 (201 MB, 4.6 TB/s); one token 4.6.
// Rows of odd size in a pass of their own: with a way aside for each row 12 us more over 3 heads of 2^17 tokens, so 4.
template <bool BF16, int LPR, Pairs P, bool BACK> __global__ __launch_bounds__(256) void k_head_norm([[maybe_unused]] HeadNorm a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int ROWS = 256 / LPR, DP = LPR * 8, ES = BF16 ? 2 : 4, U = BACK ? 2 : 4;
    __shared__ float lds[BACK ? ROWS * 2 * DP : P == APART ? ROWS * DP : 1];
    const int row = threadIdx.x / LPR, c = threadIdx.x % LPR, k = blockIdx.y;
    const bool there = c * 8 < a.D;
    // the lane's elements: pairs of halves stay together
    const bool paired = P == HALVES && c * 8 < a.rotary;
    const int lo = paired ? 4 * c : 8 * c, hi = paired ? a.rotary / 2 + 4 * c : 8 * c + 4;
    const uint32_t all = a.H + a.G, chunks = (all + a.heads - 1) / a.heads, items = (uint32_t)a.N * a.S * chunks; // below 2^31
    Eight<BF16> wq, wk;
    wq.load(a.wq.p + (int64_t)k * a.wq.worker * ES, lo, hi, there);
    wk.load(a.wk.p + (int64_t)k * a.wk.worker * ES, lo, hi, there);
    float sq[8], sk[8];
    if (BACK)
#pragma unroll
        for (int j = 0; j < 8; ++j) sq[j] = sk[j] = 0.f;
    // all rows of a wave go round alike: what a wave's last items do not have is left out row by row
    for (uint32_t base = blockIdx.x * ROWS; base < items; base += gridDim.x * ROWS) {
        const uint32_t item = base + row;
        const bool live = item < items;
        const uint32_t token = live ? item / chunks : 0;
        const int h0 = live ? (int)(item - token * chunks) * a.heads : (int)all, h1 = min(h0 + a.heads, (int)all);
        const int n = (int)(token / (uint32_t)a.S), s = (int)(token - (uint32_t)n * a.S);
        Turn<P> turn;
        turn.init(a, (a.starts ? (int64_t)a.starts[k * a.N + n] : 0) + s, lo, hi);
        const char *pq = a.q.p + byte_of(a.q, k, n, s), *pk = a.k.p + byte_of(a.k, k, n, s) - a.H * a.k.head;
        char *yq = a.yq.p + byte_of(a.yq, k, n, s), *yk = a.yk.p + byte_of(a.yk, k, n, s) - a.H * a.yk.head;
        const char *gq = BACK ? a.gq.p + byte_of(a.gq, k, n, s) : nullptr, *gk = BACK ? a.gk.p + byte_of(a.gk, k, n, s) - a.H * a.gk.head : nullptr;
        const auto has = [&](int i) { return there && i < a.heads && h0 + i < h1; };
        const auto load = [&](int i, Eight<BF16> &x, Eight<BF16> &g) __attribute__((always_inline)) {
            const int h = h0 + i;
            const bool key = h >= a.H;
            x.load(key ? pk + h * a.k.head : pq + h * a.q.head, lo, hi, has(i));
            if constexpr (BACK) g.load(key ? gk + h * a.gk.head : gq + h * a.gq.head, lo, hi, has(i));
        };
        // Whether the row's squares are such that float32 does not hold them, or not with all their digits where eps is as small.  Such rows
        // are left as they are the first time, and formed with care, from squares of the row times a power of two, the second.
        const auto form = [&](int i, Eight<BF16> x, const Eight<BF16> &g, auto careful) __attribute__((always_inline)) {
            const int h = h0 + i;
            const bool key = h >= a.H;
            float squares = 0.f, p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) squares += x.v[j] * x.v[j];
            squares = row_total<LPR>(squares);
            const bool odd = !(squares < 0x1p120f) || squares < a.least, mine = has(i) && odd == careful.value;
            float r = 1.f / sqrtf(squares / (float)a.D + a.eps);
            if constexpr (careful.value) {
                const float f = squares < a.least ? 0x1p90f : 0x1p-70f;
                squares = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) squares += x.v[j] * f * (x.v[j] * f);
                squares = row_total<LPR>(squares) / (float)a.D + a.eps * f * f;
                r = squares > 0.f ? fminf(f / sqrtf(squares), 0x1.fffffep127f) : r; // rows of zeros beside an eps of 0 stay what they are: no numbers
            }
            Eight<BF16> y;
            if constexpr (!BACK) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x.v[j] = x.v[j] * r * (key ? wk.v[j] : wq.v[j]);
                turn.partners(a, x.v, lds + row * DP, lo, hi, p);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool turned = (j < 4 ? lo + j : hi + j - 4) < a.rotary;
                    y.v[j] = turned ? x.v[j] * turn.cos[j] + p[j] * turn.sin[j] : x.v[j];
                }
            } else {
                turn.partners(a, g.v, lds + row * DP, lo, hi, p);
                float dot = 0.f, d[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool turned = (j < 4 ? lo + j : hi + j - 4) < a.rotary;
                    const float dn = turned ? g.v[j] * turn.cos[j] - p[j] * turn.sin[j] : g.v[j];
                    x.v[j] *= r;
                    d[j] = dn * x.v[j];
                    y.v[j] = dn * (key ? wk.v[j] : wq.v[j]);
                    dot += y.v[j] * x.v[j];
                }
                dot = row_total<LPR>(dot) / (float)a.D;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y.v[j] = r * (y.v[j] - x.v[j] * dot);
                    if (mine && key) sk[j] += d[j];
                    if (mine && !key) sq[j] += d[j];
                }
            }
            if (mine) y.store(key ? yk + h * a.yk.head : yq + h * a.yq.head, lo, hi);
            return odd;
        };
        for (int first = 0; first < a.heads; first += U) {
            Eight<BF16> x[U], g[BACK ? U : 1];
            bool odd = false;
#pragma unroll
            for (int u = 0; u < U; ++u) load(first + u, x[u], g[BACK ? u : 0]); // all on their way before the first is waited for
#pragma unroll
            for (int u = 0; u < U; ++u) odd |= form(first + u, x[u], g[BACK ? u : 0], Is<false>());
            if (__builtin_expect(__any(odd), 0))
#pragma unroll 1
                for (int u = 0; u < U; ++u) {
                    load(first + u, x[0], g[0]);
                    form(first + u, x[0], g[0], Is<true>());
                }
        }
    }
    if constexpr (BACK) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = j < 4 ? lo + j : hi + j - 4; // below 8 LPR, for lanes without elements too
            lds[(row * 2) * DP + e] = sq[j];
            lds[(row * 2 + 1) * DP + e] = sk[j];
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

// How many rows share a token's angles: many only where there are rows to fill the card with.  Forward, heads of 64, 4 and 16 rows: 2^19 rows
// 28.3 and 25.4 us, 2^17 9.8 and 11.6, 2^15 5.2 and 9.4.
int heads_of(const grawa_attention_plan *s, int64_t tokens)
{
    const int64_t rows = (int64_t)s->K * tokens * (s->H + s->G);
    return rows >= 1 << 18 ? 16 : 4;
}

template <bool BACK, Pairs P> hipError_t launch_one(const grawa_attention_plan *s, const HeadNorm &a, dim3 grid, hipStream_t st)
{
    if (s->dtype == GRAWA_BF16) {
        if (s->D <= 64)
            hipLaunchKernelGGL((k_head_norm<true, 8, P, BACK>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_head_norm<true, 16, P, BACK>), grid, dim3(256), 0, st, a);
    } else {
        if (s->D <= 64)
            hipLaunchKernelGGL((k_head_norm<false, 8, P, BACK>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_head_norm<false, 16, P, BACK>), grid, dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

template <bool BACK> hipError_t launch(const grawa_attention_plan *s, const HeadNorm &a, int blocks, hipStream_t st)
{
    const dim3 grid((uint32_t)blocks, (uint32_t)s->K);
    if (s->interleaved) return launch_one<BACK, NEIGHBOURS>(s, a, grid, st);
    return s->rotary % 8 ? launch_one<BACK, APART>(s, a, grid, st) : launch_one<BACK, HALVES>(s, a, grid, st);
}

// Squares below 2^-126 lose digits, which shows in sums below 2^-100 to which no larger eps is added.
float least_of(float eps) { return eps < 0x1p-110f ? 0x1p-100f : 0.f; }

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
    a.q = q, a.k = k, a.yq = qo, a.yk = ko, a.wq = qw, a.wk = kw, a.starts = starts, a.turns = s->turns, a.eps = eps, a.least = least_of(eps);
    a.N = (int)N, a.S = (int)S, a.H = s->H, a.G = s->G, a.D = s->D, a.rotary = s->rotary;
    a.heads = heads_of(s, N * S);
    return launch<false>(s, a, (int)blocks_of(s, N * S, a.heads, 1 << 20), st);
}

hipError_t grawa_launch_head_norm_backward(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads dqo, GrawaHeads dko, GrawaHeads q, GrawaHeads k,
                                           GrawaMat qw, GrawaMat kw, float eps, const int *starts, GrawaHeads dq, GrawaHeads dk, GrawaMat dqw,
                                           GrawaMat dkw, int accumulate, hipStream_t st)
{
    HeadNorm a{};
    a.q = q, a.k = k, a.yq = dq, a.yk = dk, a.gq = dqo, a.gk = dko, a.wq = qw, a.wk = kw, a.dwq = dqw, a.dwk = dkw;
    a.starts = starts, a.turns = s->turns, a.part = s->norm_part, a.eps = eps, a.least = least_of(eps), a.accumulate = accumulate;
    a.N = (int)N, a.S = (int)S, a.H = s->H, a.G = s->G, a.D = s->D, a.rotary = s->rotary;
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
