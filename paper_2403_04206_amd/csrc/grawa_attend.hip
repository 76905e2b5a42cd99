// Attention of K workers through a window, with first tokens that stay visible and a learned bias by buckets of the distance:
//   s_ij = scale q_i . k_j [+ bias[bucket(p_i - j)]],  o_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij),  lse_i = log sum_j exp(s_ij)
// over the j <= p_i < length with p_i - j < window or j < sinks, p_i = start + i.
// One pass over the keys with the running maximum and sum of the softmax; scores and exponentials stay in registers.
#include "grawa_attend.h"

namespace {

#ifdef __HIP_DEVICE_COMPILE__
// The running maximum and sum of a column's softmax: m in units of the scores, of which c is in units of log2.
struct Running {
    float m, l;
    __device__ __forceinline__ float top(float c) const { return m == -__builtin_inff() ? 0.f : m * c; }
    // A sum of the column's exponentials as one of exp2(score c - m c), of which top(c) is a rounding: what the sums of several waves or blocks
    // are joined by.  Logarithms of the sums would not do: beside a large maximum float32 has no digits for them.
    __device__ __forceinline__ float joined(float sum, float c) const
    {
        const float t = top(c);
        return m == -__builtin_inff() || fabsf(t) > LARGE ? sum : sum * __builtin_amdgcn_exp2f(-__builtin_fmaf(m, c, -t));
    }
};

// exp2 of 16 scores times c against the maximum.
__device__ __forceinline__ void exponentials(grawa_f32x16 &s, float c, const Running &run)
{
    const float top = run.top(c);
    if (__builtin_expect(__any(fabsf(top) > LARGE), 0)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fabsf(top) > LARGE ? (s[r] - run.m) * c : __builtin_fmaf(s[r], c, -top));
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -top));
    }
}

// Exponentials of a column's scores times c against its running maximum, as operands, and their sum, taken before they are rounded (the
// gradients start from it).
// The maximum need not be a tile's: the sums hold exponentials above 1 as well.  It is looked for where a column has none yet or where a
// lane's exponentials add up to more than 2^13 (or to infinity); other tiles need neither the maximum nor what the other half of the
// wave has.
template <int NS, int DT, class V>
__device__ __forceinline__ void soften(const grawa_f32x16 (&s)[NS], float c, Running &run, grawa_f32x16 (&o)[DT], V (&p)[2 * NS])
{
    float sums[2] = {0.f, 0.f};
    const float top0 = run.top(c);
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            grawa_f32x16 e;
#pragma unroll
            for (int r = 8 * h; r < 8 * h + 8; ++r) {
                e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][r], c, -top0));
                sums[r % 2] += e[r];
            }
            as_operand(e, h, p[2 * u + h]);
        }
    float sum = sums[0] + sums[1];
    if (__any(sum > 8192.f || run.m == -__builtin_inff() || fabsf(top0) > LARGE)) {
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
        top = fmaxf(top, other_half(top));
        const float m2 = fmaxf(run.m, top), f = m2 == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((run.m - m2) * c);
        run.m = m2;
        run.l *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
        sum = 0.f;
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            grawa_f32x16 e = s[u];
            exponentials(e, c, run);
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += e[r];
            as_operand(e, 0, p[2 * u]);
            as_operand(e, 1, p[2 * u + 1]);
        }
    }
    run.l += sum;
}
#endif

// A block has 128 queries of one head, a wave 32 of them, and all waves share tiles of 64 keys and values, two in LDS.
// splits > 1: that many blocks share the keys, and k_attend_join puts their results together.
// Scores are formed transposed, a lane holding one query's, so that what one product leaves in a lane's registers is what the next takes.
// Heads of 64 are bound by the vector unit: an exponential, a product-sum, a sum and half a conversion a score, 64 % of the time, matrix
// cores 38 %; 8 workers, 16 heads of 2048 tokens, bf16: 92 us, 750 TFLOP/s of the pairs that count.  Heads of 128 wait for both in turn
// (55 and 45 %): 32 heads of 16384 tokens, window 4096, 917 us, 1050 TFLOP/s.  float32 is bound by its matrix instructions, 50 % busy:
// 72 us for 4 workers' 3 ragged sequences of 600.  64 queries a wave, halving what LDS delivers: 2 waves a SIMD less, and slower.
template <bool BF16, int DP, bool BIAS>
__global__ __launch_bounds__(256, BF16 && DP == 64 ? 3 : BF16 || DP == 64 ? 2 : 1) void k_attend([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int BK = 64, ES = BF16 ? 2 : 4, KS = DP / 16, DT = DP / 32;
    typedef HeadTile<BF16, DP, BK, 4> Tile;
    typedef typename Tile::V V;
    __shared__ __attribute__((aligned(1024))) char buf0[2 * Tile::BYTES], buf1[2 * Tile::BYTES]; // keys and values
    __shared__ float table[BIAS ? GRAWA_MAX_DISTANCES : 1];              // the bias by distance
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int heads = a.K * a.N * a.H;
    const Turn turn = turn_of(blockIdx.x, a.K * a.N * a.G, a.share, a.by_xcd);
    if (turn.head >= heads) return;
    const int qb = a.blocks - 1 - turn.block / a.splits, split = turn.block % a.splits;
    const int kn = turn.head / a.H, head = turn.head - kn * a.H, k = kn / a.N, n = kn - k * a.N, g = head / a.share;
    const Place at = place_of(a, kn);

    // The lane's column.
    const int i = qb * 128 + wave * 32 + (lane & 31), pos = at.start + i;
    const bool there = i < a.Sq, counts = there && pos >= 0 && pos < at.length;
    V q[KS];
    {
        const char *row = a.q.p + (int64_t)k * a.q.worker + (int64_t)n * a.q.seq + (int64_t)i * a.q.token + (int64_t)head * a.q.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = load_line<BF16>(row, 16 * ks + 8 * half, a.D, counts);
    }
    const float c2 = a.scale * LOG2E, unit = BIAS ? 1.f : c2; // of a score as it comes, and with its bias
    float far = 0.f;
    if constexpr (BIAS) {
        const char *bias = a.bias.p + ((int64_t)k * a.bias.worker + head * a.buckets) * ES;
        far = bias_of<BF16>(bias + a.bucket_of[a.distances - 1] * ES);
        for (int d = threadIdx.x; d < a.distances; d += 256) table[d] = bias_of<BF16>(bias + a.bucket_of[d] * ES);
    }

    // Tiles: those with first tokens, then those of the window.
    const int p0 = at.start + qb * 128, p1 = at.start + min((qb + 1) * 128, a.Sq) - 1, w0 = p0 + wave * 32, w1 = w0 + 31;
    const int end = min(p1, at.length - 1) + 1, begin = max(0, max(p0, 0) - a.window + 1);
    const bool any = p1 >= 0 && p0 < at.length;
    const int t0 = begin / BK, first_tiles = any ? min(t0, (min(a.sinks, end) + BK - 1) / BK) : 0, tiles = any ? first_tiles + (end + BK - 1) / BK - t0 : 0;
    const int from = (int)((int64_t)tiles * split / a.splits), to = (int)((int64_t)tiles * (split + 1) / a.splits);
    const char *kp = a.k.p + (int64_t)k * a.k.worker + (int64_t)n * a.k.seq + (int64_t)g * a.k.head;
    const char *vp = a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)g * a.v.head;
    Tile lk, lv;
    lk.init(wave, lane, (uint32_t)a.k.token, a.D);
    lv.init(wave, lane, (uint32_t)a.v.token, a.D);
    const auto tile_of = [&](int it) { return (it < first_tiles ? it : it - first_tiles + t0) * BK; };
    Tiles<Tile, BK> tiles_at;
    const auto restart = [&]() __attribute__((always_inline)) { tiles_at.init(kp, vp, (uint32_t)a.k.token, (uint32_t)a.v.token, at.length, a.D, from, first_tiles, t0); };
    const auto load = [&](char *buf) __attribute__((always_inline)) { tiles_at.load(lk, lv, buf, wave); };
    restart();
    const auto none = [&](int j0, int j1) { return j0 > w1 || j0 >= at.length || (j1 <= w0 - a.window && j0 >= a.sinks); }; // of the wave's pairs count
    const auto all = [&](int j0, int j1) { return j1 <= w0 && (w1 - j0 < a.window || j1 < a.sinks); };
    // Scores of 32 keys: masked, with a bias in units of log2.
    const auto scores = [&](int j0, grawa_f32x16 &s) __attribute__((always_inline)) {
        if constexpr (BIAS) {
            if (w0 - (j0 + 31) >= a.distances - 1) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], c2, far);
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = __builtin_fmaf(s[r], c2, table[clamp_int(pos - (j0 + (r & 3) + 8 * (r >> 2) + 4 * half), 0, a.distances - 1)]);
            }
        }
        if (!all(j0, j0 + 31))
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? s[r] : -__builtin_inff();
    };

    grawa_f32x16 o[DT];
    Running run{-__builtin_inff(), 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = grawa_f32x16{};
    const uint32_t rows_at = Tile::rows_of(lane), columns_at = Tile::columns_of(lane);
    // 64 keys, or with float32, whose products are long, each half of them by itself where the wave sees any of it.
    const auto step = [&](int it, const char *buf) __attribute__((always_inline)) {
        constexpr int NS = BF16 ? 2 : 1, A = BF16 ? 4 : 2;
#pragma unroll
        for (int part = 0; part < 2 / NS; ++part) {
            const int j0 = tile_of(it) + 32 * part;
            if (none(j0, j0 + 32 * NS - 1)) continue;
            V f[A], p[2 * NS];
            const auto key = [&](int i) { return Tile::by_rows(buf + 32 * part * Tile::RB, rows_at, i % NS * 32, i / NS); };
            const auto value = [&](int i) { return Tile::by_columns(buf + Tile::BYTES + 32 * part * Tile::RB, columns_at, i / DT * 16, i % DT); };
            grawa_f32x16 s[NS] = {};
            ask(f, key);
            flow<NS * KS>(f, key, [&](int i, const V &x) __attribute__((always_inline)) { s[i % NS] = mfma(x, q[i / NS], s[i % NS]); });
            ask(f, value);
#pragma unroll
            for (int u = 0; u < NS; ++u) scores(j0 + 32 * u, s[u]);
            soften(s, unit, run, o, p);
            __builtin_amdgcn_sched_barrier(0);
            flow<2 * NS * DT>(f, value, [&](int i, const V &x) __attribute__((always_inline)) { o[i % DT] = mfma(x, p[i / DT], o[i % DT]); });
        }
    };
    if (from < to) load(buf0);
    for (int it = from; it < to; it += 2) {
        landed();
        if (it + 1 < to) load(buf1);
        step(it, buf0);
        if (it + 1 == to) break;
        landed();
        if (it + 2 < to) load(buf0);
        step(it + 1, buf1);
    }

    const int64_t rows = (int64_t)a.K * a.N * a.H * a.Sq, row = ((int64_t)kn * a.H + head) * a.Sq + i;
    float *part = a.part + ((int64_t)split * rows + row) * DP;
    char *out = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)i * a.o.token + (int64_t)head * a.o.head;
    const float l = run.l + other_half(run.l);
    const bool sum = counts && !(l == 0.f);
    const float f = sum ? 1.f / l : 0.f;
    if (half == 0 && there) {
        if (a.splits > 1) {
            float *const at_row = a.part + (int64_t)a.splits * rows * DP + (int64_t)split * rows + row;
            at_row[0] = run.m;
            at_row[(int64_t)a.splits * rows] = sum ? run.joined(l, unit) : 0.f;
        } else if (a.lse) {
            a.lse[row] = sum ? (run.top(unit) + __builtin_amdgcn_logf(l)) * LN2 : -__builtin_inff();
        }
    }
    const auto put = [&](int d, const grawa_f32x16 &sums) {
        if (!there) return;
        grawa_f32x16 v;
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = sum ? sums[r] * f : 0.f;
        if (a.splits > 1)
            store_column<false>((char *)part, lane, d, DP, v, 1.f);
        else
            store_column<BF16>(out, lane, d, a.D, v, 1.f);
    };
    bool odd = false;
    if (sum)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) odd |= o[d][r] != o[d][r];
    // What is no number may come from a token that the column does not see: once more then, with care.
    if (__builtin_expect(!__syncthreads_or(odd), 1)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) put(d, o[d]);
        return;
    }
#pragma unroll 1
    for (int d = 0; d < DT; ++d) {
        grawa_f32x16 sums = {};
        restart();
#pragma unroll 1
        for (int it = from; it < to; ++it) {
            landed();
            load(buf0);
            landed();
#pragma unroll 1
            for (int u = 0; u < 2; ++u) {
                const int j0 = tile_of(it) + 32 * u, j1 = j0 + 31;
                if (none(j0, j1)) continue;
                grawa_f32x16 s = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s = mfma(Tile::by_rows(buf0 + 32 * u * Tile::RB, rows_at, 0, ks), q[ks], s);
                scores(j0, s);
                exponentials(s, unit, run);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    V p;
                    as_operand(s, h, p);
                    const V v = Tile::by_columns(buf0 + Tile::BYTES + (32 * u + 16 * h) * Tile::RB, columns_at, 0, d);
                    if (all(j0, j1))
                        sums = mfma(v, p, sums);
                    else
                        product_of_some(sums, v, p, marks<V>(a, pos, j0 + 16 * h, half));
                }
            }
        }
        put(d, sums);
    }
#endif
}

// The same for few queries: a block has up to 32 columns, which are the queries of all heads that share their keys, and its NW waves
// have 32 keys each of a tile; their sums are joined at the end.  Bound by reading the cache: a token of 32 sequences over up to 16384 keys,
// window 8192, 8 groups of 4 heads of 128: 169 us, 880 MB, 5.2 TB/s; 4 x 16 heads of 64 over 2048 9 us, half of it a launch's.
template <bool BF16, int DP, bool BIAS, int NW>
__global__ __launch_bounds__(NW * 64) void k_attend_few([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int BK = 32 * NW, ES = BF16 ? 2 : 4, KS = DP / 16, DT = DP / 32;
    typedef HeadTile<BF16, DP, BK, NW> Tile;
    typedef typename Tile::V V;
    __shared__ __attribute__((aligned(1024))) char buf0[2 * Tile::BYTES], buf1[2 * Tile::BYTES]; // keys and values
    constexpr int PITCH = DP + 4;
    __shared__ float ml[NW * 64]; // of each wave, joined at the end
    static_assert(NW / 2 * 32 * PITCH * 4 <= 2 * Tile::BYTES, "room for half the waves' sums in a buffer");
    const auto sums_of = [&](int w, int column) { return (float *)(w < NW / 2 ? buf0 : buf1) + (w % (NW / 2) * 32 + column) * PITCH; };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int groups = a.K * a.N * a.G;
    const Turn turn = turn_of(blockIdx.x, groups, 1, a.by_xcd);
    if (turn.head >= groups) return;
    const int cb = turn.block / a.splits, split = turn.block % a.splits;
    const int kn = turn.head / a.G, g = turn.head - kn * a.G, k = kn / a.N, n = kn - k * a.N;
    const Place at = place_of(a, kn);

    // The lane's column.
    const int col = cb * 32 + (lane & 31), head = g * a.share + col / a.Sq, i = col % a.Sq, pos = at.start + i;
    const bool there = col < a.share * a.Sq, counts = there && pos >= 0 && pos < at.length;
    V q[KS];
    {
        const char *row = a.q.p + (int64_t)k * a.q.worker + (int64_t)n * a.q.seq + (int64_t)i * a.q.token + (int64_t)head * a.q.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = load_line<BF16>(row, 16 * ks + 8 * half, a.D, counts);
    }
    const float c2 = a.scale * LOG2E, unit = BIAS ? 1.f : c2; // of a score as it comes, and with its bias
    const char *bias = BIAS ? a.bias.p + ((int64_t)k * a.bias.worker + (there ? head : 0) * a.buckets) * ES : nullptr;
    float far = 0.f;
    if constexpr (BIAS) far = bias_of<BF16>(bias + a.bucket_of[a.distances - 1] * ES);

    const int w0 = at.start, w1 = at.start + a.Sq - 1; // positions
    const int end = min(w1, at.length - 1) + 1, begin = max(0, max(w0, 0) - a.window + 1);
    const bool any = w1 >= 0 && w0 < at.length;
    const int t0 = begin / BK, first_tiles = any ? min(t0, (min(a.sinks, end) + BK - 1) / BK) : 0, tiles = any ? first_tiles + (end + BK - 1) / BK - t0 : 0;
    const int from = (int)((int64_t)tiles * split / a.splits), to = (int)((int64_t)tiles * (split + 1) / a.splits);
    const char *kp = a.k.p + (int64_t)k * a.k.worker + (int64_t)n * a.k.seq + (int64_t)g * a.k.head;
    const char *vp = a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)g * a.v.head;
    Tile lk, lv;
    lk.init(wave, lane, (uint32_t)a.k.token, a.D);
    lv.init(wave, lane, (uint32_t)a.v.token, a.D);
    const auto tile_of = [&](int it) { return (it < first_tiles ? it : it - first_tiles + t0) * BK; };
    Tiles<Tile, BK> tiles_at;
    const auto load = [&](char *buf) __attribute__((always_inline)) { tiles_at.load(lk, lv, buf, wave); };

    grawa_f32x16 o[DT];
    Running run;
    const uint32_t rows_at = Tile::rows_of(lane) + wave * 32 * Tile::RB, columns_at = Tile::columns_of(lane) + wave * 32 * Tile::RB;
    const auto go = [&](auto careful) __attribute__((always_inline)) {
        run = Running{-__builtin_inff(), 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = grawa_f32x16{};
        const auto step = [&](int it, const char *buf) __attribute__((always_inline)) {
            const int j0 = tile_of(it) + wave * 32, j1 = j0 + 31;
            if (j0 > w1 || j0 >= at.length || (j1 <= w0 - a.window && j0 >= a.sinks)) return; // none of the wave's pairs count
            const bool all = j1 <= w0 && (w1 - j0 < a.window || j1 < a.sinks);
            grawa_f32x16 s[1] = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s[0] = mfma(Tile::by_rows(buf, rows_at, 0, ks), q[ks], s[0]);
            if constexpr (BIAS) {
                if (w0 - j1 >= a.distances - 1) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[0][r] = s[0][r] * c2 + far;
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int d = clamp_int(pos - (j0 + (r & 3) + 8 * (r >> 2) + 4 * half), 0, a.distances - 1);
                        s[0][r] = s[0][r] * c2 + bias_of<BF16>(bias + a.bucket_of[d] * ES);
                    }
                }
            }
            if (!all)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? s[0][r] : -__builtin_inff();
            V p[2];
            soften(s, unit, run, o, p);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const V v = Tile::by_columns(buf + Tile::BYTES, columns_at, 16 * h, d);
                    if (careful.value && !all)
                        product_of_some(o[d], v, p[h], marks<V>(a, pos, j0 + 16 * h, half));
                    else
                        o[d] = mfma(v, p[h], o[d]);
                }
        };
        tiles_at.init(kp, vp, (uint32_t)a.k.token, (uint32_t)a.v.token, at.length, a.D, from, first_tiles, t0);
        if (from < to) load(buf0);
        for (int it = from; it < to; it += 2) {
            landed();
            if (it + 1 < to) load(buf1);
            step(it, buf0);
            if (it + 1 == to) break;
            landed();
            if (it + 2 < to) load(buf0);
            step(it + 1, buf1);
        }
        bool odd = false;
        if (!careful.value && counts)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) odd |= o[d][r] != o[d][r];
        return __syncthreads_or(odd); // every wave is behind its last read of a tile
    };
    // What is no number may come from a token that the column does not see: once more then, with care.
    if (__builtin_expect(go(Is<false>()), 0)) go(Is<true>());

    const float l = run.l + other_half(run.l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *(grawa_f32x4v *)(sums_of(wave, lane & 31) + 32 * d + 8 * r + 4 * half) = grawa_f32x4v{o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]};
    if (half == 0) ml[wave * 64 + lane] = run.m, ml[wave * 64 + 32 + lane] = l;
    __syncthreads();
    constexpr int LPC = NW * 2, EPL = DP / LPC; // threads of a column, elements of each
    const int cl = threadIdx.x / LPC, e0 = threadIdx.x % LPC * EPL, c = cb * 32 + cl;
    if (c >= a.share * a.Sq) return;
    const int h = g * a.share + c / a.Sq, ii = c % a.Sq, p = at.start + ii;
    float top = -__builtin_inff(), total = 0.f, v[EPL];
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[w * 64 + cl]);
#pragma unroll
    for (int e = 0; e < EPL; ++e) v[e] = 0.f;
    for (int w = 0; w < NW; ++w) {
        const float mw = ml[w * 64 + cl], lw = ml[w * 64 + 32 + cl];
        if (lw == 0.f) continue;
        const float f = Running{mw, 0.f}.joined(__builtin_amdgcn_exp2f((mw - top) * unit), unit);
        total += lw * f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) v[e] += sums_of(w, cl)[e0 + e] * f;
    }
    const bool sum = p >= 0 && p < at.length && !(total == 0.f);
    const float f = sum ? 1.f / total : 0.f;
    const int64_t rows = (int64_t)a.K * a.N * a.H * a.Sq, row = ((int64_t)kn * a.H + h) * a.Sq + ii;
#pragma unroll
    for (int e = 0; e < EPL; ++e) v[e] = sum ? v[e] * f : 0.f;
    if (a.splits > 1) {
        float *part = a.part + ((int64_t)split * rows + row) * DP + e0;
#pragma unroll
        for (int e = 0; e < EPL; e += 4) *(grawa_f32x4v *)(part + e) = grawa_f32x4v{v[e], v[e + 1], v[e + 2], v[e + 3]};
        if (e0 == 0) {
            float *const at_row = a.part + (int64_t)a.splits * rows * DP + (int64_t)split * rows + row;
            at_row[0] = top;
            at_row[(int64_t)a.splits * rows] = sum ? total : 0.f;
        }
        return;
    }
    char *out = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)ii * a.o.token + (int64_t)h * a.o.head;
    constexpr int PN = GrawaPiece<BF16>::N;
#pragma unroll
    for (int e = 0; e < EPL; e += PN)
        if (e0 + e < a.D) store_piece<BF16>(out + (e0 + e) * ES, PN, v + e);
    if (a.lse && e0 == 0) a.lse[row] = sum ? (top * unit + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
#endif
}

// o = sum over the splits of o_s l_s exp2((m_s - m) unit) / l, of the splits' maxima and sums: eight elements a lane, eight splits asked for
// before the first is used.  NW = 4: each of a block's waves has every fourth split of its rows, and the waves' sums are joined in order.
template <bool BF16, int DP, int NW> __global__ __launch_bounds__(256) void k_attend_join([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = DP / 8, ES = BF16 ? 2 : 4, PN = GrawaPiece<BF16>::N, U = 8, THREADS = 256 / NW;
    __shared__ float tops[NW][THREADS], totals[NW][THREADS], sums[NW][8][NW == 1 ? 1 : THREADS];
    const int lane = threadIdx.x % THREADS, wave = threadIdx.x / THREADS, e0 = lane % LPR * 8;
    const int64_t rows = (int64_t)a.K * a.N * a.H * a.Sq, own = (int64_t)blockIdx.x * (THREADS / LPR) + lane / LPR, row = own < rows ? own : rows - 1;
    const float *tops_at = a.part + (int64_t)a.splits * rows * DP + row, *sums_at = tops_at + (int64_t)a.splits * rows, *part = a.part + row * DP + e0;
    const float unit = a.buckets ? 1.f : a.scale * LOG2E;
    float top = -__builtin_inff(), total = 0.f, v[8] = {};
    for (int s0 = wave; s0 < a.splits; s0 += NW * U) {
        float m[U], l[U];
        grawa_f32x4v x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + NW * u < a.splits ? s0 + NW * u : s0; // what is read twice is left out below
            m[u] = tops_at[s * rows];
            l[u] = sums_at[s * rows];
            x[u] = *(const grawa_f32x4v *)(part + (int64_t)s * rows * DP);
            y[u] = *(const grawa_f32x4v *)(part + (int64_t)s * rows * DP + 4);
        }
        float m2 = top;
#pragma unroll
        for (int u = 0; u < U; ++u) m2 = fmaxf(m2, m[u]);
        const float base = m2 == -__builtin_inff() ? 0.f : m2, before = __builtin_amdgcn_exp2f((top - base) * unit);
        top = m2;
        total *= before;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= before;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + NW * u >= a.splits || l[u] == 0.f) continue; // sums that are no numbers pass
            const float f = l[u] * __builtin_amdgcn_exp2f((m[u] - base) * unit);
            total += f;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += x[u][j] * f, v[4 + j] += y[u][j] * f;
        }
    }
    if constexpr (NW > 1) {
        tops[wave][lane] = top;
        totals[wave][lane] = total;
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[wave][j][lane] = v[j];
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, tops[w][lane]);
        const float base = top == -__builtin_inff() ? 0.f : top;
        total = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f((tops[w][lane] - base) * unit);
            total += totals[w][lane] * f;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += sums[w][j][lane] * f;
        }
    }
    if (own >= rows) return;
    const bool any = !(total == 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = any ? v[j] / total : 0.f;
    const int i = (int)(row % a.Sq);
    const int64_t knh = row / a.Sq;
    const int h = (int)(knh % a.H), kn = (int)(knh / a.H), k = kn / a.N, n = kn - k * a.N;
    char *out = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)i * a.o.token + (int64_t)h * a.o.head;
#pragma unroll
    for (int j = 0; j < 8; j += PN)
        if (e0 + j < a.D) store_piece<BF16>(out + (e0 + j) * ES, PN, v + j);
    if (a.lse && e0 == 0) a.lse[row] = any ? (top * unit + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
#endif
}

// Up to so many columns of a group of heads the waves of a block have keys of their own.  4 sequences over 4096 keys, by keys and by queries:
// bf16, 16 heads of 64, 64 columns 22 and 24 us, 96 columns 35 and 25; 8 groups of 4 heads of 128, 64 columns 25 and 45, 128 columns 66 and 45;
// float32, 32 columns of 64 36 and 78, 96 columns 103 and 77.
constexpr int KEYS_COLUMNS = 64;

// How many blocks share the keys: enough to give the card `target`, no more than there are tiles to share or room for their results.
int splits_of(int64_t target, int64_t blocks, int64_t rows, int DP, int64_t tiles, int64_t part_floats)
{
    int64_t s = blocks >= target * 3 / 4 ? 1 : target / blocks;
    if (s > tiles / 2) s = tiles / 2;
    const int64_t room = part_floats / (rows * (DP + 2)); // a row's result, maximum and sum
    if (s > room) s = room;
    return s < 1 ? 1 : (int)s;
}

template <bool BF16, int DP, bool BIAS> hipError_t launch(GrawaAttend a, int64_t part_floats, hipStream_t st)
{
    constexpr int KW = !BF16 && DP == 128 ? 2 : 4;
    const int64_t kn = (int64_t)a.K * a.N, rows = kn * a.H * a.Sq;
    // keys that a query can see, as far as the host knows
    int64_t seen = (int64_t)a.window + a.Sq + a.sinks;
    if (seen > a.Sk) seen = a.Sk;
    if ((int64_t)a.share * a.Sq <= KEYS_COLUMNS) {
        a.blocks = (a.share * a.Sq + 31) / 32;
        // One block a CU, which reads ahead far enough: a token over 16384 keys, 8 groups of 128, 20.3 us and with two blocks 26.8; 16 tokens
        // of 4 heads each over 4096 24.8 and 36.9; 16 x 16 heads of 64 over 4096 46.5 and 49.5; 4 x 16 over 2048 12.1 and 11.7.
        a.splits = splits_of(256, kn * a.G * a.blocks, rows, DP, (seen + 32 * KW - 1) / (32 * KW), part_floats);
        const uint32_t grid = grid_of(kn * a.G, 1, (int64_t)a.blocks * a.splits, a.by_xcd);
        hipLaunchKernelGGL((k_attend_few<BF16, DP, BIAS, KW>), dim3(grid), dim3(KW * 64), 0, st, a);
    } else {
        a.blocks = (a.Sq + 127) / 128;
        // Two blocks a CU: 32 queries of 4 heads each over 4096, 8 groups of 128, 39.3 us and with one 46.2.
        a.splits = splits_of(512, kn * a.H * a.blocks, rows, DP, (seen + 63) / 64, part_floats);
        const uint32_t grid = grid_of(kn * a.G, a.share, (int64_t)a.blocks * a.splits, a.by_xcd);
        hipLaunchKernelGGL((k_attend<BF16, DP, BIAS>), dim3(grid), dim3(256), 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    // Few rows that many blocks shared are all latency: 32 rows of 128 elements, 64 splits, attention and join 34.5 us by lanes, 26.8 by
    // waves; 1024 tokens of 8 heads of 128, two sequences, 4 splits: 28.7 by lanes, 35.2 by waves.
    if (a.splits > 8)
        hipLaunchKernelGGL((k_attend_join<BF16, DP, 4>), dim3((uint32_t)((rows * (DP / 8) + 63) / 64)), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((k_attend_join<BF16, DP, 1>), dim3((uint32_t)((rows * (DP / 8) + 255) / 256)), dim3(256), 0, st, a);
    return hipGetLastError();
}

} // namespace

hipError_t grawa_launch_attend(const grawa_attention_plan *s, GrawaAttend a, hipStream_t st)
{
    if (a.N == 0 || a.Sq == 0) return hipSuccess;
    const bool bias = a.buckets > 0, wide = grawa_padded_width(a.D) == 128;
    if (s->dtype == GRAWA_BF16) {
        if (wide) return bias ? launch<true, 128, true>(a, s->part_floats, st) : launch<true, 128, false>(a, s->part_floats, st);
        return bias ? launch<true, 64, true>(a, s->part_floats, st) : launch<true, 64, false>(a, s->part_floats, st);
    }
    if (wide) return bias ? launch<false, 128, true>(a, s->part_floats, st) : launch<false, 128, false>(a, s->part_floats, st);
    return bias ? launch<false, 64, true>(a, s->part_floats, st) : launch<false, 64, false>(a, s->part_floats, st);
}
