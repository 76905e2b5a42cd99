// Attention of K workers through a window, with first tokens that stay visible and a learned bias by buckets of the distance:
//   s_ij = scale q_i . k_j [+ bias[bucket(p_i - j)]],  o_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij),  lse_i = log sum_j exp(s_ij)
// over the j <= p_i < length with p_i - j < window or j < sinks, p_i = start + i.
// One pass over the keys with the running maximum and sum of the softmax; scores and exponentials stay in registers.
#include "grawa_attend.h"

namespace {

// KEYS = false: a block has 128 CT queries of one head, a wave 32 CT of them, and all waves share a tile of 64 keys.
// KEYS = true, for few queries: a block has up to 32 columns, which are the queries of all heads that share their keys, and its waves
// have 32 keys each of a tile; their sums are joined at the end.
// splits > 1: that many blocks share the keys, and k_attend_join puts their results together.
template <bool BF16, int DP, int CT, bool KEYS, bool BIAS, int NW>
__global__ __launch_bounds__(NW * 64, KEYS ? 1 : 2) void k_attend(GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int BK = KEYS ? 32 * NW : 64, NS = KEYS ? 1 : 2, COLS = KEYS ? 32 : 32 * CT * NW, ES = BF16 ? 2 : 4, KS = DP / 16, DT = DP / 32;
    static_assert(!KEYS || CT == 1, "one set of columns");
    typedef HeadTile<BF16, DP, BK, NW> Tile;
    typedef typename Tile::V V;
    __shared__ __attribute__((aligned(1024))) char lds[4 * Tile::BYTES]; // two buffers of keys and values
    __shared__ float table[BIAS && !KEYS ? GRAWA_MAX_DISTANCES : 1];     // the bias by distance
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int groups = KEYS ? a.G : a.H, per = a.blocks * a.splits;
    const int t = (int)run_of(blockIdx.x, gridDim.x), hd = t / per, rest = t - hd * per, split = rest % a.splits, qb = a.blocks - 1 - rest / a.splits;
    const int kn = hd / groups, k = kn / a.N, n = kn - k * a.N, g = KEYS ? hd - kn * groups : (hd - kn * groups) / a.share;
    const Place at = place_of(a, kn);

    // The lane's columns.
    int head[CT], i[CT], pos[CT];
    bool there[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int col = qb * COLS + (KEYS ? 0 : wave * 32 * CT) + 32 * c + (lane & 31);
        head[c] = KEYS ? g * a.share + col / a.Sq : hd - kn * groups;
        i[c] = KEYS ? col % a.Sq : col;
        there[c] = KEYS ? col < a.share * a.Sq : col < a.Sq;
        pos[c] = at.start + i[c];
    }
    const auto counts = [&](int c) { return there[c] && pos[c] >= 0 && pos[c] < at.length; };
    V q[CT][KS];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const char *row = a.q.p + (int64_t)k * a.q.worker + (int64_t)n * a.q.seq + (int64_t)i[c] * a.q.token + (int64_t)head[c] * a.q.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[c][ks] = load_line<BF16>(row, 16 * ks + 8 * half, a.D, counts(c));
    }
    const float c2 = a.scale * LOG2E;
    const char *bias = BIAS ? a.bias.p + (int64_t)k * a.bias.worker * ES : nullptr;
    float far[CT];
    if constexpr (BIAS) {
#pragma unroll
        for (int c = 0; c < CT; ++c) far[c] = there[c] ? load_one<BF16>(bias + (head[c] * a.buckets + a.bucket_of[a.distances - 1]) * ES) * LOG2E : 0.f;
        if constexpr (!KEYS)
            for (int d = threadIdx.x; d < a.distances; d += NW * 64) table[d] = load_one<BF16>(bias + (head[0] * a.buckets + a.bucket_of[d]) * ES) * LOG2E;
    }

    // Tiles: those with first tokens, then those of the window.
    const int p0 = KEYS ? at.start : at.start + qb * COLS, p1 = KEYS ? at.start + a.Sq - 1 : at.start + min((qb + 1) * COLS, a.Sq) - 1;
    const int w0 = KEYS ? p0 : p0 + wave * 32 * CT, w1 = KEYS ? p1 : w0 + 32 * CT - 1; // of the wave
    const int end = min(p1, at.length - 1) + 1, begin = max(0, max(p0, 0) - a.window + 1);
    const bool any = p1 >= 0 && p0 < at.length;
    const int t0 = begin / BK, first_tiles = any ? min(t0, (min(a.sinks, end) + BK - 1) / BK) : 0, tiles = any ? first_tiles + (end + BK - 1) / BK - t0 : 0;
    const int from = (int)((int64_t)tiles * split / a.splits), to = (int)((int64_t)tiles * (split + 1) / a.splits);
    const char *kp = a.k.p + (int64_t)k * a.k.worker + (int64_t)n * a.k.seq + (int64_t)g * a.k.head;
    const char *vp = a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)g * a.v.head;
    Tile lk, lv;
    lk.init(wave, lane, (uint32_t)a.k.token, a.D);
    lv.init(wave, lane, (uint32_t)a.v.token, a.D);
    const auto load = [&](int it, char *buf) {
        const int j0 = (it < first_tiles ? it : it - first_tiles + t0) * BK;
        lk.load(buf, wave, Tile::rsrc(kp + (int64_t)j0 * a.k.token, at.length - j0, (uint32_t)a.k.token, a.D));
        lv.load(buf + Tile::BYTES, wave, Tile::rsrc(vp + (int64_t)j0 * a.v.token, at.length - j0, (uint32_t)a.v.token, a.D));
    };

    grawa_f32x16 o[CT][DT];
    float m[CT], l[CT];
    const auto run = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            m[c] = -__builtin_inff();
            l[c] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[c][d] = grawa_f32x16{};
        }
        if (from < to) load(from, lds);
        for (int it = from; it < to; ++it) {
            char *buf = lds + ((it - from) & 1) * 2 * Tile::BYTES;
            landed();
            if (it + 1 < to) load(it + 1, lds + ((it + 1 - from) & 1) * 2 * Tile::BYTES);
            const int j0 = (it < first_tiles ? it : it - first_tiles + t0) * BK + (KEYS ? wave * 32 : 0), j1 = j0 + 32 * NS - 1;
            if (j0 > w1 || j0 >= at.length || (j1 <= w0 - a.window && j0 >= a.sinks)) continue; // none of the wave's pairs count
            const bool all = j1 <= w0 && (w1 - j0 < a.window || j1 < a.sinks);
            grawa_f32x16 s[CT][NS];
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int u = 0; u < NS; ++u) s[c][u] = grawa_f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int u = 0; u < NS; ++u) {
                    const V f = Tile::by_rows(buf, lane, (KEYS ? wave * 32 : 0) + 32 * u, ks);
#pragma unroll
                    for (int c = 0; c < CT; ++c) s[c][u] = mfma(f, q[c][ks], s[c][u]);
                }
            if constexpr (BIAS) {
                const bool is_far = w0 - j1 >= a.distances - 1;
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int u = 0; u < NS; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            float b = far[c];
                            if (!is_far) {
                                const int d = clamp_int(pos[c] - (j0 + 32 * u + (r & 3) + 8 * (r >> 2) + 4 * half), 0, a.distances - 1);
                                b = !KEYS ? table[d] : there[c] ? load_one<BF16>(bias + (head[c] * a.buckets + a.bucket_of[d]) * ES) * LOG2E : 0.f;
                            }
                            s[c][u][r] = s[c][u][r] * c2 + b;
                        }
            }
            if (!all) {
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int u = 0; u < NS; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int j = j0 + 32 * u + (r & 3) + 8 * (r >> 2) + 4 * half, d = pos[c] - j;
                            const bool seen = d >= 0 && (d < a.window || j < a.sinks);
                            s[c][u][r] = seen ? s[c][u][r] : -__builtin_inff();
                        }
            }
            V p[CT][NS][2];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                float top = s[c][0][0];
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[c][u][r]);
                top = fmaxf(top, other_half(top));
                if (!BIAS) top *= c2;
                // The running maximum moves only where it would grow by more than 2^8: until then the sums are of exponentials up to 2^8.
                if (__any(top > m[c] + 8.f)) {
                    const float m2 = fmaxf(m[c], top), f = m2 == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m[c] - m2);
                    m[c] = m2;
                    l[c] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[c][d] *= f;
                }
                const float base = m[c] == -__builtin_inff() ? 0.f : m[c];
#pragma unroll
                for (int u = 0; u < NS; ++u) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[c][u][r] = __builtin_amdgcn_exp2f(BIAS ? s[c][u][r] - base : __builtin_fmaf(s[c][u][r], c2, -base));
                        l[c] += s[c][u][r];
                    }
                    as_operand(s[c][u], 0, p[c][u][0]);
                    as_operand(s[c][u], 1, p[c][u][1]);
                }
            }
            const char *vt = buf + Tile::BYTES;
            if (careful.value && !all) {
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int c = 0; c < CT; ++c) {
                            V seen;
#pragma unroll
                            for (int r = 0; r < 8; ++r) {
                                const int j = j0 + 32 * u + 16 * h + (r & 3) + 8 * (r >> 2) + 4 * half, d = pos[c] - j;
                                seen[r] = d >= 0 && (d < a.window || j < a.sinks) ? 1.f : 0.f;
                            }
#pragma unroll
                            for (int d = 0; d < DT; ++d)
                                product_of_some(o[c][d], Tile::by_columns(vt, lane, (KEYS ? wave * 32 : 0) + 32 * u + 16 * h, d), p[c][u][h], seen, true);
                        }
            } else {
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const V f = Tile::by_columns(vt, lane, (KEYS ? wave * 32 : 0) + 32 * u + 16 * h, d);
#pragma unroll
                            for (int c = 0; c < CT; ++c) o[c][d] = mfma(f, p[c][u][h], o[c][d]);
                        }
            }
        }
        bool odd = false;
        if (!careful.value)
#pragma unroll
            for (int c = 0; c < CT; ++c)
                if (counts(c))
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) odd |= o[c][d][r] != o[c][d][r];
        return __syncthreads_or(odd); // every wave is behind its last read of a tile
    };
    // Where that left something that is no number it may come from a token that the column does not see: once more, with care.
    if (__builtin_expect(run(Is<false>()), 0)) run(Is<true>());
#pragma unroll
    for (int c = 0; c < CT; ++c) l[c] += other_half(l[c]);

    const int64_t rows = (int64_t)a.K * a.N * a.H * a.Sq;
    float *part = a.part + (int64_t)split * rows * DP, *part_lse = a.part + (int64_t)a.splits * rows * DP + (int64_t)split * rows;
    if constexpr (!KEYS) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            if (!there[c]) continue;
            const float lse2 = counts(c) && !(l[c] == 0.f) ? m[c] + __builtin_amdgcn_logf(l[c]) : -__builtin_inff();
            const float f = counts(c) && !(l[c] == 0.f) ? 1.f / l[c] : 0.f;
            const int64_t row = ((int64_t)kn * a.H + head[c]) * a.Sq + i[c];
            if (!counts(c))
#pragma unroll
                for (int d = 0; d < DT; ++d) o[c][d] = grawa_f32x16{};
            if (a.splits > 1) {
#pragma unroll
                for (int d = 0; d < DT; ++d) store_column<false>((char *)(part + row * DP), lane, d, DP, o[c][d], f);
                if (half == 0) part_lse[row] = lse2;
                continue;
            }
            char *out = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)i[c] * a.o.token + (int64_t)head[c] * a.o.head;
#pragma unroll
            for (int d = 0; d < DT; ++d) store_column<BF16>(out, lane, d, a.D, o[c][d], f);
            if (a.lse && half == 0) a.lse[row] = lse2 * LN2;
        }
    } else {
        constexpr int PITCH = DP + 4;
        float *sums = (float *)lds, *ml = sums + NW * 32 * PITCH; // every wave is behind its last read of a tile
        static_assert((NW * 32 * PITCH + NW * 64) * 4 <= 4 * Tile::BYTES, "room for the waves' sums");
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(grawa_f32x4v *)(sums + (wave * 32 + (lane & 31)) * PITCH + 32 * d + 8 * r + 4 * half) =
                    grawa_f32x4v{o[0][d][4 * r], o[0][d][4 * r + 1], o[0][d][4 * r + 2], o[0][d][4 * r + 3]};
        if (half == 0) ml[wave * 64 + lane] = m[0], ml[wave * 64 + 32 + lane] = l[0];
        __syncthreads();
        constexpr int LPC = NW * 2, EPL = DP / LPC; // threads of a column, elements of each
        const int cl = threadIdx.x / LPC, e0 = threadIdx.x % LPC * EPL, col = qb * 32 + cl;
        if (col < a.share * a.Sq) {
            const int h = g * a.share + col / a.Sq, ii = col % a.Sq, p = at.start + ii;
            float top = -__builtin_inff(), total = 0.f, v[EPL];
            for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[w * 64 + cl]);
#pragma unroll
            for (int e = 0; e < EPL; ++e) v[e] = 0.f;
            for (int w = 0; w < NW; ++w) {
                const float mw = ml[w * 64 + cl], f = mw == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mw - top);
                if (f == 0.f && ml[w * 64 + 32 + cl] == 0.f) continue;
                total += ml[w * 64 + 32 + cl] * f;
#pragma unroll
                for (int e = 0; e < EPL; ++e) v[e] += sums[(w * 32 + cl) * PITCH + e0 + e] * f;
            }
            const bool row_counts = p >= 0 && p < at.length && !(total == 0.f);
            const float f = row_counts ? 1.f / total : 0.f, lse2 = row_counts ? top + __builtin_amdgcn_logf(total) : -__builtin_inff();
            const int64_t row = ((int64_t)kn * a.H + h) * a.Sq + ii;
            char *out = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)ii * a.o.token + (int64_t)h * a.o.head;
#pragma unroll
            for (int e = 0; e < EPL; ++e) v[e] = row_counts ? v[e] * f : 0.f;
            if (a.splits > 1) {
#pragma unroll
                for (int e = 0; e < EPL; e += 4) *(grawa_f32x4v *)(part + row * DP + e0 + e) = grawa_f32x4v{v[e], v[e + 1], v[e + 2], v[e + 3]};
                if (e0 == 0) part_lse[row] = lse2;
            } else {
                constexpr int PN = GrawaPiece<BF16>::N;
#pragma unroll
                for (int e = 0; e < EPL; e += PN)
                    if (e0 + e < a.D) store_piece<BF16>(out + (e0 + e) * ES, PN, v + e);
                if (a.lse && e0 == 0) a.lse[row] = lse2 * LN2;
            }
        }
    }
#endif
}

// o = sum over the splits of o_s exp(lse_s - lse): a wave has 64 / (DP / 8) rows.
template <bool BF16, int DP> __global__ __launch_bounds__(256) void k_attend_join(GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = DP / 8, ES = BF16 ? 2 : 4, PN = GrawaPiece<BF16>::N;
    const int64_t rows = (int64_t)a.K * a.N * a.H * a.Sq, row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int e0 = threadIdx.x % LPR * 8;
    if (row >= rows) return;
    const float *lse = a.part + (int64_t)a.splits * rows * DP + row;
    float top = -__builtin_inff();
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, lse[s * rows]);
    float total = 0.f, v[8] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float ls = lse[s * rows];
        if (ls == -__builtin_inff()) continue;
        const float f = __builtin_amdgcn_exp2f(ls - top);
        total += f;
        const grawa_f32x4v *p = (const grawa_f32x4v *)(a.part + ((int64_t)s * rows + row) * DP + e0);
        const grawa_f32x4v x = p[0], y = p[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += x[j] * f, v[4 + j] += y[j] * f;
    }
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
    if (a.lse && e0 == 0) a.lse[row] = any ? (top + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
#endif
}

constexpr int KEYS_COLUMNS = 64; // up to this many columns of a group of heads the waves of a block have keys of their own

// How many blocks share the keys: enough to give the card 512, no more than there are tiles to share or room for their results.
int splits_of(int64_t blocks, int64_t rows, int DP, int64_t tiles, int64_t part_floats)
{
    int64_t s = blocks >= 384 ? 1 : 512 / blocks;
    if (s > tiles / 2) s = tiles / 2;
    const int64_t room = part_floats / (rows * (DP + 1));
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
        a.splits = splits_of(kn * a.G * a.blocks, rows, DP, (seen + 32 * KW - 1) / (32 * KW), part_floats);
        hipLaunchKernelGGL((k_attend<BF16, DP, 1, true, BIAS, KW>), dim3((uint32_t)(kn * a.G * a.blocks * a.splits)), dim3(KW * 64), 0, st, a);
    } else {
        const bool wide = BF16 && kn * a.H * ((a.Sq + 255) / 256) >= 512;
        a.blocks = wide ? (a.Sq + 255) / 256 : (a.Sq + 127) / 128;
        a.splits = splits_of(kn * a.H * a.blocks, rows, DP, (seen + 63) / 64, part_floats);
        const dim3 grid((uint32_t)(kn * a.H * a.blocks * a.splits));
        if (BF16 && wide)
            hipLaunchKernelGGL((k_attend<BF16, DP, BF16 ? 2 : 1, false, BIAS, 4>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_attend<BF16, DP, 1, false, BIAS, 4>), grid, dim3(256), 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    hipLaunchKernelGGL((k_attend_join<BF16, DP>), dim3((uint32_t)((rows * (DP / 8) + 255) / 256)), dim3(256), 0, st, a);
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
