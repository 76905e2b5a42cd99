// Gradients of the attention of grawa_attend.hip:
//   P_ij = exp(s_ij - lse_i), dP = do v^T, delta_i = do_i . o_i = sum_j P_ij dP_ij, dS = P (dP - delta)
//   dq = scale dS k,  dk = scale dS^T q,  dv = P^T do,  dbias[b] = sum of dS over the pairs whose distance is in bucket b
// Two kernels form P and dS tile by tile, one for blocks of queries (dq, dbias, delta), one for blocks of keys (dk and dv of all heads
// that share them): nothing is added up in an order that depends on timing.
#include "grawa_attend.h"

namespace {

// delta is do . o, and o was rounded to bfloat16: off by 2^-9 |do||o| or so, the same for all keys of a row, where each dS is off by its own
// 2^-9.  Over many keys that is little beside them as long as o is small there, values without a mean: dq is off by 0.24 % then, by 0.4 % where
// their mean is their spread, by 2.4 % where it is eight times that, dk by half as much; sums of dS for dbias are put right below.  Over few it is
// what dq and dk are off by most (windows of 32 and 4 first keys: 2.7e-3 against 2.3e-3).  Queries whose block has so few tiles of keys go over them once more before, for delta = sum P dP in float32:
// 2048 tokens without a window, 8 workers of 16 heads of 64: 4 blocks of 16, 130 us and not 122.
constexpr int OWN_DOT_TILES = 8;

// bf16: a block has 128 queries of a head, a wave 32 of them; all waves share tiles of 64 keys and values.  float32, whose products are
// eight times as long: 64 queries, and of the two waves that have the same 32 each has half of a tile's keys; the second's sums go to
// the first through LDS.  2 workers of 3 sequences of 333 tokens, 6 heads of 40, with a bias, 33 us, and 50 with blocks as in bf16; all
// gradients of 4096 tokens, 8 heads of 128, 1107 and 1420, of 4 workers' 16 heads of 2048 tokens of 64 996 and 1015.
// dS is formed transposed, so that it is an operand where it stands.  bf16, 8 workers, 16 heads of 2048 tokens of 64: 125 to 130 us,
// vector unit 50 %, matrix cores 46 %; with a bias of 32 buckets to distance 128: 230, of which the sums by distance are the difference, 35 for
// what delta is off by (with delta formed first in every block 75); 32 heads of 16384 tokens of 128, window 4096: 1230 to 1250, matrix cores 66 %.
template <bool BF16, int DP, bool BIAS>
__global__ __launch_bounds__(256, BF16 || DP == 64 ? 2 : 1) void k_attend_dq([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int BK = 64, ES = BF16 ? 2 : 4, KS = DP / 16, DT = DP / 32, BUFS = BF16 || DP == 64 ? 2 : 1, QW = grawa_dq_queries(BF16) / 32;
    typedef HeadTile<BF16, DP, BK, 4> Tile;
    typedef typename Tile::V V;
    __shared__ __attribute__((aligned(1024))) char buf0[2 * Tile::BYTES], buf1[BUFS == 2 ? 2 * Tile::BYTES : 16]; // keys and values
    __shared__ float diagonals[BIAS ? 4 : 1][BIAS ? 16 * 64 : 1]; // of each wave: dS of 16 keys, a key a row of 64, of which it has 32
    extern __shared__ float tables[];                             // the bias by distance; of each wave: sums of dS by distance; buckets by distance
    float *const table = tables, *const by_distance = tables + (1 + (threadIdx.x >> 6)) * a.distances;
    int *const bucket_of = (int *)(tables + 5 * a.distances);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int qw = wave % QW, kw = wave / QW; // the wave's queries, and its keys where they are not all
    const int heads = a.K * a.N * a.H;
    const Turn turn = turn_of(blockIdx.y * gridDim.x + blockIdx.x, a.K * a.N * a.G, a.share, a.by_xcd);
    if (turn.head >= heads || turn.block >= a.blocks) return;
    const int qb = a.blocks - 1 - turn.block;
    const int kn = turn.head / a.H, head = turn.head - kn * a.H, k = kn / a.N, n = kn - k * a.N, g = head / a.share;
    const Place at = place_of(a, kn);
    const int i = qb * (32 * QW) + qw * 32 + (lane & 31);
    const bool there = i < a.Sq, placed = there && at.start + i >= 0 && at.start + i < at.length;

    V q[KS], go[KS];
    float delta = 0.f;
    {
        const char *pq = a.q.p + (int64_t)k * a.q.worker + (int64_t)n * a.q.seq + (int64_t)i * a.q.token + (int64_t)head * a.q.head;
        const char *pg = a.go.p + (int64_t)k * a.go.worker + (int64_t)n * a.go.seq + (int64_t)i * a.go.token + (int64_t)head * a.go.head;
        const char *po = a.o.p + (int64_t)k * a.o.worker + (int64_t)n * a.o.seq + (int64_t)i * a.o.token + (int64_t)head * a.o.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks] = load_line<BF16>(pq, 16 * ks + 8 * half, a.D, placed);
            go[ks] = load_line<BF16>(pg, 16 * ks + 8 * half, a.D, placed);
            const V o = load_line<BF16>(po, 16 * ks + 8 * half, a.D, placed);
#pragma unroll
            for (int j = 0; j < 8; ++j) delta += (float)o[j] * (float)go[ks][j];
        }
        delta += other_half(delta);
    }
    float lse = placed ? a.lse[((int64_t)kn * a.H + head) * a.Sq + i] * LOG2E : __builtin_inff();
    if (lse == -__builtin_inff()) lse = __builtin_inff(); // the row sees nothing
    // P = exp2(score - lse) is at most 1, but beside a large lse the four roundings on its way here (the maximum's, the sum's, to natural
    // logarithms and back; the constants' product is 0.2 more) could make it any number: one that is 6 of them larger is above all scores.
    if (fabsf(lse) > LARGE) lse = __builtin_fmaf(fabsf(lse), 0x1.8p-22f, lse);
    // Columns that count for nothing stand where they see no key: 0 would not be enough for what they have with one that is no number.
    const bool counts = lse != __builtin_inff();
    const int pos = counts ? at.start + i : -1;
    const bool whole = __all(counts);
    delta = counts ? delta : 0.f;

    const float c2 = a.scale * LOG2E;
    float far = 0.f;
    bool fold = true; // the last distance's bias and lse into one number: not where the bias leaves no digits for the other
    if constexpr (BIAS) {
        const char *bias = a.bias.p + ((int64_t)k * a.bias.worker + head * a.buckets) * ES;
        far = bias_of<BF16>(bias + a.bucket_of[a.distances - 1] * ES);
        fold = __builtin_amdgcn_readfirstlane(!(fabsf(far) > LARGE && fabsf(far) < __builtin_inff()));
        for (int d = threadIdx.x; d < a.distances; d += 256) {
            bucket_of[d] = a.bucket_of[d];
            table[d] = bias_of<BF16>(bias + bucket_of[d] * ES);
        }
        for (int d = lane; d < a.distances; d += 64) by_distance[d] = 0.f;
        for (int d = lane; d < 16 * 64; d += 64) diagonals[wave][d] = 0.f;
    }

    const int p0 = at.start + qb * (32 * QW), p1 = at.start + min((qb + 1) * (32 * QW), a.Sq) - 1, w0 = p0 + qw * 32, w1 = w0 + 31;
    const int end = min(p1, at.length - 1) + 1, begin = max(0, max(p0, 0) - a.window + 1);
    const bool any = p1 >= 0 && p0 < at.length;
    const int t0 = begin / BK, first_tiles = any ? min(t0, (min(a.sinks, end) + BK - 1) / BK) : 0, tiles = any ? first_tiles + (end + BK - 1) / BK - t0 : 0;
    const char *kp = a.k.p + (int64_t)k * a.k.worker + (int64_t)n * a.k.seq + (int64_t)g * a.k.head;
    const char *vp = a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)g * a.v.head;
    Tile lk, lv;
    lk.init(wave, lane, (uint32_t)a.k.token, a.D);
    lv.init(wave, lane, (uint32_t)a.v.token, a.D);
    const auto tile_of = [&](int it) { return (it < first_tiles ? it : it - first_tiles + t0) * BK; };
    Tiles<Tile, BK> tiles_at;
    const auto restart = [&](int from) __attribute__((always_inline)) { tiles_at.init(kp, vp, (uint32_t)a.k.token, (uint32_t)a.v.token, at.length, a.D, from, first_tiles, t0); };
    const auto load = [&](char *buf) __attribute__((always_inline)) { tiles_at.load(lk, lv, buf, wave); };
    const auto none = [&](int j0) { return j0 > w1 || j0 >= at.length || (j0 + 31 <= w0 - a.window && j0 >= a.sinks); }; // of the wave's pairs count
    const auto all = [&](int j0) { return whole && j0 + 31 <= w0 && (w1 - j0 < a.window || j0 + 31 < a.sinks); };
    const uint32_t rows_at = Tile::rows_of(lane), columns_at = Tile::columns_of(lane);
    grawa_f32x16 minus_dot = {};
    constexpr int A = BF16 ? 4 : 2;
    float far_weight = 0.f; // sum of the column's P from the last distance of the table on, as far as it is asked for
    // dS of 32 keys; leaves the first fragments of `then` in f.
    const auto slopes = [&](const char *buf, int u, int j0, V (&f)[A], auto &&then, auto weigh) __attribute__((always_inline)) {
        grawa_f32x16 s = {}, dp = minus_dot;
        const auto both = [&](int i) { return Tile::by_rows(buf + i % 2 * Tile::BYTES, rows_at + 32 * u * Tile::RB, 0, i / 2); };
        ask(f, both);
        flow<2 * KS>(f, both, [&](int i, const V &x) __attribute__((always_inline)) {
            if (i % 2)
                dp = mfma(x, go[i / 2], dp);
            else
                s = mfma(x, q[i / 2], s);
        });
        ask(f, then);
        if (BIAS && (w0 - (j0 + 31) < a.distances - 1 || !fold)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float bias = table[clamp_int(pos - (j0 + (r & 3) + 8 * (r >> 2) + 4 * half), 0, a.distances - 1)];
                s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, bias) - lse) * dp[r]; // the score as the forward pass has it
            }
        } else if constexpr (weigh.value) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, far - lse));
            if (!all(j0))
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? s[r] : 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                far_weight += s[r];
                s[r] *= dp[r];
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, far - lse)) * dp[r];
        }
        if (!all(j0))
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? s[r] : 0.f;
        return s;
    };

    // All of the wave's pairs from a tile on, 32 keys at a time.
    const auto walk = [&](int from, auto &&step) __attribute__((always_inline)) {
        restart(from);
        const auto both_halves = [&](int it, const char *buf) __attribute__((always_inline)) {
            for (int u = BF16 ? 0 : kw; u < (BF16 ? 2 : kw + 1); ++u) {
                const int j0 = tile_of(it) + 32 * u;
                if (!none(j0)) step(buf, u, j0);
            }
        };
        if constexpr (BUFS == 2) {
            if (from < tiles) load(buf0);
            for (int it = from; it < tiles; it += 2) {
                landed();
                if (it + 1 < tiles) load(buf1);
                both_halves(it, buf0);
                if (it + 1 == tiles) break;
                landed();
                if (it + 2 < tiles) load(buf0);
                both_halves(it + 1, buf1);
            }
        } else {
            for (int it = from; it < tiles; ++it) {
                landed();
                load(buf0);
                landed();
                both_halves(it, buf0);
            }
        }
    };
    if constexpr (BF16) {
        if (tiles <= OWN_DOT_TILES) {
            delta = 0.f;
            walk(0, [&](const char *buf, int u, int j0) __attribute__((always_inline)) {
                V f[A];
                const grawa_f32x16 s = slopes(buf, u, j0, f, [&](int) { return V{}; }, Is<false>());
#pragma unroll
                for (int r = 0; r < 16; ++r) delta += s[r];
            });
            delta += other_half(delta);
            delta = counts ? delta : 0.f;
            landed();
        }
    }
    if (half == 0 && kw == 0 && i < a.row_pitch) {
        const int64_t row = ((int64_t)kn * a.H + head) * a.row_pitch + i;
        a.row_lse[row] = lse;
        a.row_dot[row] = -delta;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_dot[r] = -delta;

    grawa_f32x16 dq[DT];
    // Sums of dS: of the lane's column where all distances are the table's last or beyond, of the lane's column where they are not, and of such
    // distances found there.
    float far_sum = 0.f, near_sum = 0.f, far_diagonals = 0.f;
    // Sums by distance, 16 keys at a time: key y and query c are c - y + 15 places along row y, so that a column has one distance; what a row does not
    // have there stays 0.  A lane adds up a column.
    const auto add_by_distance = [&](const grawa_f32x16 &s, int j0) __attribute__((always_inline)) {
        if constexpr (BIAS)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float *const at_row = diagonals[wave] + (lane & 31) + 15;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int y = (r & 3) + 8 * (r >> 2) + 4 * half;
                    at_row[y * 63] = s[8 * h + r];
                }
                wave_order();
                float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int y = 0; y < 16; ++y) sums[y % 4] += diagonals[wave][y * 64 + lane];
                const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
                const int d = w0 - (j0 + 16 * h) + lane - 15;
                if (d >= a.distances - 1)
                    far_diagonals += sum;
                else if (d >= 0)
                    by_distance[d] += sum;
                wave_order();
            }
    };
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = grawa_f32x16{};
    const auto step = [&](const char *buf, int u, int j0) __attribute__((always_inline)) {
        V f[A];
        const auto columns = [&](int i) { return Tile::by_columns(buf, columns_at + 32 * u * Tile::RB, i / DT * 16, i % DT); };
        const grawa_f32x16 s = slopes(buf, u, j0, f, columns, Is<BF16 && BIAS>());
        if constexpr (BIAS) {
            if (w0 - (j0 + 31) >= a.distances - 1) {
#pragma unroll
                for (int r = 0; r < 16; ++r) far_sum += s[r];
            } else {
                if constexpr (BF16)
#pragma unroll
                    for (int r = 0; r < 16; ++r) near_sum += s[r];
                add_by_distance(s, j0);
            }
        }
        V w[2];
        as_operand(s, 0, w[0]);
        as_operand(s, 1, w[1]);
        __builtin_amdgcn_sched_barrier(0);
        flow<2 * DT>(f, columns, [&](int i, const V &x) __attribute__((always_inline)) { dq[i % DT] = mfma(x, w[i / DT], dq[i % DT]); });
    };
    walk(0, step);
    if constexpr (!BF16) {
        landed();
        float *const other = (float *)buf0 + qw * (DT * 16 * 64) + lane;
        static_assert(2 * DT * 16 * 64 * 4 <= 2 * Tile::BYTES, "room for two waves' sums");
        if (kw)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) other[(d * 16 + r) * 64] = dq[d][r];
        __syncthreads();
        if (!kw)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) dq[d][r] += other[(d * 16 + r) * 64];
    }
    bool odd = false;
    if (counts)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) odd |= dq[d][r] != dq[d][r];
    char *out = a.dq.p + (int64_t)k * a.dq.worker + (int64_t)n * a.dq.seq + (int64_t)i * a.dq.token + (int64_t)head * a.dq.head;
    const auto put = [&](int d, const grawa_f32x16 &sums) {
        if (!there || kw) return;
        grawa_f32x16 v;
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = counts ? sums[r] : 0.f;
        store_column<BF16>(out, lane, d, a.D, v, a.scale);
    };
    // What is no number may come from a token that the query does not see: once more then, with care.
    if (__builtin_expect(!__syncthreads_or(odd), 1)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) put(d, dq[d]);
    } else {
#pragma unroll 1
        for (int d = 0; d < DT; ++d) {
            grawa_f32x16 sums = {};
            restart(0);
            for (int it = 0; it < tiles; ++it) {
                landed();
                load(buf0);
                landed();
#pragma unroll 1
                for (int u = 0; u < 2; ++u) {
                    const int j0 = tile_of(it) + 32 * u;
                    if (none(j0)) continue;
                    V f[A];
                    const grawa_f32x16 s = slopes(buf0, u, j0, f, [&](int) { return V{}; }, Is<false>());
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        V w;
                        as_operand(s, h, w);
                        const V c = Tile::by_columns(buf0 + (32 * u + 16 * h) * Tile::RB, columns_at, 0, d);
                        if (all(j0))
                            sums = mfma(c, w, sums);
                        else
                            product_of_some(sums, c, w, marks<V>(a, pos, j0 + 16 * h, half));
                    }
                }
            }
            put(d, sums);
        }
    }
    if constexpr (BF16 && BIAS) {
        if (tiles > OWN_DOT_TILES) {
            // dS of a row add up to 0.  What they add up to instead is what delta is off by, and each of them is off by P times that: it comes off the
            // sums by distance, the last distance's by the P added up on the way, the others' in one more walk over the tiles that have any of them.
            float off = near_sum + far_sum;
            off += other_half(off);
            off = counts ? off : 0.f;
            int from = tiles;
            while (from > 0 && p0 - (tile_of(from - 1) + BK - 1) < a.distances - 1) --from;
            landed();
            walk(from, [&](const char *buf, int u, int j0) __attribute__((always_inline)) {
                if (w0 - (j0 + 31) >= a.distances - 1) return;
                V f[A];
                const auto keys = [&](int i) { return Tile::by_rows(buf, rows_at + 32 * u * Tile::RB, 0, i); };
                grawa_f32x16 s = {};
                ask(f, keys);
                flow<KS>(f, keys, [&](int i, const V &x) __attribute__((always_inline)) { s = mfma(x, q[i], s); });
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float bias = table[clamp_int(pos - (j0 + (r & 3) + 8 * (r >> 2) + 4 * half), 0, a.distances - 1)];
                    s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, bias) - lse) * -off;
                }
                if (!all(j0))
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = sees(a, pos, j0 + (r & 3) + 8 * (r >> 2) + 4 * half) ? s[r] : 0.f;
                add_by_distance(s, j0);
            });
            far_sum -= off * far_weight;
        }
        far_sum += far_diagonals;
    } else if constexpr (BIAS) {
        far_sum += far_diagonals;
    }
    if constexpr (BIAS) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) far_sum += __shfl_xor(far_sum, m, 64);
        if (lane == 0) by_distance[a.distances - 1] = far_sum;
        __syncthreads();
        for (int d = threadIdx.x; d < a.distances; d += 256) {
            float sum = 0.f;
#pragma unroll
            for (int w = 1; w < 5; ++w) sum += tables[w * a.distances + d];
            table[d] = sum;
        }
        __syncthreads();
        for (int b = threadIdx.x; b < a.buckets; b += 256) {
            float sum = 0.f;
#pragma unroll 8
            for (int d = 0; d < a.distances; ++d) sum += bucket_of[d] == b ? table[d] : 0.f;
            a.bias_part[(((int64_t)kn * a.H + head) * a.blocks + qb) * a.buckets + b] = sum;
        }
    }
#endif
}

// dbias of a head: the sums of its blocks, in order.
template <bool BF16> __global__ __launch_bounds__(256) void k_bias_sums([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int head = blockIdx.x, k = blockIdx.y, b = threadIdx.x;
    if (b >= a.buckets) return;
    float sum = 0.f;
    for (int n = 0; n < a.N; ++n) {
        const float *p = a.bias_part + ((int64_t)(k * a.N + n) * a.H + head) * a.blocks * a.buckets + b;
#pragma unroll 8
        for (int i = 0; i < a.blocks; ++i) sum += p[(int64_t)i * a.buckets];
    }
    char *out = a.dbias.p + ((int64_t)k * a.dbias.worker + (int64_t)head * a.buckets + b) * (BF16 ? 2 : 4);
    store_one<BF16>(out, a.accumulate ? load_one<BF16>(out) + sum : sum);
#endif
}

// A block has 32 keys for each of its NW waves; all waves share tiles of 64 queries and the gradients of their outputs, of one head
// after the other.  Keys and the sums of dk and dv stay in registers, values too where heads have 64 elements; with 128 they do not fit
// and are read from LDS (in registers all the same they were spilled: 32 heads of 16384 tokens, window 4096, 22.6 ms and not 2.0).
// splits > 1 (sink_splits for the keys that all queries see): that many blocks share the queries of a block of keys.
// The four products of a pair and its exponential: 8 workers, 16 heads of 2048 tokens of 64, bf16, 164 us, vector unit 46 %, matrix cores
// 42 %; heads of 128 as above 1890 to 2010, 49 and 48 %, with eight waves on a CU that wait for each other at every tile.
template <bool BF16, int DP, bool BIAS, int NW>
__global__ __launch_bounds__(NW * 64, NW == 8 ? 1 : DP == 64 ? 2 : 1) void k_attend_dkv([[maybe_unused]] GrawaAttend a)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int BQ = 64, BKV = 32 * NW, ES = BF16 ? 2 : 4, KS = DP / 16, DT = DP / 32, BUFS = BF16 ? 2 : 1;
    constexpr bool KEEP = BF16 && DP == 64; // values in registers
    typedef HeadTile<BF16, DP, BQ, NW> Tile;
    typedef HeadTile<BF16, DP, BKV, NW> Values;
    typedef typename Tile::V V;
    __shared__ __attribute__((aligned(1024))) char buf0[2 * Tile::BYTES], buf1[BUFS == 2 ? 2 * Tile::BYTES : 16]; // queries and gradients of outputs
    __shared__ __attribute__((aligned(1024))) float rows0[2 * BQ], rows1[2 * BQ]; // log2 of the sums of exponentials, -do . o
    __shared__ __attribute__((aligned(1024))) char values[KEEP ? 16 : Values::BYTES];
    __shared__ float table[BIAS ? GRAWA_MAX_DISTANCES : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int sink_items = a.sink_blocks * a.sink_splits, groups = a.K * a.N * a.G;
    const Turn turn = turn_of(blockIdx.x, groups, 1, a.by_xcd);
    if (turn.head >= groups) return;
    const int hd = turn.head, item = turn.block;
    const bool sink = item < sink_items;
    const int splits = sink ? a.sink_splits : a.splits, kb = sink ? item / a.sink_splits : a.sink_blocks + (item - sink_items) / a.splits;
    const int split = sink ? item % a.sink_splits : (item - sink_items) % a.splits, slot = sink || a.sink_splits > 1 ? item : item - sink_items;
    const int kn = hd / a.G, g = hd - kn * a.G, k = kn / a.N, n = kn - k * a.N;
    const Place at = place_of(a, kn);
    const int b0 = kb * BKV, w0 = b0 + wave * 32, w1 = w0 + 31, j = w0 + (lane & 31);
    const bool there = j < a.Sk, counts = j < at.length;

    V kf[KS], vf[KEEP ? KS : 1];
    {
        const char *pk = a.k.p + (int64_t)k * a.k.worker + (int64_t)n * a.k.seq + (int64_t)j * a.k.token + (int64_t)g * a.k.head;
        const char *pv = a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)j * a.v.token + (int64_t)g * a.v.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = load_line<BF16>(pk, 16 * ks + 8 * half, a.D, counts);
            if constexpr (KEEP) vf[ks] = load_line<BF16>(pv, 16 * ks + 8 * half, a.D, counts);
        }
    }
    if constexpr (!KEEP) { // lands before the first tile does
        Values lv;
        lv.init(wave, lane, (uint32_t)a.v.token, a.D);
        lv.load(values, wave, Values::rsrc(a.v.p + (int64_t)k * a.v.worker + (int64_t)n * a.v.seq + (int64_t)b0 * a.v.token + (int64_t)g * a.v.head,
                                           at.length - b0, (uint32_t)a.v.token, a.D));
    }
    const uint32_t values_at = Values::rows_of(lane) + wave * 32 * Values::RB;
    const auto value = [&](int ks) {
        if constexpr (KEEP)
            return vf[ks];
        else
            return Values::by_rows(values, here(values_at), 0, ks);
    };
    const float c2 = a.scale * LOG2E;

    // Queries that see any of the block's keys: rows i0 ... i1 of the call, by tiles, of each head.
    const int last = min(at.length - 1 - at.start, a.Sq - 1);
    const int i0 = max(0, b0 - at.start), i1 = sink ? last : min(last, b0 + BKV - 1 + a.window - 1 - at.start);
    const int t0 = i0 / BQ, tiles = b0 < at.length && i1 >= i0 ? i1 / BQ - t0 + 1 : 0, all_tiles = tiles * a.share;
    const int from = (int)((int64_t)all_tiles * split / splits), to = (int)((int64_t)all_tiles * (split + 1) / splits);
    Tile lq, lg;
    lq.init(wave, lane, (uint32_t)a.q.token, a.D);
    lg.init(wave, lane, (uint32_t)a.go.token, a.D);
    const char *qp = a.q.p + (int64_t)k * a.q.worker + (int64_t)n * a.q.seq, *gp = a.go.p + (int64_t)k * a.go.worker + (int64_t)n * a.go.seq;
    struct At {
        int h, tile; // head of the group, first query of the tile
        const char *q, *go;
        const float *rows;
    };
    const auto head_of = [&](int h, int tile) __attribute__((always_inline)) {
        const int head = g * a.share + h;
        return At{h, tile, qp + (int64_t)tile * a.q.token + (int64_t)head * a.q.head, gp + (int64_t)tile * a.go.token + (int64_t)head * a.go.head,
                  (wave ? a.row_dot : a.row_lse) + ((int64_t)kn * a.H + head) * a.row_pitch + tile};
    };
    const auto place = [&](int it) {
        const int h = it / tiles;
        return head_of(h, (t0 + it - h * tiles) * BQ);
    };
    const uint32_t q_token = (uint32_t)a.q.token, go_token = (uint32_t)a.go.token, bytes = a.D * ES;
    const auto load = [&](At t, char *buf, float *rows) __attribute__((always_inline)) {
        const uint32_t n = last + 1 - t.tile < BQ ? last + 1 - t.tile : BQ; // more than 0
        lq.load(buf, wave, __builtin_amdgcn_make_buffer_rsrc((void *)t.q, 0, (n - 1) * q_token + bytes, 0x00020000));
        lg.load(buf + Tile::BYTES, wave, __builtin_amdgcn_make_buffer_rsrc((void *)t.go, 0, (n - 1) * go_token + bytes, 0x00020000));
        if (wave < 2) // rows up to the pitch, a multiple of a tile, are there
            __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)t.rows, 0, BQ * 4, 0x00020000),
                                                     (GRAWA_LDS_AT void *)(rows + wave * BQ), 4, (uint32_t)lane * 4, 0, 0, 0);
    };
    const auto next = [&](At t) __attribute__((always_inline)) {
        if (t.tile + BQ >= (t0 + tiles) * BQ) return head_of(t.h + 1, t0 * BQ);
        return At{t.h, t.tile + BQ, t.q + (int64_t)BQ * a.q.token, t.go + (int64_t)BQ * a.go.token, t.rows + BQ};
    };
    int table_of = -1;
    const auto tabulate = [&](int h) {
        if constexpr (BIAS) {
            if (h == table_of) return;
            // the other waves are behind their last look at the table of the head before
            const char *bias = a.bias.p + ((int64_t)k * a.bias.worker + (int64_t)(g * a.share + h) * a.buckets) * ES;
            for (int d = threadIdx.x; d < a.distances; d += NW * 64) table[d] = bias_of<BF16>(bias + a.bucket_of[d] * ES);
            table_of = h;
            __syncthreads();
        }
    };
    // p0: position of the first of 32 queries
    const auto none = [&](int p0) { return w0 > p0 + 31 || w0 >= at.length || (w1 <= p0 - a.window && w0 >= a.sinks); }; // of the wave's pairs count
    const auto all = [&](int p0) { return w1 <= p0 && (p0 + 31 - w0 < a.window || w1 < a.sinks); };
    const uint32_t rows_at = Tile::rows_of(lane), columns_at = Tile::columns_of(lane);
    constexpr int A = BF16 ? (DP == 128 ? 2 : 4) : 2;
    // P and dS of 32 queries; leaves the first fragments of `then` in f.
    const auto slopes = [&](const char *buf, const float *of_rows, int u, int p0, grawa_f32x16 &s, grawa_f32x16 &dp, V (&f)[A], auto &&then) __attribute__((always_inline)) {
        const uint32_t at = rows_at + 32 * u * Tile::RB;
        const auto rows = [&](int i) { return Tile::by_rows(buf + i / KS * Tile::BYTES, KEEP ? at : here(at), 0, i % KS); };
        s = grawa_f32x16{};
        ask(f, rows);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const grawa_f32x4v dot = *(const grawa_f32x4v *)(of_rows + BQ + 32 * u + 8 * x + 4 * half);
#pragma unroll
            for (int y = 0; y < 4; ++y) dp[4 * x + y] = dot[y];
        }
        V v[KEEP ? 1 : 2]; // values, asked for two before they are used
        if constexpr (!KEEP) v[0] = value(0), v[1] = value(1);
        flow<2 * KS>(f, rows, [&](int i, const V &x) __attribute__((always_inline)) {
            if (i < KS) {
                s = mfma(x, kf[i], s);
            } else if constexpr (KEEP) {
                dp = mfma(x, value(i - KS), dp);
            } else {
                dp = mfma(x, v[i % 2], dp);
                if (i + 2 < 2 * KS) v[i % 2] = value(i + 2 - KS);
            }
        });
        ask(f, then);
        const float far = BIAS ? table[a.distances - 1] : 0.f;
        const auto form = [&](auto near) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const grawa_f32x4v lse = *(const grawa_f32x4v *)(of_rows + 32 * u + 8 * x + 4 * half);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    if constexpr (BIAS) { // the score as the forward pass has it
                        const float bias = near.value ? table[clamp_int(p0 + 8 * x + 4 * half + y - j, 0, a.distances - 1)] : far;
                        s[4 * x + y] = __builtin_fmaf(s[4 * x + y], c2, bias) - lse[y];
                    } else {
                        s[4 * x + y] = __builtin_fmaf(s[4 * x + y], c2, -lse[y]);
                    }
                }
            }
        };
        if (BIAS && p0 - w1 < a.distances - 1)
            form(Is<BIAS>());
        else
            form(Is<false>());
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r]);
            dp[r] *= s[r];
        }
        if (!all(p0))
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool seen = sees(a, p0 + (r & 3) + 8 * (r >> 2) + 4 * half, j);
                s[r] = seen ? s[r] : 0.f;
                dp[r] = seen ? dp[r] : 0.f;
            }
    };

    grawa_f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = grawa_f32x16{};
    // One way through the step, masked or not: with two the sums change their registers between them.
    const auto step = [&](At t, const char *buf, const float *of_rows) __attribute__((always_inline)) {
        tabulate(t.h);
#pragma unroll 1
        for (int u = 0; u < 2; ++u) {
            const int p0 = at.start + t.tile + 32 * u;
            if (none(p0)) continue;
            grawa_f32x16 s, dp;
            V f[A], w[4];
            const uint32_t lines = columns_at + 32 * u * Tile::RB;
            const auto columns = [&](int i) { return Tile::by_columns(buf + (1 - i / (2 * DT)) * Tile::BYTES, KEEP ? lines : here(lines), i / DT % 2 * 16, i % DT); };
            slopes(buf, of_rows, u, p0, s, dp, f, columns);
            as_operand(s, 0, w[0]);
            as_operand(s, 1, w[1]);
            as_operand(dp, 0, w[2]);
            as_operand(dp, 1, w[3]);
            __builtin_amdgcn_sched_barrier(0);
            flow<4 * DT>(f, columns, [&](int i, const V &x) __attribute__((always_inline)) {
                if (i < 2 * DT)
                    dv[i % DT] = mfma(x, w[i / DT], dv[i % DT]);
                else
                    dk[i % DT] = mfma(x, w[i / DT], dk[i % DT]);
            });
        }
    };
    if (from < to) {
        At t = place(from);
        if constexpr (BUFS == 2) {
            load(t, buf0, rows0);
            for (int it = from; it < to; it += 2) {
                const At t1 = next(t), t2 = next(t1);
                landed();
                if (it + 1 < to) load(t1, buf1, rows1);
                step(t, buf0, rows0);
                if (it + 1 == to) break;
                landed();
                if (it + 2 < to) load(t2, buf0, rows0);
                step(t1, buf1, rows1);
                t = t2;
            }
        } else {
            for (int it = from; it < to; ++it, t = next(t)) {
                landed();
                load(t, buf0, rows0);
                landed();
                step(t, buf0, rows0);
            }
        }
    }
    bool odd = false;
    if (counts)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) odd |= dk[d][r] != dk[d][r] || dv[d][r] != dv[d][r];
    const auto put = [&](bool keys, int d, const grawa_f32x16 &sums) {
        if (!there) return;
        grawa_f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = counts ? sums[r] : 0.f;
        const GrawaHeads &to = keys ? a.dk : a.dv;
        if (splits > 1)
            store_column<false>((char *)(a.part + (((int64_t)hd * a.slots + slot) * BKV + (j - b0)) * 2 * DP + (keys ? 0 : DP)), lane, d, DP, x, keys ? a.scale : 1.f);
        else
            store_column<BF16>(to.p + (int64_t)k * to.worker + (int64_t)n * to.seq + (int64_t)j * to.token + (int64_t)g * to.head, lane, d, a.D, x, keys ? a.scale : 1.f);
    };
    // What is no number may come from a query that does not see the key, or from one that counts for nothing: its 0 x exp2(-infinity) is no
    // number beside a key that is none.  Once more then, with care.
    if (__builtin_expect(!__syncthreads_or(odd), 1)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) put(false, d, dv[d]), put(true, d, dk[d]);
        return;
    }
#pragma unroll 1
    for (int x = 0; x < 2 * DT; ++x) {
        const bool keys = x >= DT;
        const int d = x % DT;
        grawa_f32x16 sums = {};
#pragma unroll 1
        for (int it = from; it < to; ++it) {
            const At t = place(it);
            landed();
            load(t, buf0, rows0);
            landed();
            tabulate(t.h);
#pragma unroll 1
            for (int u = 0; u < 2; ++u) {
                const int p0 = at.start + t.tile + 32 * u;
                if (none(p0)) continue;
                grawa_f32x16 s, dp;
                V f[A];
                slopes(buf0, rows0, u, p0, s, dp, f, [&](int) { return V{}; });
                // Rows that count for nothing, queries that are not there among them: what they have may be no number, theirs or with this key.
                const auto counting = [&](int r) { return rows0[32 * u + (r & 3) + 8 * (r >> 2) + 4 * half] != __builtin_inff(); };
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = !counting(r) ? 0.f : keys ? dp[r] : s[r];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    V w, seen;
#pragma unroll
                    for (int r = 0; r < 8; ++r) seen[r] = counting(8 * h + r) && sees(a, p0 + 16 * h + (r & 3) + 8 * (r >> 2) + 4 * half, j) ? 1.f : 0.f;
                    as_operand(s, h, w);
                    product_of_some(sums, Tile::by_columns(buf0 + (keys ? 0 : Tile::BYTES) + (32 * u + 16 * h) * Tile::RB, columns_at, 0, d), w, seen);
                }
            }
        }
        put(keys, d, sums);
    }
#endif
}

// dk and dv of the keys whose queries several blocks shared: their sums, in order.
template <bool BF16, int DP, int BKV> __global__ __launch_bounds__(256) void k_attend_dkv_join([[maybe_unused]] GrawaAttend a, [[maybe_unused]] int first, [[maybe_unused]] int blocks)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int LPR = 2 * DP / 8, ES = BF16 ? 2 : 4, PN = GrawaPiece<BF16>::N; // threads of a key: half have dk, half dv
    const int64_t id = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;    // [K N][G][blocks][BKV]
    const int x = threadIdx.x % LPR, which = x / (LPR / 2), e0 = x % (LPR / 2) * 8;
    const int key = (int)(id % BKV), kb = first + (int)(id / BKV % blocks);
    const int64_t hd = id / BKV / blocks;
    const int j = kb * BKV + key;
    if (hd >= (int64_t)a.K * a.N * a.G || j >= a.Sk) return;
    const bool sink = kb < a.sink_blocks;
    const int splits = sink ? a.sink_splits : a.splits;
    const int slot = sink ? kb * a.sink_splits : (a.sink_splits > 1 ? a.sink_blocks * a.sink_splits : 0) + (kb - a.sink_blocks) * a.splits;
    float v[8] = {};
    for (int s = 0; s < splits; ++s) {
        const grawa_f32x4v *p = (const grawa_f32x4v *)(a.part + ((hd * a.slots + slot + s) * BKV + key) * 2 * DP + which * DP + e0);
        const grawa_f32x4v b = p[0], c = p[1];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += b[q], v[4 + q] += c[q];
    }
    const int kn = (int)(hd / a.G), g = (int)(hd - (int64_t)kn * a.G), k = kn / a.N, n = kn - k * a.N;
    const GrawaHeads &to = which ? a.dv : a.dk;
    char *out = to.p + (int64_t)k * to.worker + (int64_t)n * to.seq + (int64_t)j * to.token + (int64_t)g * to.head;
#pragma unroll
    for (int q = 0; q < 8; q += PN)
        if (e0 + q < a.D) store_piece<BF16>(out + (e0 + q) * ES, PN, v + q);
#endif
}

template <bool BF16, int DP, bool BIAS> hipError_t launch(GrawaAttend a, int64_t part_floats, hipStream_t st)
{
    const int64_t kn = (int64_t)a.K * a.N;
    hipError_t e;
    if (a.Sq > 0) {
        a.blocks = (a.Sq + grawa_dq_queries(BF16) - 1) / grawa_dq_queries(BF16);
        const uint32_t grid = grid_of(kn * a.G, a.share, a.blocks, a.by_xcd);
        // 2^24 blocks, which float32 comes to, are more threads than an axis of a grid takes: two rows of them then, each of whole turns of the XCDs.
        const uint32_t rows = grid < 1u << 24 ? 1 : 2;
        hipLaunchKernelGGL((k_attend_dq<BF16, DP, BIAS>), dim3(rows == 1 ? grid : (grid + 15) / 16 * 8, rows), dim3(256), BIAS ? (uint32_t)a.distances * 6 * sizeof(float) : 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (BIAS) {
        if (a.Sq == 0) a.blocks = 0;
        hipLaunchKernelGGL((k_bias_sums<BF16>), dim3((uint32_t)a.H, (uint32_t)a.K), dim3(256), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.Sk == 0) return hipSuccess;
    constexpr int NW = BF16 && DP == 128 ? 8 : 4, BKV = 32 * NW;
    a.key_blocks = (a.Sk + BKV - 1) / BKV;
    // Blocks of keys that all later queries see, and not only those that the window lets through.
    const int64_t window_tiles = ((int64_t)a.window + BKV + 63) / 64, tiles = (a.Sq + 63) / 64, sink_blocks = ((int64_t)a.sinks + BKV - 1) / BKV;
    a.sink_blocks = a.window == GRAWA_NO_WINDOW ? 0 : (int)(sink_blocks < a.key_blocks ? sink_blocks : a.key_blocks);
    const int64_t groups = kn * a.G, room = part_floats / ((int64_t)BKV * 2 * DP) / groups; // for so many blocks of a group
    const int64_t regular = a.key_blocks - a.sink_blocks, most = (tiles < window_tiles ? tiles : window_tiles) * a.share;
    // Items enough for every CU (twice as many, float32, 4 workers of 3 sequences of 600 and less: no faster).  A block of first keys is
    // shared as often as makes its items as long as the others.
    const int64_t as_long = a.sink_blocks && most > 0 ? (tiles * a.share + most - 1) / most : 1;
    int64_t splits = regular ? 512 / (groups * regular) : 1;
    if (splits > most / 2) splits = most / 2;
    if (splits > room / (regular + a.sink_blocks * as_long)) splits = room / (regular + a.sink_blocks * as_long);
    if (splits < 1) splits = 1;
    int64_t sink_splits = as_long * splits;
    const int64_t left = room - (splits > 1 ? regular * splits : 0);
    if (a.sink_blocks && sink_splits > left / a.sink_blocks) sink_splits = left / a.sink_blocks;
    if (!a.sink_blocks || sink_splits < 1) sink_splits = 1;
    a.splits = (int)splits;
    a.sink_splits = (int)sink_splits;
    a.slots = (int)((sink_splits > 1 ? a.sink_blocks * sink_splits : 0) + (splits > 1 ? regular * splits : 0));
    const int64_t per = (int64_t)a.sink_blocks * a.sink_splits + regular * a.splits;
    const uint32_t grid = grid_of(groups, 1, per, a.by_xcd);
    hipLaunchKernelGGL((k_attend_dkv<BF16, DP, BIAS, NW>), dim3(grid), dim3(NW * 64), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int first = a.sink_splits > 1 ? 0 : a.sink_blocks, end = a.splits > 1 ? a.key_blocks : a.sink_blocks;
    if (end <= first) return hipSuccess;
    const int64_t ids = groups * (end - first) * BKV;
    hipLaunchKernelGGL((k_attend_dkv_join<BF16, DP, BKV>), dim3((uint32_t)(ids * (DP / 4) / 256)), dim3(256), 0, st, a, first, end - first);
    return hipGetLastError();
}

} // namespace

hipError_t grawa_launch_attend_backward(const grawa_attention_plan *s, GrawaAttend a, hipStream_t st)
{
    if (a.N == 0) { // nothing but the bias's gradient, of no pairs
        if (!a.buckets) return hipSuccess;
        a.blocks = 0;
        if (s->dtype == GRAWA_BF16)
            hipLaunchKernelGGL((k_bias_sums<true>), dim3((uint32_t)a.H, (uint32_t)a.K), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_bias_sums<false>), dim3((uint32_t)a.H, (uint32_t)a.K), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const bool bias = a.buckets > 0, wide = grawa_padded_width(a.D) == 128;
    if (s->dtype == GRAWA_BF16) {
        if (wide) return bias ? launch<true, 128, true>(a, s->part_floats, st) : launch<true, 128, false>(a, s->part_floats, st);
        return bias ? launch<true, 64, true>(a, s->part_floats, st) : launch<true, 64, false>(a, s->part_floats, st);
    }
    if (wide) return bias ? launch<false, 128, true>(a, s->part_floats, st) : launch<false, 128, false>(a, s->part_floats, st);
    return bias ? launch<false, 64, true>(a, s->part_floats, st) : launch<false, 64, false>(a, s->part_floats, st);
}
