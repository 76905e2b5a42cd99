// Layer norm over the last axis of [K][T][d], forward and backward, each worker with its own weight and bias:
//   mean = sum x / d;  rstd = (sum (x - mean)^2 / d + eps)^(-1/2);  xhat = (x - mean) rstd;  y = xhat w + b
//   a = dy w;  dx = rstd (a - mean(a) - xhat mean(a xhat)) [+ add];  dw = sum_t dy xhat;  db = sum_t dy
// Both passes are bound by memory.  A row is read once and stays in registers, so that the variance is that of the centered
// values (no difference of large sums).  Results are stored past the caches, whose place the second reading of x then has:
// 8 x 2048 x 1024 in bfloat16, forward and backward, 43.4 us by cached stores, 37.7 so.  Followed by a copy of its result a
// norm by itself is up to 11 % slower for it (8 x 2048 x 1024 in float32, 40.8 us and 45.5) or 5 % faster (8 x 512 in bfloat16); a sublayer's evaluation
// and training step, 64 to 4096 tokens of 1 to 16 workers, take the same within 2 % either way.  Everything is summed in float32; the sums over tokens are split over blocks, each block's
// kept in registers, left in a workspace and added in a fixed order by a second launch: results do not depend on timing.
#include "grawa_elements.h"
#include "grawa_sublayer.h"

namespace {

__device__ __forceinline__ float wave_sum_f(float v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// Sum over the TPR threads of a row; every thread gets it.  sm: one float per wave, not in use by an earlier call's readers (two
// buffers in turn).
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *sm)
{
    v = wave_sum_f(v);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0) sm[wave] = v;
        __syncthreads();
        v = sm[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) v += sm[i];
    }
    return v;
}

// A block of BLOCK threads holds BLOCK / TPR rows side by side; thread c of a row has the 16-byte pieces j TPR + c of it, j < NV.
// Rows up to 1024 elements are a wave's, which needs no barrier.  8 x 2048 x 1024 in bfloat16: 12.5 us, 5.4 TB/s.
template <bool BF16, int NV, int TPR, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_norm(GrawaRows x, GrawaMat w, GrawaMat b, float eps, GrawaRows y, float *stats, int64_t t0, int64_t T, int d)
{
    typedef GrawaPiece<BF16> Piece;
    constexpr int S = Piece::S, N = Piece::N;
    static_assert(TPR == 64 || TPR == BLOCK, "a row is a wave's or the block's");
    __shared__ float sm[2][BLOCK / 64];
    const int c = threadIdx.x % TPR, k = blockIdx.y;
    const int64_t t = t0 + (int64_t)blockIdx.x * (BLOCK / TPR) + threadIdx.x / TPR;
    if (t >= T) return; // whole waves of a row that is one wave's, or the whole block
    const char *px = x.p + ((int64_t)k * x.worker + t * x.row) * S;
    const char *pw = w.p + (int64_t)k * w.worker * S, *pb = b.p ? b.p + (int64_t)k * b.worker * S : nullptr;
    Piece v[NV], ww[NV], bb[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) { // all on their way before the first is waited for
        const int e = (j * TPR + c) * N;
        if (e >= d) continue;
        v[j].load(px + (int64_t)e * S, d - e);
        ww[j].load(pw + (int64_t)e * S, d - e);
        if (pb) bb[j].load(pb + (int64_t)e * S, d - e);
    }
    float sum = 0.f, sq = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if ((j * TPR + c) * N < d)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += v[j][i];
    const float mean = row_sum<TPR>(sum, sm[0]) / (float)d;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((j * TPR + c) * N + i < d) sq += (v[j][i] - mean) * (v[j][i] - mean);
    const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, sm[1]) / (float)d + eps);
    if (stats && c == 0) *(float2 *)(stats + 2 * ((int64_t)k * T + t)) = make_float2(mean, rstd);
    char *py = y.p + ((int64_t)k * y.worker + t * y.row) * S;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int e = (j * TPR + c) * N;
        if (e >= d) continue;
        float r[N];
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = (v[j][i] - mean) * rstd * ww[j][i] + (pb ? bb[j][i] : 0.f);
        store_piece<BF16, true>(py + (int64_t)e * S, d - e, r);
    }
}

// Rows that no block holds: they are read three times.
template <bool BF16> __global__ __launch_bounds__(1024) void k_norm_long(GrawaRows x, GrawaMat w, GrawaMat b, float eps, GrawaRows y, float *stats, int64_t t0, int64_t T, int d)
{
    constexpr int S = BF16 ? 2 : 4;
    __shared__ float sm[2][16];
    const int c = threadIdx.x, k = blockIdx.y;
    const int64_t t = t0 + blockIdx.x;
    const char *px = x.p + ((int64_t)k * x.worker + t * x.row) * S;
    float sum = 0.f, sq = 0.f, v, ww, bb = 0.f;
    for (int e = c; e < d; e += 1024) {
        v = load_one<BF16>(px + (int64_t)e * S);
        sum += v;
    }
    const float mean = row_sum<1024>(sum, sm[0]) / (float)d;
    for (int e = c; e < d; e += 1024) {
        v = load_one<BF16>(px + (int64_t)e * S);
        sq += (v - mean) * (v - mean);
    }
    const float rstd = 1.f / sqrtf(row_sum<1024>(sq, sm[1]) / (float)d + eps);
    if (stats && c == 0) *(float2 *)(stats + 2 * ((int64_t)k * T + t)) = make_float2(mean, rstd);
    char *py = y.p + ((int64_t)k * y.worker + t * y.row) * S;
    const char *pw = w.p + (int64_t)k * w.worker * S, *pb = b.p ? b.p + (int64_t)k * b.worker * S : nullptr;
    for (int e = c; e < d; e += 1024) { // y may be x: a thread writes what only it reads again
        v = load_one<BF16>(px + (int64_t)e * S);
        ww = load_one<BF16>(pw + (int64_t)e * S);
        if (pb) bb = load_one<BF16>(pb + (int64_t)e * S);
        v = (v - mean) * rstd * ww + bb;
        store_one<BF16>(py + (int64_t)e * S, v);
    }
}

// The backward pass of rows t0, t0 + step, ... of a worker; the next row is on its way while one is worked on.  part:
// [K][gridDim.x][2][d], the block's sums of dw and db.  8 x 2048 x 1024 in bfloat16: 23.0 us, 4.4 TB/s, and 4.7 for the sums.
template <bool BF16, int NV, int TPR, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_norm_back(GrawaRows dy, GrawaRows x, GrawaMat w, const float *stats, GrawaRows add, GrawaRows dx,
                                                     float *part, int64_t T, int d)
{
    typedef GrawaPiece<BF16> Piece;
    constexpr int S = Piece::S, N = Piece::N, ROWS = BLOCK / TPR;
    static_assert(TPR == 64 || TPR == BLOCK, "a row is a wave's or the block's");
    __shared__ float sm[4][BLOCK / 64];
    __shared__ float cols[ROWS > 1 ? NV * TPR * N : 1];
    const int c = threadIdx.x % TPR, k = blockIdx.y;
    const char *pw = w.p + (int64_t)k * w.worker * S;
    Piece ww[NV], nx[NV], ndy[NV], nadd[NV];
    float dw[NV][N] = {}, db[NV][N] = {};
    float2 nst = make_float2(0.f, 0.f);
    auto fetch = [&](int64_t t) {
        const char *px = x.p + ((int64_t)k * x.worker + t * x.row) * S, *pdy = dy.p + ((int64_t)k * dy.worker + t * dy.row) * S;
        const char *padd = add.p ? add.p + ((int64_t)k * add.worker + t * add.row) * S : nullptr;
        nst = *(const float2 *)(stats + 2 * ((int64_t)k * T + t));
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (j * TPR + c) * N;
            if (e >= d) continue;
            nx[j].load(px + (int64_t)e * S, d - e);
            ndy[j].load(pdy + (int64_t)e * S, d - e);
            if (padd) nadd[j].load(padd + (int64_t)e * S, d - e);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR, step = (int64_t)gridDim.x * ROWS;
    if (first < T) fetch(first);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if ((j * TPR + c) * N < d) ww[j].load(pw + (int64_t)(j * TPR + c) * N * S, d - (j * TPR + c) * N);
    int turn = 0; // which pair of `sm`: a wave may be one row ahead of another
    for (int64_t t = first; t < T; t += step, turn ^= 2) {
        const float2 st = nst;
        Piece px[NV], pdy[NV], padd[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) px[j] = nx[j], pdy[j] = ndy[j], padd[j] = nadd[j];
        // dx may be dy or add: a row is read by nobody but those who write it
        if (t + step < T) fetch(t + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if ((j * TPR + c) * N >= d) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) { // behind the row's end dy is 0
                const float h = (px[j][i] - st.x) * st.y, a = pdy[j][i] * ww[j][i];
                dw[j][i] += pdy[j][i] * h;
                db[j][i] += pdy[j][i];
                s1 += a;
                s2 += a * h;
            }
        }
        const float m1 = row_sum<TPR>(s1, sm[turn]) / (float)d, m2 = row_sum<TPR>(s2, sm[turn + 1]) / (float)d;
        char *pdx = dx.p + ((int64_t)k * dx.worker + t * dx.row) * S;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (j * TPR + c) * N;
            if (e >= d) continue;
            float r[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float h = (px[j][i] - st.x) * st.y, a = pdy[j][i] * ww[j][i];
                r[i] = st.y * (a - m1 - h * m2) + (add.p ? padd[j][i] : 0.f);
            }
            store_piece<BF16, true>(pdx + (int64_t)e * S, d - e, r);
        }
    }
    float *out = part + ((int64_t)k * gridDim.x + blockIdx.x) * 2 * d;
    if constexpr (ROWS > 1) { // the block's rows one after the other, in order
#pragma unroll
        for (int what = 0; what < 2; ++what) {
            for (int r = 0; r < ROWS; ++r) {
                __syncthreads();
                if (threadIdx.x / TPR == r)
#pragma unroll
                    for (int j = 0; j < NV; ++j)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const int e = (j * TPR + c) * N + i;
                            const float v = what ? db[j][i] : dw[j][i];
                            cols[e] = r ? cols[e] + v : v;
                        }
            }
            __syncthreads();
            for (int e = threadIdx.x; e < d; e += BLOCK) out[(int64_t)what * d + e] = cols[e];
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = (j * TPR + c) * N + i;
                if (e < d) {
                    out[e] = dw[j][i];
                    out[d + e] = db[j][i];
                }
            }
    }
}

// Rows that no block holds: dx by a block for each row, dw and db by a thread for each column of a range of rows.
template <bool BF16> __global__ __launch_bounds__(1024) void k_norm_back_long(GrawaRows dy, GrawaRows x, GrawaMat w, const float *stats, GrawaRows add, GrawaRows dx, int64_t t0, int64_t T, int d)
{
    constexpr int S = BF16 ? 2 : 4;
    __shared__ float sm[2][16];
    const int c = threadIdx.x, k = blockIdx.y;
    const int64_t t = t0 + blockIdx.x;
    const char *px = x.p + ((int64_t)k * x.worker + t * x.row) * S, *pdy = dy.p + ((int64_t)k * dy.worker + t * dy.row) * S;
    const char *pw = w.p + (int64_t)k * w.worker * S;
    const float2 st = *(const float2 *)(stats + 2 * ((int64_t)k * T + t));
    float s1 = 0.f, s2 = 0.f, v, a, ww;
    for (int e = c; e < d; e += 1024) {
        v = load_one<BF16>(px + (int64_t)e * S);
        a = load_one<BF16>(pdy + (int64_t)e * S);
        ww = load_one<BF16>(pw + (int64_t)e * S);
        a *= ww;
        s1 += a;
        s2 += a * (v - st.x) * st.y;
    }
    const float m1 = row_sum<1024>(s1, sm[0]) / (float)d, m2 = row_sum<1024>(s2, sm[1]) / (float)d;
    char *pdx = dx.p + ((int64_t)k * dx.worker + t * dx.row) * S;
    const char *padd = add.p ? add.p + ((int64_t)k * add.worker + t * add.row) * S : nullptr;
    for (int e = c; e < d; e += 1024) {
        float r = 0.f;
        v = load_one<BF16>(px + (int64_t)e * S);
        a = load_one<BF16>(pdy + (int64_t)e * S);
        ww = load_one<BF16>(pw + (int64_t)e * S);
        if (padd) r = load_one<BF16>(padd + (int64_t)e * S);
        r += st.y * (a * ww - m1 - (v - st.x) * st.y * m2);
        store_one<BF16>(pdx + (int64_t)e * S, r);
    }
}

template <bool BF16> __global__ __launch_bounds__(256) void k_norm_back_cols(GrawaRows dy, GrawaRows x, const float *stats, float *part, int64_t T, int d)
{
    constexpr int S = BF16 ? 2 : 4;
    const int e = blockIdx.y * 256 + threadIdx.x, k = blockIdx.z;
    if (e >= d) return;
    float dw = 0.f, db = 0.f, v, a;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        v = load_one<BF16>(x.p + ((int64_t)k * x.worker + t * x.row + e) * S);
        a = load_one<BF16>(dy.p + ((int64_t)k * dy.worker + t * dy.row + e) * S);
        const float2 st = *(const float2 *)(stats + 2 * ((int64_t)k * T + t));
        dw += a * (v - st.x) * st.y;
        db += a;
    }
    float *out = part + ((int64_t)k * gridDim.x + blockIdx.x) * 2 * d;
    out[e] = dw;
    out[d + e] = db;
}

// The blocks' sums added up: 64 columns a block, its sixteen waves take every sixteenth of the n parts.
template <bool BF16> __global__ __launch_bounds__(1024) void k_norm_sums(const float *part, int n, GrawaMat dw, GrawaMat db, int accumulate, int d)
{
    constexpr int S = BF16 ? 2 : 4;
    __shared__ float sm[16][64];
    const int c = threadIdx.x % 64, g = threadIdx.x / 64, k = blockIdx.y, what = blockIdx.z;
    const int e = blockIdx.x * 64 + c;
    float s = 0.f;
    if (e < d) {
#pragma unroll 8
        for (int i = g; i < n; i += 16) s += part[(((int64_t)k * n + i) * 2 + what) * d + e];
    }
    sm[g][c] = s;
    __syncthreads();
    const GrawaMat &m = what ? db : dw;
    if (g || e >= d || !m.p) return;
    char *p = m.p + ((int64_t)k * m.worker + e) * S;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 4) v += (sm[i][c] + sm[i + 1][c]) + (sm[i + 2][c] + sm[i + 3][c]);
    if (accumulate) v += load_one<BF16>(p);
    store_one<BF16>(p, v);
}

// What takes a row of d elements: the fewest threads that hold it in at most 32 registers each.
#define GRAWA_NORM_FORMS(GO, GOLONG, BF)                                   \
    do {                                                                   \
        constexpr int N = GrawaPiece<BF>::N;                               \
        if (d <= 8 * 64) GO(BF, (8 / N), 64, 256);                         \
        else if (d <= 16 * 64) GO(BF, (16 / N), 64, 256);                  \
        else if (d <= 16 * 256) GO(BF, (16 / N), 256, 256);                \
        else if (d <= 32 * 256) GO(BF, (32 / N), 256, 256);                \
        else if (d <= 16 * 1024) GO(BF, (16 / N), 1024, 1024);             \
        else GOLONG(BF);                                                   \
    } while (0)

} // namespace

// Blocks of a worker in the backward pass: at most four for each CU over all workers, and each with rows enough (two for every one
// that it holds at a time) that its sums are little beside them.  That leaves CUs idle where rows are few: 3 x 517 rows of 1003 are 195 blocks.
int grawa_norm_blocks(int K, int64_t T, int64_t d)
{
    const int64_t rows = d <= 1024 ? 4 : 1, groups = (T + 2 * rows - 1) / (2 * rows);
    const int64_t want = 1024 / K > 1 ? 1024 / K : 1;
    const int64_t n = groups < want ? groups : want;
    return (int)(n > 0 ? n : 1);
}

// T rows by blocks that hold `rows` each: a launch has fewer than 2^32 threads along x, so very many rows take several.
template <class F> static void launch_rows(int64_t T, int rows, int threads, const F &launch)
{
    const int64_t most = ((int64_t)1 << 31) / threads * rows;
    for (int64_t t0 = 0; t0 < T; t0 += most) {
        const int64_t n = T - t0 < most ? T - t0 : most;
        launch((unsigned)((n + rows - 1) / rows), t0);
    }
}

hipError_t grawa_launch_layer_norm(const grawa_sublayer *s, int64_t T, GrawaRows x, GrawaMat w, GrawaMat b, float eps, GrawaRows y,
                                   float *stats, hipStream_t st)
{
    if (!T) return hipSuccess;
    const int d = (int)s->d;
    const unsigned K = (unsigned)s->K;
#define GO(BF, NV, TPR, BLOCK)                                                                                           \
    launch_rows(T, BLOCK / TPR, BLOCK, [&](unsigned n, int64_t t0) { k_norm<BF, NV, TPR, BLOCK><<<dim3(n, K), BLOCK, 0, st>>>(x, w, b, eps, y, stats, t0, T, d); })
#define GOLONG(BF) launch_rows(T, 1, 1024, [&](unsigned n, int64_t t0) { k_norm_long<BF><<<dim3(n, K), 1024, 0, st>>>(x, w, b, eps, y, stats, t0, T, d); })
    if (s->dtype == GRAWA_BF16) GRAWA_NORM_FORMS(GO, GOLONG, true);
    else GRAWA_NORM_FORMS(GO, GOLONG, false);
#undef GO
#undef GOLONG
    return hipGetLastError();
}

hipError_t grawa_launch_layer_norm_backward(const grawa_sublayer *s, int64_t T, GrawaRows dy, GrawaRows x, GrawaMat w, const float *stats,
                                            GrawaRows add, GrawaRows dx, GrawaMat dw, GrawaMat db, int accumulate, hipStream_t st)
{
    const int d = (int)s->d, nb = T ? grawa_norm_blocks(s->K, T, d) : 0;
    float *part = s->norm_part;
    if (T) {
        const dim3 grid((unsigned)nb, (unsigned)s->K);
#define GO(BF, NV, TPR, BLOCK) k_norm_back<BF, NV, TPR, BLOCK><<<grid, BLOCK, 0, st>>>(dy, x, w, stats, add, dx, part, T, d)
#define GOLONG(BF)                                                                                                               \
    do {                                                                                                                         \
        k_norm_back_cols<BF><<<dim3((unsigned)nb, (unsigned)((d + 255) / 256), (unsigned)s->K), 256, 0, st>>>(dy, x, stats, part, T, d); \
        launch_rows(T, 1, 1024, [&](unsigned n, int64_t t0) { k_norm_back_long<BF><<<dim3(n, (unsigned)s->K), 1024, 0, st>>>(dy, x, w, stats, add, dx, t0, T, d); }); \
    } while (0)
        if (s->dtype == GRAWA_BF16) GRAWA_NORM_FORMS(GO, GOLONG, true);
        else GRAWA_NORM_FORMS(GO, GOLONG, false);
#undef GO
#undef GOLONG
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 sums((unsigned)((d + 63) / 64), (unsigned)s->K, 2);
    if (s->dtype == GRAWA_BF16)
        k_norm_sums<true><<<sums, 1024, 0, st>>>(part, nb, dw, db, accumulate, d);
    else
        k_norm_sums<false><<<sums, 1024, 0, st>>>(part, nb, dw, db, accumulate, d);
    return hipGetLastError();
}
