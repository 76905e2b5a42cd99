// Dropout with a mask that is made from a counter each time it is needed, and the residual sum that goes with it:
//   y = residual + keep(x) / (1 - p)
// The backward pass is the same call on dy without a residual.  The bound is memory, two or three arrays of K T d elements; just below it
// stands the counter's function, 28 products of 32 by 32 bits for four elements, about 20 us of the vector units for 8 x 4096 x 1024.
// Both passes of that size in bfloat16, 335 MB: 62 us, 5.4 TB/s, when other data has passed through the caches in between, 55 us when not.
// Results are stored past the caches: 58 us against 67; what reads them next did not get slower for it.
#include "grawa_elements.h"
#include "grawa_sublayer.h"

namespace {

// A thread takes eight columns of a row, two counters.  Blocks walk a worker's rows in y, the row's columns in x.
template <bool BF16, bool RES>
__global__ __launch_bounds__(256) void k_dropout(GrawaRows x, GrawaRows res, GrawaDrop drop, GrawaRows y, uint32_t T, uint32_t d, uint32_t lanes)
{
    constexpr int S = BF16 ? 2 : 4, P = 8 / GrawaPiece<BF16>::N;
    const GrawaDropKey key = drop.threshold ? grawa_drop_key(drop) : GrawaDropKey{0, 0, 0};
    // `lanes` (a power of two) threads side by side in a row
    const uint32_t col = (blockIdx.x * lanes + (threadIdx.x & (lanes - 1))) * 8, per = 256 / lanes;
    if (col >= d) return;
    const int left = (int)(d - col);
    const uint32_t k = blockIdx.z;
    for (uint32_t t = blockIdx.y * per + threadIdx.x / lanes; t < T; t += gridDim.y * per) {
        const char *px = x.p + ((int64_t)k * x.worker + (int64_t)t * x.row + col) * S;
        const char *pr = RES ? res.p + ((int64_t)k * res.worker + (int64_t)t * res.row + col) * S : nullptr;
        char *py = y.p + ((int64_t)k * y.worker + (int64_t)t * y.row + col) * S;
        GrawaPiece<BF16> a[P], r[P] = {};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int n = left - i * GrawaPiece<BF16>::N;
            if (n <= 0) break;
            a[i].load(px + 16 * i, n);
            if (RES) r[i].load(pr + 16 * i, n);
        }
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = a[j / GrawaPiece<BF16>::N][j % GrawaPiece<BF16>::N];
        if (drop.threshold) {
            grawa_drop4(drop, key, k * T + t, col / 4, v);
            grawa_drop4(drop, key, k * T + t, col / 4 + 1, v + 4);
        }
        if (RES)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += r[j / GrawaPiece<BF16>::N][j % GrawaPiece<BF16>::N];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int n = left - i * GrawaPiece<BF16>::N;
            if (n > 0) store_piece<BF16, true>(py + 16 * i, n, v + i * GrawaPiece<BF16>::N);
        }
    }
}

} // namespace

hipError_t grawa_launch_dropout(int K, int64_t T, int64_t d, grawa_dtype_t dtype, GrawaRows x, GrawaRows residual, GrawaDrop drop,
                                GrawaRows y, hipStream_t st)
{
    const int64_t groups = (d + 7) / 8;
    if (!T) return hipSuccess;
    uint32_t lanes = 1;
    while (lanes < 256 && lanes < groups) lanes *= 2;
    const int64_t across = (groups + lanes - 1) / lanes, down = (T + 256 / lanes - 1) / (256 / lanes);
    // A block for every row group up to what fills the card many times over; beyond, blocks walk on.
    const int64_t most = across * K < 65535 ? 65535 / (across * K) : 1;
    const dim3 grid((unsigned)across, (unsigned)(down < most ? down : most), (unsigned)K);
#define GO(B, R) k_dropout<B, R><<<grid, 256, 0, st>>>(x, residual, drop, y, (uint32_t)T, (uint32_t)d, lanes)
    if (dtype == GRAWA_BF16) {
        if (residual.p) GO(true, true);
        else GO(true, false);
    } else {
        if (residual.p) GO(false, true);
        else GO(false, false);
    }
#undef GO
    return hipGetLastError();
}
