// Dropout with a mask that is made from a counter each time it is needed, and the residual sum that goes with it:
//   y = residual + keep(x) / (1 - p)
// The backward pass is the same call on dy without a residual.  The bound is memory: two or three arrays of K T d elements.
#include "grawa_elements.h"
#include "grawa_sublayer.h"

namespace {

// A thread takes eight columns of a row, two counters.  WIDE: every row starts on a 16-byte boundary and d is a multiple of 8.
template <bool BF16, bool WIDE, bool RES>
__global__ __launch_bounds__(256) void k_dropout(GrawaRows x, GrawaRows res, GrawaDrop drop, GrawaRows y, uint32_t T, uint32_t d,
                                                 uint32_t groups, uint64_t total)
{
    constexpr int S = BF16 ? 2 : 4;
    const GrawaDropKey key = drop.threshold ? grawa_drop_key(drop) : GrawaDropKey{0, 0, 0};
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)(i / groups), col = (uint32_t)(i - (uint64_t)row * groups) * 8;
        const uint32_t k = row / T, t = row - k * T;
        const char *px = x.p + ((int64_t)k * x.worker + (int64_t)t * x.row) * S;
        const char *pr = RES ? res.p + ((int64_t)k * res.worker + (int64_t)t * res.row) * S : nullptr;
        char *py = y.p + ((int64_t)k * y.worker + (int64_t)t * y.row) * S;
        const int n = WIDE ? 8 : (int)(d - col < 8 ? d - col : 8);
        float v[8] = {}, r[8] = {};
        if (WIDE) {
            load_elements<BF16, 8>(px + (int64_t)col * S, v);
            if (RES) load_elements<BF16, 8>(pr + (int64_t)col * S, r);
        } else {
            for (int j = 0; j < n; ++j) {
                load_elements<BF16, 1>(px + (int64_t)(col + j) * S, v + j);
                if (RES) load_elements<BF16, 1>(pr + (int64_t)(col + j) * S, r + j);
            }
        }
        if (drop.threshold) {
            grawa_drop4(drop, key, row, col / 4, v);
            grawa_drop4(drop, key, row, col / 4 + 1, v + 4);
        }
        if (RES)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += r[j];
        if (WIDE)
            store_elements<BF16, 8>(py + (int64_t)col * S, v);
        else
            for (int j = 0; j < n; ++j) store_elements<BF16, 1>(py + (int64_t)(col + j) * S, v + j);
    }
}

bool aligned(const GrawaRows &r, int S) { return !(((uintptr_t)r.p | (uint64_t)r.worker * S | (uint64_t)r.row * S) & 15); }

} // namespace

hipError_t grawa_launch_dropout(int K, int64_t T, int64_t d, grawa_dtype_t dtype, GrawaRows x, GrawaRows residual, GrawaDrop drop,
                                GrawaRows y, hipStream_t st)
{
    const bool bf = dtype == GRAWA_BF16;
    const int S = bf ? 2 : 4;
    const bool wide = d % 8 == 0 && aligned(x, S) && aligned(y, S) && (!residual.p || aligned(residual, S));
    const uint64_t groups = (uint64_t)(d + 7) / 8, total = (uint64_t)K * T * groups;
    if (!total) return hipSuccess;
    const uint64_t want = (total + 255) / 256;
    const dim3 grid((unsigned)(want < 16384 ? want : 16384));
#define GO(B, W, R) k_dropout<B, W, R><<<grid, 256, 0, st>>>(x, residual, drop, y, (uint32_t)T, (uint32_t)d, (uint32_t)groups, total)
    if (residual.p) {
        if (bf) { if (wide) GO(true, true, true); else GO(true, false, true); }
        else { if (wide) GO(false, true, true); else GO(false, false, true); }
    } else {
        if (bf) { if (wide) GO(true, true, false); else GO(true, false, false); }
        else { if (wide) GO(false, true, false); else GO(false, false, false); }
    }
#undef GO
    return hipGetLastError();
}
