// Host side of the feed-forward sublayer's entry points (include/grawa.h): argument checks, the plan and its workspace.  The
// operators run in the kernels of grawa_layernorm.hip, grawa_dropout.hip and grawa_ffn.hip.
#include <cmath>
#include <cstring>
#include <new>

#include "grawa_sublayer.h"

namespace {

constexpr int64_t MAX_WIDTH = (int64_t)1 << 20, MAX_TOKENS = (int64_t)1 << 30;

struct OnDevice { // the plan's kernels run on the device the plan was made on
    int prev = -1;
    bool ok = true;
    explicit OnDevice(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess || (prev != dev && hipSetDevice(dev) != hipSuccess)) ok = false;
    }
    ~OnDevice()
    {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }
inline int64_t element(grawa_dtype_t dt) { return dt == GRAWA_BF16 ? 2 : 4; }

grawa_status_t check_shape(int K, int64_t T, int64_t d, int64_t f, grawa_dtype_t dt)
{
    if (K < 1 || T < 0 || d < 1 || f < 0) return GRAWA_ERR_INVALID_ARG;
    if (dt != GRAWA_F32 && dt != GRAWA_BF16) return GRAWA_ERR_UNSUPPORTED;
    if (K > GRAWA_MAX_WORKERS || T > MAX_TOKENS / K || d >= MAX_WIDTH || f >= MAX_WIDTH) return GRAWA_ERR_UNSUPPORTED;
    return GRAWA_OK;
}

// Strides whose products with the counts stay far from 63 bits, element alignment; outputs with rows that do not overlap.
grawa_status_t check_rows(const grawa_rows_t *r, int K, int64_t T, int64_t width, grawa_dtype_t dt, bool out, GrawaRows &v)
{
    if (!r || (!r->data && T > 0) || r->worker < 0 || r->row < 0) return GRAWA_ERR_INVALID_ARG;
    if (r->worker >= ((int64_t)1 << 48) || r->row >= ((int64_t)1 << 30)) return GRAWA_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(r->data) % element(dt)) return GRAWA_ERR_ALIGNMENT;
    if (out && T > 0) { // workers apart and rows apart inside, or the other way round
        const bool rows_inside = (T == 1 || r->row >= width) && (K == 1 || r->worker >= (T - 1) * r->row + width);
        const bool workers_inside = (K == 1 || r->worker >= width) && (T == 1 || r->row >= (K - 1) * r->worker + width);
        if (!rows_inside && !workers_inside) return GRAWA_ERR_INVALID_ARG;
    }
    v = GrawaRows{static_cast<char *>(r->data), r->worker, r->row};
    return GRAWA_OK;
}

grawa_status_t check_mats(const grawa_mats_t *m, int K, int64_t n, grawa_dtype_t dt, bool out, GrawaMat &v)
{
    if (!m || !m->data || m->worker < 0) return GRAWA_ERR_INVALID_ARG;
    if (m->worker >= ((int64_t)1 << 48)) return GRAWA_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(m->data) % element(dt)) return GRAWA_ERR_ALIGNMENT;
    if (out && K > 1 && m->worker < n) return GRAWA_ERR_INVALID_ARG;
    v = GrawaMat{static_cast<char *>(m->data), m->worker};
    return GRAWA_OK;
}

grawa_status_t check_drop(float p, const int64_t *rng, uint32_t site, GrawaDrop &d)
{
    if (!std::isfinite(p) || p < 0.f || p >= 1.f) return GRAWA_ERR_INVALID_ARG;
    const uint32_t threshold = (uint32_t)((double)p * 4294967296.0);
    if (p > 0.f && !rng) return GRAWA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(rng) % 8) return GRAWA_ERR_ALIGNMENT;
    d = GrawaDrop{reinterpret_cast<const uint64_t *>(rng), threshold, site, (float)(1.0 / (1.0 - (double)p))};
    return GRAWA_OK;
}

grawa_status_t check_tokens(const grawa_sublayer *s, int64_t T)
{
    return !s || T < 0 || T > s->T ? GRAWA_ERR_INVALID_ARG : GRAWA_OK;
}

inline grawa_status_t status_of(hipError_t e) { return e == hipSuccess ? GRAWA_OK : GRAWA_ERR_HIP; }

#define GRAWA_TRY(expr)                            \
    do {                                           \
        const grawa_status_t st_ = (expr);         \
        if (st_ != GRAWA_OK) return st_;           \
    } while (0)

} // namespace

extern "C" {

grawa_status_t grawa_sublayer_create(grawa_sublayer_t **out, int K, int64_t T, int64_t d, int64_t f, grawa_dtype_t dtype, grawa_act_t act)
{
    if (!out) return GRAWA_ERR_INVALID_ARG;
    *out = nullptr;
    GRAWA_TRY(check_shape(K, T, d, f, dtype));
    if (act != GRAWA_ACT_SILU && act != GRAWA_ACT_GELU && act != GRAWA_ACT_RELU) return GRAWA_ERR_INVALID_ARG;
    grawa_sublayer *s = new (std::nothrow) grawa_sublayer();
    if (!s) return GRAWA_ERR_WORKSPACE;
    std::memset(s, 0, sizeof(*s));
    s->K = K;
    s->T = T;
    s->d = d;
    s->f = f;
    s->dp = grawa_round64(d);
    s->fp = grawa_round64(f);
    s->dtype = dtype;
    s->act = act;
    s->planes = dtype == GRAWA_BF16 ? 1 : 3;
    s->norm_blocks = grawa_norm_blocks(K, T, d);
    if (hipGetDevice(&s->device) != hipSuccess) {
        delete s;
        return GRAWA_ERR_HIP;
    }
    // Everything below fits 63 bits: K <= 2^10, T K <= 2^30, widths < 2^20.
    const size_t plane = (size_t)s->planes * (size_t)K * 2;
    const size_t b_norm = round256((size_t)K * (size_t)s->norm_blocks * 2 * (size_t)d * 4);
    const size_t b_tok = f ? round256(plane * (size_t)T * (size_t)s->dp) : 0, b_inner = f ? round256(plane * (size_t)T * (size_t)s->fp) : 0;
    const size_t b_up = f ? round256(plane * (size_t)f * (size_t)s->dp) : 0, b_down = f ? round256(plane * (size_t)d * (size_t)s->fp) : 0;
    s->part_floats = f ? grawa_ffn_part_floats(s) : 0;
    const size_t b_part = round256((size_t)s->part_floats * 4);
    if (hipMalloc(&s->ws, b_norm + 2 * b_tok + 3 * b_inner + 2 * b_up + b_down + b_part) != hipSuccess) {
        (void)hipGetLastError();
        delete s;
        return GRAWA_ERR_WORKSPACE;
    }
    char *p = s->ws;
    auto carve = [&](size_t n) { char *at = p; p += n; return at; };
    s->norm_part = (float *)carve(b_norm);
    s->x = carve(b_tok);
    s->dy = carve(b_tok);
    s->h = carve(b_inner);
    s->dg = carve(b_inner);
    s->du = carve(b_inner);
    s->wg = carve(b_up);
    s->wu = carve(b_up);
    s->wd = carve(b_down);
    s->part = (float *)carve(b_part);
    *out = s;
    return GRAWA_OK;
}

grawa_status_t grawa_sublayer_destroy(grawa_sublayer_t *s)
{
    if (!s) return GRAWA_OK;
    grawa_status_t r = GRAWA_OK;
    {
        OnDevice dev(s->device);
        if (!dev.ok || hipFree(s->ws) != hipSuccess) r = GRAWA_ERR_HIP;
    }
    delete s;
    return r;
}

grawa_status_t grawa_sublayer_save_bytes(const grawa_sublayer_t *s, int64_t T, int64_t *bytes)
{
    GRAWA_TRY(check_tokens(s, T));
    if (!bytes || !s->f) return GRAWA_ERR_INVALID_ARG;
    *bytes = grawa_save_bytes(s, T);
    return GRAWA_OK;
}

grawa_status_t grawa_layer_norm(grawa_sublayer_t *s, int64_t T, const grawa_rows_t *x, const grawa_mats_t *weight, const grawa_mats_t *bias,
                                float eps, const grawa_rows_t *y, float *stats, void *stream)
{
    GRAWA_TRY(check_tokens(s, T));
    if (!std::isfinite(eps) || eps < 0.f) return GRAWA_ERR_INVALID_ARG;
    GrawaRows vx, vy;
    GrawaMat vw, vb{};
    GRAWA_TRY(check_rows(x, s->K, T, s->d, s->dtype, false, vx));
    GRAWA_TRY(check_rows(y, s->K, T, s->d, s->dtype, true, vy));
    GRAWA_TRY(check_mats(weight, s->K, s->d, s->dtype, false, vw));
    if (bias) GRAWA_TRY(check_mats(bias, s->K, s->d, s->dtype, false, vb));
    if (reinterpret_cast<uintptr_t>(stats) % 8) return GRAWA_ERR_ALIGNMENT;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_layer_norm(s, T, vx, vw, vb, eps, vy, stats, static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_layer_norm_backward(grawa_sublayer_t *s, int64_t T, const grawa_rows_t *dy, const grawa_rows_t *x, const grawa_mats_t *weight,
                                         const float *stats, const grawa_rows_t *add, const grawa_rows_t *dx, const grawa_mats_t *dweight,
                                         const grawa_mats_t *dbias, int accumulate, void *stream)
{
    GRAWA_TRY(check_tokens(s, T));
    GrawaRows vdy, vx, vadd{}, vdx;
    GrawaMat vw, vdw, vdb{};
    GRAWA_TRY(check_rows(dy, s->K, T, s->d, s->dtype, false, vdy));
    GRAWA_TRY(check_rows(x, s->K, T, s->d, s->dtype, false, vx));
    if (add) GRAWA_TRY(check_rows(add, s->K, T, s->d, s->dtype, false, vadd));
    GRAWA_TRY(check_rows(dx, s->K, T, s->d, s->dtype, true, vdx));
    GRAWA_TRY(check_mats(weight, s->K, s->d, s->dtype, false, vw));
    GRAWA_TRY(check_mats(dweight, s->K, s->d, s->dtype, true, vdw));
    if (dbias) GRAWA_TRY(check_mats(dbias, s->K, s->d, s->dtype, true, vdb));
    if (!stats && T > 0) return GRAWA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(stats) % 8) return GRAWA_ERR_ALIGNMENT;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_layer_norm_backward(s, T, vdy, vx, vw, stats, vadd, vdx, vdw, vdb, accumulate ? 1 : 0, static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_ffn(grawa_sublayer_t *s, int64_t T, const grawa_rows_t *x, const grawa_mats_t *wg, const grawa_mats_t *wu, const grawa_mats_t *wd,
                         const grawa_rows_t *residual, float p, const int64_t *rng, uint32_t site, const grawa_rows_t *y, void *save, void *stream)
{
    GRAWA_TRY(check_tokens(s, T));
    if (!s->f) return GRAWA_ERR_INVALID_ARG;
    GrawaRows vx, vy, vr{};
    GrawaMat vg, vu, vd;
    GrawaDrop drop;
    GRAWA_TRY(check_rows(x, s->K, T, s->d, s->dtype, false, vx));
    GRAWA_TRY(check_rows(y, s->K, T, s->d, s->dtype, true, vy));
    if (residual) GRAWA_TRY(check_rows(residual, s->K, T, s->d, s->dtype, false, vr));
    GRAWA_TRY(check_mats(wg, s->K, s->d * s->f, s->dtype, false, vg));
    GRAWA_TRY(check_mats(wu, s->K, s->d * s->f, s->dtype, false, vu));
    GRAWA_TRY(check_mats(wd, s->K, s->d * s->f, s->dtype, false, vd));
    GRAWA_TRY(check_drop(p, rng, site, drop));
    if (reinterpret_cast<uintptr_t>(save) % 16) return GRAWA_ERR_ALIGNMENT;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_ffn(s, T, vx, vg, vu, vd, vr, drop, vy, static_cast<char *>(save), static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_ffn_backward(grawa_sublayer_t *s, int64_t T, const grawa_rows_t *dy, const grawa_rows_t *x, const grawa_mats_t *wg,
                                  const grawa_mats_t *wu, const grawa_mats_t *wd, const void *save, const grawa_rows_t *dx, const grawa_mats_t *dwg,
                                  const grawa_mats_t *dwu, const grawa_mats_t *dwd, int accumulate, void *stream)
{
    GRAWA_TRY(check_tokens(s, T));
    if (!s->f) return GRAWA_ERR_INVALID_ARG;
    GrawaRows vdy, vx, vdx;
    GrawaMat vg, vu, vd, gg, gu, gd;
    const int64_t n = s->d * s->f;
    GRAWA_TRY(check_rows(dy, s->K, T, s->d, s->dtype, false, vdy));
    GRAWA_TRY(check_rows(x, s->K, T, s->d, s->dtype, false, vx));
    GRAWA_TRY(check_rows(dx, s->K, T, s->d, s->dtype, true, vdx));
    GRAWA_TRY(check_mats(wg, s->K, n, s->dtype, false, vg));
    GRAWA_TRY(check_mats(wu, s->K, n, s->dtype, false, vu));
    GRAWA_TRY(check_mats(wd, s->K, n, s->dtype, false, vd));
    GRAWA_TRY(check_mats(dwg, s->K, n, s->dtype, true, gg));
    GRAWA_TRY(check_mats(dwu, s->K, n, s->dtype, true, gu));
    GRAWA_TRY(check_mats(dwd, s->K, n, s->dtype, true, gd));
    if (!save && T > 0) return GRAWA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(save) % 16) return GRAWA_ERR_ALIGNMENT;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_ffn_backward(s, T, vdy, vx, vg, vu, vd, static_cast<const char *>(save), vdx, gg, gu, gd, accumulate ? 1 : 0, static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_dropout(int K, int64_t T, int64_t d, grawa_dtype_t dtype, const grawa_rows_t *x, const grawa_rows_t *residual, float p,
                             const int64_t *rng, uint32_t site, const grawa_rows_t *y, void *stream)
{
    GRAWA_TRY(check_shape(K, T, d, 0, dtype));
    GrawaRows vx, vy, vr{};
    GrawaDrop drop;
    GRAWA_TRY(check_rows(x, K, T, d, dtype, false, vx));
    GRAWA_TRY(check_rows(y, K, T, d, dtype, true, vy));
    if (residual) GRAWA_TRY(check_rows(residual, K, T, d, dtype, false, vr));
    GRAWA_TRY(check_drop(p, rng, site, drop));
    return status_of(grawa_launch_dropout(K, T, d, dtype, vx, vr, drop, vy, static_cast<hipStream_t>(stream)));
}

} // extern "C"
