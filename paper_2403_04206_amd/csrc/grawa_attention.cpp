// Host side of the attention's entry points (include/grawa.h): argument checks, the plan, its tables and workspace.  The operators run
// in the kernels of grawa_heads.hip, grawa_attend.hip and grawa_attend_back.hip.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "grawa_attention.h"

namespace {

constexpr int64_t PART_FLOATS = (int64_t)16 << 20;

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

grawa_status_t check_shape(const grawa_attention_shape_t *s)
{
    if (!s || s->K < 1 || s->sequences < 0 || s->length < 0 || s->heads < 1 || s->kv_heads < 1 || s->width < 1) return GRAWA_ERR_INVALID_ARG;
    if (s->heads % s->kv_heads || s->window < 0 || s->sinks < 0 || !std::isfinite(s->scale) || s->scale <= 0.f) return GRAWA_ERR_INVALID_ARG;
    if (s->rotary < 0 || s->rotary % 2 || s->rotary > s->width || (s->rotary && !s->frequencies)) return GRAWA_ERR_INVALID_ARG;
    if (s->buckets < 0 || (s->buckets && (s->distances < 1 || !s->bucket_of))) return GRAWA_ERR_INVALID_ARG;
    if (s->dtype != GRAWA_F32 && s->dtype != GRAWA_BF16) return GRAWA_ERR_UNSUPPORTED;
    if (s->K > GRAWA_MAX_WORKERS || s->width % 8 || s->width > 128 || s->buckets > GRAWA_MAX_BUCKETS) return GRAWA_ERR_UNSUPPORTED;
    if (s->buckets && s->distances > GRAWA_MAX_DISTANCES) return GRAWA_ERR_UNSUPPORTED;
    const int64_t heads = (int64_t)1 << 20, rows = (int64_t)1 << 30;
    if (s->heads > heads || s->sequences > heads / s->heads / s->K) return GRAWA_ERR_UNSUPPORTED;
    const int64_t knh = std::max<int64_t>(s->sequences, 1) * s->heads * s->K;
    if (s->length > rows / knh || s->length > (int64_t)1 << 28) return GRAWA_ERR_UNSUPPORTED; // positions and windows add up in 32 bits
    for (int i = 0; i < s->rotary / 2; ++i)
        if (!std::isfinite(s->frequencies[i])) return GRAWA_ERR_INVALID_ARG;
    for (int64_t i = 0; s->buckets && i < s->distances; ++i)
        if (s->bucket_of[i] < 0 || s->bucket_of[i] >= s->buckets) return GRAWA_ERR_INVALID_ARG;
    return GRAWA_OK;
}

// Rows that lie within 2^56 elements of the first one, so that no address passes 63 bits (heads of keys are counted from the H of queries on,
// which 2^20 times a stride of 2^40 elements still allows); outputs with rows that do not overlap, whatever the order of the axes.  By
// tiles: what the attention's loads ask for.
grawa_status_t check_heads(const grawa_attention_plan *s, const grawa_heads_t *r, int64_t N, int64_t S, int heads, bool tiles, bool out, GrawaHeads &v)
{
    if (!r) return GRAWA_ERR_INVALID_ARG;
    const int64_t counts[4] = {s->K, N, S, heads}, es = element(s->dtype), limit = (int64_t)1 << 40;
    int64_t strides[4] = {r->worker, r->sequence, r->token, r->head}, room = (int64_t)1 << 56;
    for (int i = 0; i < 4; ++i) {
        if (strides[i] < 0) return GRAWA_ERR_INVALID_ARG;
        if (counts[i] <= 1) strides[i] = 0;
    }
    for (int i = 0; i < 4; ++i) {
        if (strides[i] >= limit || (counts[i] > 1 && strides[i] > room / (counts[i] - 1))) return GRAWA_ERR_UNSUPPORTED;
        if (counts[i] > 1) room -= strides[i] * (counts[i] - 1);
    }
    v = GrawaHeads{static_cast<char *>(r->data), strides[0] * es, strides[1] * es, strides[2] * es, strides[3] * es};
    if (N == 0 || S == 0) return GRAWA_OK; // no row is looked at
    if (!r->data) return GRAWA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(r->data) % es) return GRAWA_ERR_ALIGNMENT;
    if (tiles) {
        if (reinterpret_cast<uintptr_t>(r->data) % 16 || (v.worker | v.seq | v.token | v.head) % 16) return GRAWA_ERR_ALIGNMENT;
        if (v.token >= (int64_t)1 << 24) return GRAWA_ERR_UNSUPPORTED;
    }
    if (out) {
        int axes[4] = {0, 1, 2, 3};
        std::sort(axes, axes + 4, [&](int a, int b) { return strides[a] < strides[b]; });
        int64_t extent = s->D;
        for (int a : axes) {
            if (counts[a] <= 1) continue;
            if (strides[a] < extent) return GRAWA_ERR_INVALID_ARG;
            extent += strides[a] * (counts[a] - 1);
        }
    }
    return GRAWA_OK;
}

grawa_status_t check_mats(const grawa_attention_plan *s, const grawa_mats_t *m, int64_t n, bool out, GrawaMat &v)
{
    if (!m || !m->data || m->worker < 0) return GRAWA_ERR_INVALID_ARG;
    if (m->worker >= ((int64_t)1 << 48)) return GRAWA_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(m->data) % element(s->dtype)) return GRAWA_ERR_ALIGNMENT;
    if (out && s->K > 1 && m->worker < n) return GRAWA_ERR_INVALID_ARG;
    v = GrawaMat{static_cast<char *>(m->data), m->worker};
    return GRAWA_OK;
}

grawa_status_t check_counts(const grawa_attention_plan *s, int64_t N, int64_t Sq, int64_t Sk)
{
    if (!s || N < 0 || Sq < 0 || Sk < 0 || N > s->N || Sq > s->S || Sk > s->S) return GRAWA_ERR_INVALID_ARG;
    return GRAWA_OK;
}

grawa_status_t check_words(const void *a, const void *b = nullptr)
{
    return (reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % 4 ? GRAWA_ERR_ALIGNMENT : GRAWA_OK;
}

inline grawa_status_t status_of(hipError_t e) { return e == hipSuccess ? GRAWA_OK : GRAWA_ERR_HIP; }

#define GRAWA_TRY(expr)                            \
    do {                                           \
        const grawa_status_t st_ = (expr);         \
        if (st_ != GRAWA_OK) return st_;           \
    } while (0)

// What both directions of the attention have.
grawa_status_t fill(const grawa_attention_plan *s, int64_t N, int64_t Sq, int64_t Sk, const grawa_heads_t *q, const grawa_heads_t *k,
                    const grawa_heads_t *v, const grawa_mats_t *bias, const int32_t *lengths, const int32_t *starts, GrawaAttend &a)
{
    GRAWA_TRY(check_counts(s, N, Sq, Sk));
    GRAWA_TRY(check_heads(s, q, N, Sq, s->H, true, false, a.q));
    GRAWA_TRY(check_heads(s, k, N, Sk, s->G, true, false, a.k));
    GRAWA_TRY(check_heads(s, v, N, Sk, s->G, true, false, a.v));
    if ((bias != nullptr) != (s->buckets > 0)) return GRAWA_ERR_INVALID_ARG;
    if (bias) GRAWA_TRY(check_mats(s, bias, (int64_t)s->H * s->buckets, false, a.bias));
    GRAWA_TRY(check_words(lengths, starts));
    a.lengths = lengths;
    a.starts = starts;
    a.bucket_of = s->bucket_of;
    a.row_pitch = grawa_round256(Sq);
    a.row_lse = s->rows;
    a.row_dot = s->rows + (int64_t)s->K * N * s->H * a.row_pitch;
    a.bias_part = s->bias_part;
    a.part = s->part;
    a.K = s->K, a.N = (int)N, a.H = s->H, a.G = s->G, a.D = s->D, a.Sq = (int)Sq, a.Sk = (int)Sk, a.share = s->H / s->G;
    a.window = s->window, a.sinks = s->sinks, a.buckets = s->buckets, a.distances = s->distances;
    a.scale = s->scale;
    return GRAWA_OK;
}

} // namespace

extern "C" {

grawa_status_t grawa_attention_create(grawa_attention_plan_t **out, const grawa_attention_shape_t *shape)
{
    if (!out) return GRAWA_ERR_INVALID_ARG;
    *out = nullptr;
    GRAWA_TRY(check_shape(shape));
    grawa_attention_plan *s = new (std::nothrow) grawa_attention_plan();
    if (!s) return GRAWA_ERR_WORKSPACE;
    std::memset(s, 0, sizeof(*s));
    s->K = shape->K;
    s->N = shape->sequences;
    s->S = shape->length;
    s->H = shape->heads;
    s->G = shape->kv_heads;
    s->D = shape->width;
    s->dtype = shape->dtype;
    s->scale = shape->scale;
    s->window = shape->window > 0 && shape->window < GRAWA_NO_WINDOW ? (int)shape->window : GRAWA_NO_WINDOW;
    s->sinks = (int)std::min<int64_t>(shape->sinks, GRAWA_NO_WINDOW);
    s->rotary = shape->rotary;
    s->interleaved = shape->interleaved ? 1 : 0;
    s->buckets = shape->buckets;
    s->distances = shape->buckets ? (int)shape->distances : 0;
    s->norm_blocks = grawa_head_norm_blocks(s);
    if (hipGetDevice(&s->device) != hipSuccess) {
        delete s;
        return GRAWA_ERR_HIP;
    }
    // Everything below fits 63 bits: K N H <= 2^20, K N H S <= 2^30.
    const int64_t knh = (int64_t)s->K * s->N * s->H;
    s->part_floats = std::min<int64_t>(PART_FLOATS, 64 * (int64_t)s->K * s->N * (s->H + 2 * s->G) * grawa_round256(s->S) * grawa_padded_width(s->D));
    const size_t b_turns = round256((size_t)s->rotary / 2 * sizeof(double)), b_bucket = round256((size_t)s->distances * sizeof(int));
    const size_t b_rows = round256((size_t)knh * (size_t)grawa_round256(s->S) * 2 * sizeof(float));
    const size_t b_norm = round256((size_t)s->K * (size_t)s->norm_blocks * 2 * (size_t)s->D * sizeof(float));
    const int block = grawa_dq_queries(s->dtype == GRAWA_BF16);
    const size_t b_bias = round256((size_t)knh * (size_t)((s->S + block - 1) / block) * (size_t)s->buckets * sizeof(float));
    const size_t b_part = round256((size_t)s->part_floats * sizeof(float));
    if (hipMalloc(&s->ws, b_turns + b_bucket + b_rows + b_norm + b_bias + b_part) != hipSuccess) {
        (void)hipGetLastError();
        delete s;
        return GRAWA_ERR_WORKSPACE;
    }
    char *p = s->ws;
    auto carve = [&](size_t n) { char *at = p; p += n; return at; };
    s->turns = (double *)carve(b_turns);
    s->bucket_of = (int *)carve(b_bucket);
    s->rows = (float *)carve(b_rows);
    s->norm_part = (float *)carve(b_norm);
    s->bias_part = (float *)carve(b_bias);
    s->part = (float *)carve(b_part);
    double turns[64];
    for (int i = 0; i < s->rotary / 2; ++i) turns[i] = (double)((long double)shape->frequencies[i] / 6.283185307179586476925286766559L);
    if ((s->rotary && hipMemcpy(s->turns, turns, (size_t)s->rotary / 2 * sizeof(double), hipMemcpyHostToDevice) != hipSuccess) ||
        (s->distances && hipMemcpy(s->bucket_of, shape->bucket_of, (size_t)s->distances * sizeof(int), hipMemcpyHostToDevice) != hipSuccess)) {
        (void)hipGetLastError();
        (void)hipFree(s->ws);
        delete s;
        return GRAWA_ERR_HIP;
    }
    *out = s;
    return GRAWA_OK;
}

grawa_status_t grawa_attention_destroy(grawa_attention_plan_t *s)
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

grawa_status_t grawa_head_norm(grawa_attention_plan_t *s, int64_t N, int64_t S, const grawa_heads_t *q, const grawa_heads_t *k,
                               const grawa_mats_t *qweight, const grawa_mats_t *kweight, float eps, const int32_t *starts,
                               const grawa_heads_t *q_out, const grawa_heads_t *k_out, void *stream)
{
    GRAWA_TRY(check_counts(s, N, S, S));
    if (!std::isfinite(eps) || eps < 0.f) return GRAWA_ERR_INVALID_ARG;
    GrawaHeads vq, vk, vqo, vko;
    GrawaMat wq, wk;
    GRAWA_TRY(check_heads(s, q, N, S, s->H, false, false, vq));
    GRAWA_TRY(check_heads(s, k, N, S, s->G, false, false, vk));
    GRAWA_TRY(check_heads(s, q_out, N, S, s->H, false, true, vqo));
    GRAWA_TRY(check_heads(s, k_out, N, S, s->G, false, true, vko));
    GRAWA_TRY(check_mats(s, qweight, s->D, false, wq));
    GRAWA_TRY(check_mats(s, kweight, s->D, false, wk));
    GRAWA_TRY(check_words(starts));
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_head_norm(s, N, S, vq, vk, wq, wk, eps, starts, vqo, vko, static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_head_norm_backward(grawa_attention_plan_t *s, int64_t N, int64_t S, const grawa_heads_t *dq_out, const grawa_heads_t *dk_out,
                                        const grawa_heads_t *q, const grawa_heads_t *k, const grawa_mats_t *qweight, const grawa_mats_t *kweight,
                                        float eps, const int32_t *starts, const grawa_heads_t *dq, const grawa_heads_t *dk,
                                        const grawa_mats_t *dqweight, const grawa_mats_t *dkweight, int accumulate, void *stream)
{
    GRAWA_TRY(check_counts(s, N, S, S));
    if (!std::isfinite(eps) || eps < 0.f) return GRAWA_ERR_INVALID_ARG;
    GrawaHeads vdqo, vdko, vq, vk, vdq, vdk;
    GrawaMat wq, wk, gq, gk;
    GRAWA_TRY(check_heads(s, dq_out, N, S, s->H, false, false, vdqo));
    GRAWA_TRY(check_heads(s, dk_out, N, S, s->G, false, false, vdko));
    GRAWA_TRY(check_heads(s, q, N, S, s->H, false, false, vq));
    GRAWA_TRY(check_heads(s, k, N, S, s->G, false, false, vk));
    GRAWA_TRY(check_heads(s, dq, N, S, s->H, false, true, vdq));
    GRAWA_TRY(check_heads(s, dk, N, S, s->G, false, true, vdk));
    GRAWA_TRY(check_mats(s, qweight, s->D, false, wq));
    GRAWA_TRY(check_mats(s, kweight, s->D, false, wk));
    GRAWA_TRY(check_mats(s, dqweight, s->D, true, gq));
    GRAWA_TRY(check_mats(s, dkweight, s->D, true, gk));
    GRAWA_TRY(check_words(starts));
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_head_norm_backward(s, N, S, vdqo, vdko, vq, vk, wq, wk, eps, starts, vdq, vdk, gq, gk, accumulate ? 1 : 0,
                                                     static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_attention(grawa_attention_plan_t *s, int64_t N, int64_t Sq, int64_t Sk, const grawa_heads_t *q, const grawa_heads_t *k,
                               const grawa_heads_t *v, const grawa_mats_t *bias, const int32_t *lengths, const int32_t *starts,
                               const grawa_heads_t *o, float *lse, void *stream)
{
    GrawaAttend a{};
    GRAWA_TRY(fill(s, N, Sq, Sk, q, k, v, bias, lengths, starts, a));
    GRAWA_TRY(check_heads(s, o, N, Sq, s->H, true, true, a.o));
    GRAWA_TRY(check_words(lse));
    a.lse = lse;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_attend(s, a, static_cast<hipStream_t>(stream)));
}

grawa_status_t grawa_attention_backward(grawa_attention_plan_t *s, int64_t N, int64_t Sq, int64_t Sk, const grawa_heads_t *d_o, const grawa_heads_t *q,
                                        const grawa_heads_t *k, const grawa_heads_t *v, const grawa_mats_t *bias, const int32_t *lengths,
                                        const int32_t *starts, const grawa_heads_t *o, const float *lse, const grawa_heads_t *dq,
                                        const grawa_heads_t *dk, const grawa_heads_t *dv, const grawa_mats_t *dbias, int accumulate, void *stream)
{
    GrawaAttend a{};
    GRAWA_TRY(fill(s, N, Sq, Sk, q, k, v, bias, lengths, starts, a));
    GRAWA_TRY(check_heads(s, d_o, N, Sq, s->H, true, false, a.go));
    GRAWA_TRY(check_heads(s, o, N, Sq, s->H, true, false, a.o));
    GRAWA_TRY(check_heads(s, dq, N, Sq, s->H, true, true, a.dq));
    GRAWA_TRY(check_heads(s, dk, N, Sk, s->G, true, true, a.dk));
    GRAWA_TRY(check_heads(s, dv, N, Sk, s->G, true, true, a.dv));
    if ((dbias != nullptr) != (s->buckets > 0)) return GRAWA_ERR_INVALID_ARG;
    if (dbias) GRAWA_TRY(check_mats(s, dbias, (int64_t)s->H * s->buckets, true, a.dbias));
    if (!lse && N > 0 && Sq > 0) return GRAWA_ERR_INVALID_ARG;
    GRAWA_TRY(check_words(lse));
    a.lse = const_cast<float *>(lse);
    a.accumulate = accumulate ? 1 : 0;
    OnDevice dev(s->device);
    if (!dev.ok) return GRAWA_ERR_HIP;
    return status_of(grawa_launch_attend_backward(s, a, static_cast<hipStream_t>(stream)));
}

} // extern "C"
