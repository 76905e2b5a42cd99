// Host side of the attention's entry points (grawa_attention.cpp) with the HIP runtime and the kernels replaced by stubs: which
// arguments are refused, that a refused call launches nothing, and what is reported where a launch or an allocation fails.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "grawa_attention.h"

static int launches, fail_launch, no_memory, fail_copy, device, allocated;
static size_t last_bytes;
static GrawaAttend last;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = device; return hipSuccess; }
hipError_t hipSetDevice(int d) { device = d; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    last_bytes = n;
    if (no_memory || n > ((size_t)1 << 31)) return hipErrorOutOfMemory;
    ++allocated;
    *p = std::malloc(n ? n : 1);
    return *p ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipFree(void *p) { --allocated; std::free(p); return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipMemcpy(void *to, const void *from, size_t n, hipMemcpyKind)
{
    if (fail_copy) return hipErrorInvalidValue;
    std::memcpy(to, from, n);
    return hipSuccess;
}
}

static hipError_t launched()
{
    ++launches;
    return fail_launch ? hipErrorLaunchFailure : hipSuccess;
}
int grawa_head_norm_blocks(const grawa_attention_plan *) { return 4; }
hipError_t grawa_launch_head_norm(const grawa_attention_plan *s, int64_t, int64_t, GrawaHeads, GrawaHeads, GrawaMat, GrawaMat, float, const int *, GrawaHeads, GrawaHeads, hipStream_t)
{
    return device == s->device ? launched() : hipErrorInvalidDevice;
}
hipError_t grawa_launch_head_norm_backward(const grawa_attention_plan *, int64_t, int64_t, GrawaHeads, GrawaHeads, GrawaHeads, GrawaHeads, GrawaMat, GrawaMat, float, const int *, GrawaHeads,
                                           GrawaHeads, GrawaMat, GrawaMat, int, hipStream_t)
{
    return launched();
}
hipError_t grawa_launch_attend(const grawa_attention_plan *, GrawaAttend a, hipStream_t) { last = a; return launched(); }
hipError_t grawa_launch_attend_backward(const grawa_attention_plan *, GrawaAttend a, hipStream_t) { last = a; return launched(); }

#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            std::printf("line %d: %s\n", __LINE__, #cond);                  \
            return 1;                                                       \
        }                                                                   \
    } while (0)

static const grawa_status_t OK = GRAWA_OK, ARG = GRAWA_ERR_INVALID_ARG, ALIGN = GRAWA_ERR_ALIGNMENT, NOT = GRAWA_ERR_UNSUPPORTED;

int main()
{
    alignas(16) static char room[1 << 16];
    const int K = 2, N = 3, S = 4, H = 4, G = 2, D = 16, B = 3;
    const double freq[8] = {1, .5, .25, .1, .05, .01, .005, .001};
    const int32_t of[4] = {0, 1, 1, 2};
    const grawa_attention_shape_t good = {K, N, S, H, G, D, GRAWA_BF16, 0.25f, 3, 1, 8, 0, freq, B, 4, of};
    grawa_attention_plan_t *p = nullptr, *q = nullptr;
    grawa_attention_shape_t s;

    // shapes
    EXPECT(grawa_attention_create(nullptr, &good) == ARG);
    EXPECT(grawa_attention_create(&q, nullptr) == ARG);
#define SHAPE(status, change)                                       \
    do {                                                            \
        s = good;                                                   \
        s.change;                                                   \
        q = (grawa_attention_plan_t *)room;                         \
        EXPECT(grawa_attention_create(&q, &s) == status && !q);     \
    } while (0)
    SHAPE(ARG, K = 0);
    SHAPE(ARG, sequences = -1);
    SHAPE(ARG, length = -1);
    SHAPE(ARG, heads = 0);
    SHAPE(ARG, kv_heads = 0);
    SHAPE(ARG, kv_heads = 3);
    SHAPE(ARG, width = 0);
    SHAPE(ARG, window = -1);
    SHAPE(ARG, sinks = -1);
    SHAPE(ARG, scale = 0.f);
    SHAPE(ARG, scale = -1.f);
    SHAPE(ARG, scale = NAN);
    SHAPE(ARG, scale = INFINITY);
    SHAPE(ARG, rotary = 3);
    SHAPE(ARG, rotary = 18);
    SHAPE(ARG, rotary = -2);
    SHAPE(ARG, frequencies = nullptr);
    SHAPE(ARG, buckets = -1);
    SHAPE(ARG, buckets = 2);                                        // bucket 2 is in the table
    SHAPE(ARG, distances = 0);
    SHAPE(ARG, bucket_of = nullptr);
    SHAPE(NOT, dtype = (grawa_dtype_t)7);
    SHAPE(NOT, K = GRAWA_MAX_WORKERS + 1);
    SHAPE(NOT, width = 12);
    SHAPE(NOT, width = 136);
    SHAPE(NOT, buckets = GRAWA_MAX_BUCKETS + 1);
    SHAPE(NOT, distances = GRAWA_MAX_DISTANCES + 1);
    SHAPE(NOT, sequences = (int64_t)1 << 40);
    SHAPE(NOT, length = (int64_t)1 << 40);
    SHAPE(NOT, length = ((int64_t)1 << 28) + 1);
    const double bad_freq[8] = {1, INFINITY};
    const int32_t bad_of[4] = {0, -1, 0, 0};
    SHAPE(ARG, frequencies = bad_freq);
    SHAPE(ARG, bucket_of = bad_of);
    no_memory = 1;
    SHAPE(GRAWA_ERR_WORKSPACE, K = K);
    no_memory = 0;
    fail_copy = 1;
    SHAPE(GRAWA_ERR_HIP, K = K);
    fail_copy = 0;
    EXPECT(allocated == 0);
    device = 1;
    EXPECT(grawa_attention_create(&p, &good) == OK && p && allocated == 1);
    device = 0;
    EXPECT(p->window == 3 && p->turns[0] == (double)(1.0L / 6.283185307179586476925286766559L) && p->bucket_of[3] == 2);
    // the carved parts lie in the allocation, in order and apart
    EXPECT((char *)p->turns == p->ws && (char *)(p->part + p->part_floats) <= p->ws + last_bytes);
    EXPECT((char *)p->bucket_of >= (char *)(p->turns + 4) && (char *)p->rows >= (char *)(p->bucket_of + 4));
    EXPECT((char *)p->norm_part >= (char *)(p->rows + 2 * K * N * H * 256) && (char *)p->bias_part >= (char *)(p->norm_part + K * 4 * 2 * D));
    EXPECT((char *)p->part >= (char *)(p->bias_part + K * N * H * B));
    // a plan without bias, without rotation, without a window
    s = good;
    s.buckets = 0, s.bucket_of = nullptr, s.distances = 0, s.rotary = 0, s.frequencies = nullptr, s.window = 0, s.sinks = (int64_t)1 << 50;
    EXPECT(grawa_attention_create(&q, &s) == OK && q->window == GRAWA_NO_WINDOW && q->distances == 0);

    // calls
    const int64_t qs[4] = {N * S * H * D, S * H * D, H * D, D}, ks[4] = {N * S * G * D, S * G * D, G * D, D};
    const grawa_heads_t hq = {room, qs[0], qs[1], qs[2], qs[3]}, hk = {room, ks[0], ks[1], ks[2], ks[3]};
    const grawa_mats_t w = {room, 64}, bias = {room, 64};
    int32_t places[K * N] = {};
    float lse[K * N * H * S];
#define NORM(plan, n, t, a, b, c, d, e, st, f, g) grawa_head_norm(plan, n, t, a, b, c, d, e, st, f, g, nullptr)
#define NORM_BACK(plan, n, t, a, b, c, d, wa, wb, e, f, g, ga, gb) grawa_head_norm_backward(plan, n, t, a, b, c, d, wa, wb, e, nullptr, f, g, ga, gb, 0, nullptr)
#define ATT(plan, n, t, u, a, b, c, m, le, st, o, l) grawa_attention(plan, n, t, u, a, b, c, m, le, st, o, l, nullptr)
#define ATT_BACK(plan, n, t, u, g, a, b, c, m, o, l, da, db, dc, dm) grawa_attention_backward(plan, n, t, u, g, a, b, c, m, nullptr, nullptr, o, l, da, db, dc, dm, 0, nullptr)
    EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, 1e-6f, places, &hq, &hk) == OK);
    EXPECT(NORM_BACK(p, N, S, &hq, &hk, &hq, &hk, &w, &w, 1e-6f, &hq, &hk, &w, &w) == OK);
    EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &bias, places, places, &hq, lse) == OK && last.share == 2 && last.row_pitch == 256);
    EXPECT(last.q.token == H * D * 2 && last.k.head == D * 2 && last.row_dot - last.row_lse == K * N * H * 256);
    EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, &bias) == OK);
    EXPECT(launches == 4 && device == 0);
    launches = 0;
    // counts
    EXPECT(ATT(nullptr, N, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT(p, N + 1, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT(p, N, S + 1, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT(p, N, S, S + 1, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT(p, -1, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(NORM(p, N, S + 1, &hq, &hk, &w, &w, 1e-6f, nullptr, &hq, &hk) == ARG);
    EXPECT(NORM(nullptr, N, S, &hq, &hk, &w, &w, 1e-6f, nullptr, &hq, &hk) == ARG);
    // bias and plan
    EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, nullptr, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT(q, N, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == ARG);
    EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, nullptr) == ARG);
    EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, nullptr, &hq, &hk, &hk, &bias) == ARG);
    EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, -1.f, nullptr, &hq, &hk) == ARG);
    EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, NAN, nullptr, &hq, &hk) == ARG);
    EXPECT(NORM(p, N, S, &hq, &hk, &w, nullptr, 1e-6f, nullptr, &hq, &hk) == ARG);
    // every tensor of heads in every place
    for (int i = 0; i < 10; ++i) {
        grawa_heads_t b = hq;
        grawa_status_t in = ARG, out = ARG, norm_in = ARG, norm_out = ARG;
        switch (i) {
        case 0: b.data = nullptr; break;
        case 1: b.token = -8; break;
        case 2: b.sequence = (int64_t)1 << 41; in = out = norm_in = norm_out = NOT; break;
        case 3: b.data = room + 2; in = out = ALIGN; norm_in = norm_out = OK; break;           // norms take any place of whole elements
        case 4: b.data = room + 1; in = out = norm_in = norm_out = ALIGN; break;
        case 5: b.token += 4; in = out = ALIGN; norm_in = OK; norm_out = ARG; break;             // and rows that no longer fit a sequence
        case 6: b.head = 0; in = norm_in = OK; break;                                          // heads may share a row to be read
        case 7: b.worker = 0; in = norm_in = OK; break;
        case 8: b.token = (int64_t)1 << 24; in = out = NOT; norm_in = OK; norm_out = OK; b.worker = (int64_t)1 << 36; b.sequence = (int64_t)1 << 30; break;
        case 9: b.head = S * N * K * D, b.token = D, b.sequence = S * D, b.worker = N * S * D; in = out = norm_in = norm_out = OK; break; // heads outermost
        }
        const grawa_heads_t kb = {b.data, i >= 5 && i <= 8 ? b.worker : hk.worker, i == 2 || i == 8 ? b.sequence : hk.sequence, i == 1 || i == 5 || i == 8 ? b.token - (i == 5 ? (H - G) * D : 0) : hk.token, i == 6 ? 0 : hk.head};
        EXPECT(ATT(p, N, S, S, &b, &hk, &hk, &bias, nullptr, nullptr, &hq, lse) == in);
        EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &b, lse) == out);
        EXPECT(ATT_BACK(p, N, S, S, &b, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, &bias) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &b, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, &bias) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &b, lse, &hq, &hk, &hk, &bias) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &b, &hk, &hk, &bias) == out);
        EXPECT(NORM(p, N, S, &b, &hk, &w, &w, 1e-6f, nullptr, &hq, &hk) == norm_in);
        EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, 1e-6f, nullptr, &b, &hk) == norm_out);
        EXPECT(NORM_BACK(p, N, S, &b, &hk, &hq, &hk, &w, &w, 1e-6f, &hq, &hk, &w, &w) == norm_in);
        EXPECT(NORM_BACK(p, N, S, &hq, &hk, &b, &hk, &w, &w, 1e-6f, &hq, &hk, &w, &w) == norm_in);
        EXPECT(NORM_BACK(p, N, S, &hq, &hk, &hq, &hk, &w, &w, 1e-6f, &b, &hk, &w, &w) == norm_out);
        if (i == 9) continue;
        EXPECT(ATT(p, N, S, S, &hq, &kb, &hk, &bias, nullptr, nullptr, &hq, lse) == in);
        EXPECT(ATT(p, N, S, S, &hq, &hk, &kb, &bias, nullptr, nullptr, &hq, lse) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &kb, &hk, &bias, &hq, lse, &hq, &hk, &hk, &bias) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &kb, &bias, &hq, lse, &hq, &hk, &hk, &bias) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &kb, &hk, &bias) == out);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &kb, &bias) == out);
        EXPECT(NORM(p, N, S, &hq, &kb, &w, &w, 1e-6f, nullptr, &hq, &hk) == norm_in);
        EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, 1e-6f, nullptr, &hq, &kb) == norm_out);
    }
    // parameters
    for (int i = 0; i < 5; ++i) {
        grawa_mats_t b = w;
        grawa_status_t in = ARG, out = ARG;
        if (i == 0) b.data = nullptr;
        if (i == 1) b.worker = -1;
        if (i == 2) b.worker = (int64_t)1 << 48, in = out = NOT;
        if (i == 3) b.data = room + 1, in = out = ALIGN;
        if (i == 4) b.worker = 0, in = OK;                          // all workers may read one, not write it
        EXPECT(NORM(p, N, S, &hq, &hk, &b, &w, 1e-6f, nullptr, &hq, &hk) == in);
        EXPECT(NORM(p, N, S, &hq, &hk, &w, &b, 1e-6f, nullptr, &hq, &hk) == in);
        EXPECT(NORM_BACK(p, N, S, &hq, &hk, &hq, &hk, &b, &w, 1e-6f, &hq, &hk, &w, &w) == in);
        EXPECT(NORM_BACK(p, N, S, &hq, &hk, &hq, &hk, &w, &w, 1e-6f, &hq, &hk, &b, &w) == out);
        EXPECT(NORM_BACK(p, N, S, &hq, &hk, &hq, &hk, &w, &w, 1e-6f, &hq, &hk, &w, &b) == out);
        EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &b, nullptr, nullptr, &hq, lse) == in);
        EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, &b) == out);
    }
    EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &bias, (int32_t *)(room + 2), nullptr, &hq, lse) == ALIGN);
    EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &bias, nullptr, (int32_t *)(room + 1), &hq, lse) == ALIGN);
    EXPECT(ATT(p, N, S, S, &hq, &hk, &hk, &bias, nullptr, nullptr, &hq, (float *)(room + 2)) == ALIGN);
    EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, 1e-6f, (int32_t *)(room + 2), &hq, &hk) == ALIGN);
    // tensors of no rows are not looked at; strides of axes of one are not either
    const grawa_heads_t none = {nullptr, 0, 0, 0, 0}, odd = {room, 5, 3, H * D, D};
    launches = 0;
    EXPECT(ATT(p, 0, S, S, &none, &none, &none, &bias, nullptr, nullptr, &none, nullptr) == OK);
    EXPECT(ATT(p, N, S, 0, &hq, &none, &none, &bias, nullptr, nullptr, &hq, nullptr) == OK);
    EXPECT(ATT_BACK(p, N, 0, S, &none, &none, &hk, &hk, &bias, &none, nullptr, &none, &hk, &hk, &bias) == OK);
    EXPECT(launches == 3);
    s = good;
    s.K = 1, s.sequences = 1;
    grawa_attention_plan_t *one = nullptr;
    EXPECT(grawa_attention_create(&one, &s) == OK);
    EXPECT(ATT(one, 1, S, S, &odd, &hk, &hk, &bias, nullptr, nullptr, &odd, nullptr) == OK);
    EXPECT(grawa_attention_destroy(one) == OK);
    // failures
    fail_launch = 1;
    EXPECT(NORM(p, N, S, &hq, &hk, &w, &w, 1e-6f, nullptr, &hq, &hk) == GRAWA_ERR_HIP);
    EXPECT(ATT_BACK(p, N, S, S, &hq, &hq, &hk, &hk, &bias, &hq, lse, &hq, &hk, &hk, &bias) == GRAWA_ERR_HIP);
    EXPECT(device == 0);
    EXPECT(grawa_attention_destroy(nullptr) == OK && grawa_attention_destroy(p) == OK && grawa_attention_destroy(q) == OK && allocated == 0);
    std::printf("ok\n");
    return 0;
}
