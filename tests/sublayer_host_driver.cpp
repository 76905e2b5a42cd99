// Host side of the feed-forward sublayer's entry points (grawa_sublayer.cpp) with the HIP runtime and the kernels replaced by
// stubs: which arguments are refused, that a refused call launches nothing, and what is reported where a launch fails.
#include <cmath>
#include <cstdio>
#include <cstdlib>

#include "grawa_sublayer.h"

static int launches, fail_launch, no_memory, device, allocated;
static size_t last_bytes;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = device; return hipSuccess; }
hipError_t hipSetDevice(int d) { device = d; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    last_bytes = n;
    if (no_memory || n > ((size_t)1 << 30)) return hipErrorOutOfMemory;
    ++allocated;
    *p = std::malloc(n ? n : 1);
    return *p ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipFree(void *p) { --allocated; std::free(p); return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
}

static hipError_t launched()
{
    ++launches;
    return fail_launch ? hipErrorLaunchFailure : hipSuccess;
}
hipError_t grawa_launch_layer_norm(const grawa_sublayer *s, int64_t, GrawaRows, GrawaMat, GrawaMat, float, GrawaRows, float *, hipStream_t)
{
    return device == s->device ? launched() : hipErrorInvalidDevice;
}
hipError_t grawa_launch_layer_norm_backward(const grawa_sublayer *, int64_t, GrawaRows, GrawaRows, GrawaMat, const float *, GrawaRows, GrawaRows, GrawaMat, GrawaMat, int, hipStream_t) { return launched(); }
int grawa_norm_blocks(int, int64_t T, int64_t) { return T > 4 ? 4 : T > 0 ? (int)T : 1; }
hipError_t grawa_launch_dropout(int, int64_t, int64_t, grawa_dtype_t, GrawaRows, GrawaRows, GrawaDrop, GrawaRows, hipStream_t) { return launched(); }
int64_t grawa_ffn_part_floats(const grawa_sublayer *) { return 64; }
hipError_t grawa_launch_ffn(const grawa_sublayer *, int64_t, GrawaRows, GrawaMat, GrawaMat, GrawaMat, GrawaRows, GrawaDrop, GrawaRows, char *, hipStream_t) { return launched(); }
hipError_t grawa_launch_ffn_backward(const grawa_sublayer *, int64_t, GrawaRows, GrawaRows, GrawaMat, GrawaMat, GrawaMat, const char *, GrawaRows, GrawaMat, GrawaMat, GrawaMat, int, hipStream_t) { return launched(); }

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
    const int K = 3, T = 5, d = 8, f = 16;
    grawa_sublayer_t *p = nullptr, *q = nullptr;

    // shapes
    EXPECT(grawa_sublayer_create(nullptr, K, T, d, f, GRAWA_BF16, GRAWA_ACT_SILU) == ARG);
    const struct { int K; int64_t T, d, f; int dt, act; grawa_status_t want; } shapes[] = {
        {0, T, d, f, 1, 0, ARG}, {K, -1, d, f, 1, 0, ARG}, {K, T, 0, f, 1, 0, ARG}, {K, T, d, -1, 1, 0, ARG}, {K, T, d, f, 2, 0, NOT}, {K, T, d, f, 1, 3, ARG},
        {GRAWA_MAX_WORKERS + 1, T, d, f, 1, 0, NOT}, {2, ((int64_t)1 << 29) + 1, d, f, 1, 0, NOT}, {K, T, 1 << 20, f, 1, 0, NOT}, {K, T, d, 1 << 20, 1, 0, NOT},
        {1, (int64_t)1 << 62, d, f, 1, 0, NOT}, {K, T, (int64_t)1 << 62, f, 1, 0, NOT}};
    for (const auto &s : shapes) {
        q = (grawa_sublayer_t *)room;
        EXPECT(grawa_sublayer_create(&q, s.K, s.T, s.d, s.f, (grawa_dtype_t)s.dt, (grawa_act_t)s.act) == s.want && !q);
    }
    EXPECT(grawa_sublayer_create(&q, 1024, 1 << 20, (1 << 20) - 1, (1 << 20) - 1, GRAWA_F32, GRAWA_ACT_SILU) == GRAWA_ERR_WORKSPACE && !q);
    EXPECT(last_bytes > ((size_t)1 << 50)); // the sizes did not wrap round
    no_memory = 1;
    EXPECT(grawa_sublayer_create(&q, K, T, d, f, GRAWA_BF16, GRAWA_ACT_SILU) == GRAWA_ERR_WORKSPACE && !q);
    no_memory = 0;
    EXPECT(grawa_sublayer_destroy(nullptr) == OK);

    device = 2;
    EXPECT(grawa_sublayer_create(&p, K, T, d, f, GRAWA_BF16, GRAWA_ACT_SILU) == OK && p);
    EXPECT(grawa_sublayer_create(&q, K, T, d, 0, GRAWA_F32, GRAWA_ACT_RELU) == OK && q); // the layer norm alone
    device = 0;
    int64_t bytes = 0;
    EXPECT(grawa_sublayer_save_bytes(p, T, &bytes) == OK && bytes == K * (16 * 16 * (3 + 3) + T * 64 * 2)); // 5 tokens take a fragment of 16, rows are 64 wide
    EXPECT(grawa_sublayer_save_bytes(p, T + 1, &bytes) == ARG && grawa_sublayer_save_bytes(p, -1, &bytes) == ARG);
    EXPECT(grawa_sublayer_save_bytes(p, T, nullptr) == ARG && grawa_sublayer_save_bytes(nullptr, T, &bytes) == ARG && grawa_sublayer_save_bytes(q, T, &bytes) == ARG);

    const grawa_rows_t x{room, T * d, d}, y{room + 4096, T * d, d};
    const grawa_mats_t w{room + 8192, 64}, m{room + 16384, d * f};
    const int64_t rng[2] = {1, 2};
    float *stats = (float *)(room + 2048);
    void *save = room + 32768;

    const auto norm = [&](const grawa_rows_t *x, const grawa_mats_t *w, const grawa_mats_t *b, float eps, const grawa_rows_t *y, float *st, int64_t t) {
        return grawa_layer_norm(p, t, x, w, b, eps, y, st, nullptr);
    };
    const auto ffn = [&](const grawa_rows_t *x, const grawa_mats_t *a, const grawa_mats_t *b, const grawa_mats_t *c, const grawa_rows_t *r, float pr, const int64_t *g,
                         const grawa_rows_t *y, void *sv, int64_t t) { return grawa_ffn(p, t, x, a, b, c, r, pr, g, 0, y, sv, nullptr); };
    const auto back = [&](const grawa_rows_t *dy, const grawa_mats_t *a, void *sv, const grawa_rows_t *dx, const grawa_mats_t *da, int64_t t) {
        return grawa_ffn_backward(p, t, dy, &x, a, &m, &m, sv, dx, da, &m, &m, 0, nullptr);
    };
    const auto drop = [&](int K, int64_t T, int64_t d, int dt, const grawa_rows_t *x, const grawa_rows_t *r, float pr, const int64_t *g, const grawa_rows_t *y) {
        return grawa_dropout(K, T, d, (grawa_dtype_t)dt, x, r, pr, g, 0, y, nullptr);
    };
    // what is in order
    EXPECT(norm(&x, &w, &w, 1e-5f, &y, stats, T) == OK && norm(&x, &w, nullptr, 0.f, &x, nullptr, 1) == OK && device == 0);
    EXPECT(grawa_layer_norm_backward(p, T, &y, &x, &w, stats, nullptr, &y, &w, nullptr, 1, nullptr) == OK);
    EXPECT(ffn(&x, &m, &m, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == OK && ffn(&x, &m, &m, &m, &x, 0.5f, rng, &y, save, T) == OK);
    EXPECT(back(&y, &m, save, &y, &m, T) == OK);
    EXPECT(drop(K, T, d, 1, &x, nullptr, 0.5f, rng, &y) == OK && drop(K, T, d, 0, &x, &y, 0.f, nullptr, &y) == OK && launches == 8);
    const grawa_rows_t none{nullptr, 0, 0};
    EXPECT(norm(&none, &w, &w, 1e-5f, &none, nullptr, 0) == OK && ffn(&none, &m, &m, &m, nullptr, 0.f, nullptr, &none, nullptr, 0) == OK);
    EXPECT(drop(K, 0, d, 1, &none, nullptr, 0.5f, rng, &none) == OK);
    const grawa_rows_t shared{room, 0, d}, first{room + 4096, d, K * d}; // one batch for all workers; tokens outside, workers inside
    EXPECT(norm(&shared, &w, &w, 1e-5f, &first, stats, T) == OK);
    fail_launch = 1;
    EXPECT(norm(&x, &w, &w, 1e-5f, &y, stats, T) == GRAWA_ERR_HIP && ffn(&x, &m, &m, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == GRAWA_ERR_HIP);
    EXPECT(back(&y, &m, save, &y, &m, T) == GRAWA_ERR_HIP && drop(K, T, d, 1, &x, nullptr, 0.5f, rng, &y) == GRAWA_ERR_HIP);
    fail_launch = launches = 0;

    // tokens, plans
    EXPECT(norm(&x, &w, &w, 1e-5f, &y, stats, T + 1) == ARG && norm(&x, &w, &w, 1e-5f, &y, stats, -1) == ARG);
    EXPECT(grawa_layer_norm(nullptr, T, &x, &w, &w, 1e-5f, &y, stats, nullptr) == ARG);
    EXPECT(grawa_layer_norm_backward(nullptr, T, &y, &x, &w, stats, nullptr, &y, &w, nullptr, 1, nullptr) == ARG);
    EXPECT(grawa_ffn(nullptr, T, &x, &m, &m, &m, nullptr, 0.f, nullptr, 0, &y, nullptr, nullptr) == ARG);
    EXPECT(grawa_ffn(q, T, &x, &m, &m, &m, nullptr, 0.f, nullptr, 0, &y, nullptr, nullptr) == ARG); // a plan without an inner width
    EXPECT(grawa_ffn_backward(q, T, &y, &x, &m, &m, &m, save, &y, &m, &m, &m, 0, nullptr) == ARG);
    EXPECT(grawa_ffn_backward(nullptr, T, &y, &x, &m, &m, &m, save, &y, &m, &m, &m, 0, nullptr) == ARG);
    // rows
    const struct { grawa_rows_t r; grawa_status_t in, out; } rows[] = {
        {{nullptr, T * d, d}, ARG, ARG}, {{room, -1, d}, ARG, ARG}, {{room, T * d, -1}, ARG, ARG}, {{room + 1, T * d, d}, ALIGN, ALIGN}, {{room, (int64_t)1 << 48, d}, NOT, NOT},
        {{room, T * d, (int64_t)1 << 30}, NOT, NOT}, {{room, T * d, d - 1}, OK, ARG}, {{room, T * d - 1, d}, OK, ARG}, {{room, 0, d}, OK, ARG}, {{room, d, K * d - 1}, OK, ARG}};
    for (const auto &r : rows) {
        EXPECT(norm(&r.r, &w, &w, 1e-5f, &y, stats, T) == r.in && norm(&x, &w, &w, 1e-5f, &r.r, stats, T) == r.out);
        EXPECT(ffn(&r.r, &m, &m, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == r.in && ffn(&x, &m, &m, &m, nullptr, 0.f, nullptr, &r.r, nullptr, T) == r.out);
        EXPECT(ffn(&x, &m, &m, &m, &r.r, 0.f, nullptr, &y, nullptr, T) == r.in);
        EXPECT(back(&r.r, &m, save, &y, &m, T) == r.in && back(&x, &m, save, &r.r, &m, T) == r.out);
        EXPECT(drop(K, T, d, 1, &r.r, nullptr, 0.5f, rng, &y) == r.in && drop(K, T, d, 1, &x, nullptr, 0.5f, rng, &r.r) == r.out && drop(K, T, d, 1, &x, &r.r, 0.5f, rng, &y) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &x, &x, &w, stats, &r.r, &y, &w, nullptr, 0, nullptr) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &r.r, &x, &w, stats, nullptr, &y, &w, nullptr, 0, nullptr) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &x, &r.r, &w, stats, nullptr, &y, &w, nullptr, 0, nullptr) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &x, &x, &w, stats, nullptr, &r.r, &w, nullptr, 0, nullptr) == r.out);
    }
    EXPECT(norm(nullptr, &w, &w, 1e-5f, &y, stats, T) == ARG && norm(&x, &w, &w, 1e-5f, nullptr, stats, T) == ARG);
    EXPECT(drop(K, T, d, 1, nullptr, nullptr, 0.5f, rng, &y) == ARG && drop(K, T, d, 1, &x, nullptr, 0.5f, rng, nullptr) == ARG);
    EXPECT(back(nullptr, &m, save, &y, &m, T) == ARG && back(&x, &m, save, nullptr, &m, T) == ARG);
    // matrices and vectors
    const struct { grawa_mats_t m; grawa_status_t in, out; } mats[] = {{{nullptr, 4096}, ARG, ARG}, {{room, -1}, ARG, ARG}, {{room + 1, 4096}, ALIGN, ALIGN}, {{room, (int64_t)1 << 48}, NOT, NOT}, {{room, d - 1}, OK, ARG}, {{room, 0}, OK, ARG}};
    for (const auto &r : mats) {
        EXPECT(norm(&x, &r.m, &w, 1e-5f, &y, stats, T) == r.in && norm(&x, &w, &r.m, 1e-5f, &y, stats, T) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &y, &x, &r.m, stats, nullptr, &y, &w, nullptr, 0, nullptr) == r.in);
        EXPECT(grawa_layer_norm_backward(p, T, &y, &x, &w, stats, nullptr, &y, &r.m, nullptr, 0, nullptr) == r.out && grawa_layer_norm_backward(p, T, &y, &x, &w, stats, nullptr, &y, &w, &r.m, 0, nullptr) == r.out);
        EXPECT(ffn(&x, &r.m, &m, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == r.in && ffn(&x, &m, &r.m, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == r.in && ffn(&x, &m, &m, &r.m, nullptr, 0.f, nullptr, &y, nullptr, T) == r.in);
        EXPECT(back(&y, &r.m, save, &y, &m, T) == r.in && back(&y, &m, save, &y, &r.m, T) == r.out);
    }
    EXPECT(norm(&x, nullptr, &w, 1e-5f, &y, stats, T) == ARG && ffn(&x, &m, nullptr, &m, nullptr, 0.f, nullptr, &y, nullptr, T) == ARG && back(&y, &m, save, &y, nullptr, T) == ARG);
    // numbers and the other buffers
    for (const float bad : {-1e-6f, INFINITY, NAN}) EXPECT(norm(&x, &w, &w, bad, &y, stats, T) == ARG);
    EXPECT(norm(&x, &w, &w, 1e-5f, &y, stats + 1, T) == ALIGN);
    EXPECT(grawa_layer_norm_backward(p, T, &y, &x, &w, nullptr, nullptr, &y, &w, nullptr, 0, nullptr) == ARG && grawa_layer_norm_backward(p, T, &y, &x, &w, stats + 1, nullptr, &y, &w, nullptr, 0, nullptr) == ALIGN);
    EXPECT(ffn(&x, &m, &m, &m, nullptr, 0.f, nullptr, &y, room + 8, T) == ALIGN && back(&y, &m, room + 8, &y, &m, T) == ALIGN && back(&y, &m, nullptr, &y, &m, T) == ARG);
    for (const float bad : {-0.1f, 1.f, 2.f, INFINITY, NAN}) {
        EXPECT(drop(K, T, d, 1, &x, nullptr, bad, rng, &y) == ARG && ffn(&x, &m, &m, &m, nullptr, bad, rng, &y, nullptr, T) == ARG);
    }
    EXPECT(drop(K, T, d, 1, &x, nullptr, 0.5f, nullptr, &y) == ARG && ffn(&x, &m, &m, &m, nullptr, 0.5f, nullptr, &y, nullptr, T) == ARG);
    EXPECT(drop(K, T, d, 1, &x, nullptr, 0.5f, (const int64_t *)((const char *)rng + 4), &y) == ALIGN);
    EXPECT(drop(0, T, d, 1, &x, nullptr, 0.5f, rng, &y) == ARG && drop(K, -1, d, 1, &x, nullptr, 0.5f, rng, &y) == ARG && drop(K, T, 0, 1, &x, nullptr, 0.5f, rng, &y) == ARG);
    EXPECT(drop(K, T, d, 2, &x, nullptr, 0.5f, rng, &y) == NOT && drop(K, (int64_t)1 << 30, d, 1, &x, nullptr, 0.5f, rng, &y) == NOT);
    EXPECT(launches == 4 * 9 + 2 * 7); // of the four rows and two matrices above that are in order as inputs, and of nothing refused
    EXPECT(grawa_sublayer_destroy(p) == OK && grawa_sublayer_destroy(q) == OK && allocated == 0 && device == 0);
    std::puts("ok");
    return 0;
}
