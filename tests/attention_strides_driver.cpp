// Distances between rows (grawa_attention.cpp) with the HIP runtime and the kernels replaced by stubs: calls whose rows would be further apart than
// addresses reach are refused, and no sum of them is formed that 63 bits do not hold (built with the sanitizers).
#include <cstdio>

#include "grawa_attention.h"

static int launches;
extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t) { *p = (void *)((uintptr_t)1 << 44); return hipSuccess; }
hipError_t hipFree(void *) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { return hipSuccess; }
}
int grawa_head_norm_blocks(const grawa_attention_plan *) { return 4; }
// What a kernel forms of the largest indexes.
static hipError_t reach(const grawa_attention_plan *s, int64_t N, int64_t S, int heads, const GrawaHeads &h)
{
    const int64_t far = (int64_t)(s->K - 1) * h.worker + (N - 1) * h.seq + (S - 1) * h.token + (int64_t)(heads - 1) * h.head, all = (int64_t)s->H * h.head;
    return far < 0 || all < 0 ? hipErrorInvalidValue : hipSuccess;
}
hipError_t grawa_launch_head_norm(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads q, GrawaHeads k, GrawaMat, GrawaMat, float, const int *, GrawaHeads qo, GrawaHeads ko, hipStream_t)
{
    ++launches;
    for (const GrawaHeads *h : {&q, &qo})
        if (reach(s, N, S, s->H, *h) != hipSuccess) return hipErrorInvalidValue;
    for (const GrawaHeads *h : {&k, &ko})
        if (reach(s, N, S, s->G, *h) != hipSuccess) return hipErrorInvalidValue;
    return hipSuccess;
}
hipError_t grawa_launch_head_norm_backward(const grawa_attention_plan *, int64_t, int64_t, GrawaHeads, GrawaHeads, GrawaHeads, GrawaHeads, GrawaMat, GrawaMat, float, const int *, GrawaHeads,
                                           GrawaHeads, GrawaMat, GrawaMat, int, hipStream_t)
{
    return hipSuccess;
}
hipError_t grawa_launch_attend(const grawa_attention_plan *, GrawaAttend, hipStream_t) { return hipSuccess; }
hipError_t grawa_launch_attend_backward(const grawa_attention_plan *, GrawaAttend, hipStream_t) { return hipSuccess; }

#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            std::printf("line %d: %s\n", __LINE__, #cond);                  \
            return 1;                                                       \
        }                                                                   \
    } while (0)

int main()
{
    char *const at = (char *)((uintptr_t)1 << 40);
    const int64_t S = (int64_t)1 << 28, most = ((int64_t)1 << 40) - 1;
    const int D = 8;
    for (const grawa_dtype_t dt : {GRAWA_F32, GRAWA_BF16}) {
        const grawa_attention_shape_t shape = {1, 1, S, 2, 2, D, dt, 1.f, 0, 0, 0, 0, nullptr, 0, 0, nullptr};
        grawa_attention_plan_t *p = nullptr;
        EXPECT(grawa_attention_create(&p, &shape) == GRAWA_OK);
        const grawa_mats_t w = {at, D};
        const auto call = [&](const grawa_heads_t &in, const grawa_heads_t &out) { return grawa_head_norm(p, 1, S, &in, &out, &w, &w, 0.f, nullptr, &out, &out, nullptr); };
        const grawa_heads_t near = {at, 0, 0, 2 * D, D};
        EXPECT(call(near, near) == GRAWA_OK && launches == 1);
        launches = 0;
        // tokens far apart, read and written
        for (const int64_t token : {most, most / 2, ((int64_t)1 << 36) + 8, ((int64_t)1 << 28) + 8}) {
            EXPECT(call({at, 0, 0, token, D}, near) == GRAWA_ERR_UNSUPPORTED);
            EXPECT(call(near, {at, 0, 0, token, D}) == GRAWA_ERR_UNSUPPORTED);
        }
        EXPECT(launches == 0);
        // as far as they may be, and heads that are far apart beside them
        EXPECT(call({at, 0, 0, ((int64_t)1 << 28) - D, D}, {at, 0, 0, ((int64_t)1 << 28) - D, D}) == GRAWA_OK && launches == 1);
        EXPECT(call({at, 0, 0, 2 * D, most}, {at, 0, 0, D, most}) == GRAWA_OK && launches == 2);
        launches = 0;
        EXPECT(grawa_attention_destroy(p) == GRAWA_OK);
        // every axis alone within its bound, their sum not
        const grawa_attention_shape_t wide = {1024, 8, 2048, 64, 64, D, dt, 1.f, 0, 0, 0, 0, nullptr, 0, 0, nullptr};
        EXPECT(grawa_attention_create(&p, &wide) == GRAWA_OK);
        const grawa_heads_t all = {at, most, most, most, most}, good = {at, 8 * 2048 * 64 * D, 2048 * 64 * D, 64 * D, D};
        EXPECT(grawa_head_norm(p, 8, 2048, &all, &good, &w, &w, 0.f, nullptr, &good, &good, nullptr) == GRAWA_OK && launches == 1);
        launches = 0;
        EXPECT(grawa_attention_destroy(p) == GRAWA_OK);
    }
    std::printf("ok\n");
    return 0;
}
