// Elements of either type, one by one or by 16 bytes at any alignment, widened to float32 (device side of the feed-forward sublayer).
#pragma once
#include "grawa_device.h"

typedef __bf16 grawa_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t GrawaAny16 __attribute__((ext_vector_type(4), aligned(2))); // 16 bytes anywhere: one instruction all the same
typedef uint32_t GrawaAny8 __attribute__((ext_vector_type(2), aligned(2)));

template <bool BF16> __device__ __forceinline__ float load_one(const char *p) { return BF16 ? bf16_one(*(const uint16_t *)p) : *(const float *)p; }

template <bool BF16> __device__ __forceinline__ void store_one(char *p, float v)
{
    if constexpr (BF16)
        *(__bf16 *)p = (__bf16)v;
    else
        *(float *)p = v;
}

// 16 bytes: eight bfloat16 or four float32.
template <bool BF16> struct GrawaPiece {
    static constexpr int N = BF16 ? 8 : 4, S = BF16 ? 2 : 4;
    uint32_t w[4];

    // n (> 0) elements are left of the row; what it does not have is 0.
    __device__ __forceinline__ void load(const char *p, int n)
    {
        if (n >= N) {
            const GrawaAny16 v = *(const GrawaAny16 *)p;
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            w[0] = w[1] = w[2] = w[3] = 0;
#pragma unroll
            for (int j = 0; j < N - 1; ++j)
                if (j < n) {
                    if constexpr (BF16)
                        w[j / 2] |= (uint32_t)((const uint16_t *)p)[j] << (j % 2 * 16);
                    else
                        w[j] = ((const uint32_t *)p)[j];
                }
        }
    }
    __device__ __forceinline__ float operator[](int j) const { return BF16 ? (j % 2 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2])) : __uint_as_float(w[j]); }
};

// NT: for what nobody reads again soon.
template <bool BF16, bool NT = false> __device__ __forceinline__ void store_piece(char *p, int n, const float *v)
{
    constexpr int N = GrawaPiece<BF16>::N, S = GrawaPiece<BF16>::S;
    if (n >= N) {
        GrawaAny16 u;
        if constexpr (BF16) {
            grawa_bf16x8 b;
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = (__bf16)v[j];
            u = __builtin_bit_cast(GrawaAny16, b);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = __float_as_uint(v[j]);
        }
        if (NT)
            __builtin_nontemporal_store(u, (GrawaAny16 *)p);
        else
            *(GrawaAny16 *)p = u;
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < n) store_one<BF16>(p + j * S, v[j]);
    }
}
