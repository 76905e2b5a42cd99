// Elements of either type by the one or by the 16 bytes, widened to float32 (device side of the feed-forward sublayer).
#pragma once
#include "grawa_device.h"

typedef __bf16 grawa_bf16x8 __attribute__((ext_vector_type(8)));

// VEC consecutive elements from p on: 16 bytes at a time where VEC is more than one, p then on a 16-byte boundary.
template <bool BF16, int VEC> __device__ __forceinline__ void load_elements(const char *p, float *v)
{
    if constexpr (VEC == 1) {
        v[0] = BF16 ? bf16_one(*(const uint16_t *)p) : *(const float *)p;
    } else if constexpr (BF16) {
        static_assert(VEC % 8 == 0, "16 bytes");
#pragma unroll
        for (int q = 0; q < VEC / 8; ++q) {
            const uint4 u = ((const uint4 *)p)[q];
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * q + 2 * j] = bf16_lo(w[j]);
                v[8 * q + 2 * j + 1] = bf16_hi(w[j]);
            }
        }
    } else {
        static_assert(VEC % 4 == 0, "16 bytes");
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
            const float4 u = ((const float4 *)p)[q];
            v[4 * q] = u.x, v[4 * q + 1] = u.y, v[4 * q + 2] = u.z, v[4 * q + 3] = u.w;
        }
    }
}

template <bool BF16, int VEC> __device__ __forceinline__ void store_elements(char *p, const float *v)
{
    if constexpr (VEC == 1) {
        if constexpr (BF16)
            *(__bf16 *)p = (__bf16)v[0];
        else
            *(float *)p = v[0];
    } else if constexpr (BF16) {
#pragma unroll
        for (int q = 0; q < VEC / 8; ++q) {
            grawa_bf16x8 u;
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = (__bf16)v[8 * q + j];
            ((grawa_bf16x8 *)p)[q] = u;
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) ((float4 *)p)[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    }
}
