// Random words of a counter: Philox4x32 with 7 rounds, from the formulas of Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3" (2011), who report 7 rounds as the fewest that pass BigCrush.  Seven and not the customary ten: the
// rounds are the only work of a dropout beside its loads and stores.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

struct GrawaWords {
    uint32_t w[4];
};

// The compiler makes two instructions of a ^ b ^ c.
__device__ __forceinline__ uint32_t grawa_xor3(uint32_t a, uint32_t b, uint32_t c)
{
#ifdef __HIP_DEVICE_COMPILE__
    return (uint32_t)__builtin_amdgcn_bitop3_b32((int)a, (int)b, (int)c, 0x96);
#else
    return a ^ b ^ c; // plain C++ includes this header for its types
#endif
}

__device__ __forceinline__ GrawaWords grawa_philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
        c0 = grawa_xor3((uint32_t)(q >> 32), c1, k0);
        c1 = (uint32_t)q;
        c2 = grawa_xor3((uint32_t)(p >> 32), c3, k1);
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return GrawaWords{{c0, c1, c2, c3}};
}

// What a dropout goes by: element (row, column) is kept if word column % 4 of the counter (column / 4, row, site, step) is at least
// `threshold` = floor(p 2^32); what is kept is multiplied by `scale` = 1 / (1 - p).  rng: seed and step, on the device.
struct GrawaDrop {
    const uint64_t *rng; // null: nothing is dropped
    uint32_t threshold, site;
    float scale;
};

struct GrawaDropKey {
    uint32_t k0, k1, step;
};

__device__ __forceinline__ GrawaDropKey grawa_drop_key(const GrawaDrop &d)
{
    const uint64_t seed = d.rng[0], step = d.rng[1];
    return GrawaDropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step};
}

// Four elements from column 4 quad on.  A dropped one is 0 whatever it held, an infinity or a NaN too.
__device__ __forceinline__ void grawa_drop4(const GrawaDrop &d, const GrawaDropKey &k, uint32_t row, uint32_t quad, float *v)
{
    const GrawaWords r = grawa_philox(quad, row, d.site, k.step, k.k0, k.k1);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = r.w[j] >= d.threshold ? v[j] * d.scale : 0.f;
}
