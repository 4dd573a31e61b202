// Codes as vectors at any address of their element size (the device loads and stores unaligned vectors).
#pragma once
#include "common.hpp"

namespace adapt {

template <typename T>
__device__ __forceinline__ void load8(const T *p, int (&c)[8])
{
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(c, p, 32);
    } else {
        uint32_t w[2 * sizeof(T)];
        __builtin_memcpy(w, p, sizeof(w));
#pragma unroll
        for (int j = 0; j < 8; ++j)
            c[j] = sizeof(T) == 1 ? (int)(int8_t)(w[j >> 2] >> (8 * (j & 3))) : (int)(int16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const int (&c)[8])
{
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(p, c, 32);
    } else {
        uint32_t w[2 * sizeof(T)];
#pragma unroll
        for (int k = 0; k < (int)(2 * sizeof(T)); ++k)
            w[k] = sizeof(T) == 1 ? (uint32_t)(c[4 * k] & 0xff) | ((uint32_t)(c[4 * k + 1] & 0xff) << 8) | ((uint32_t)(c[4 * k + 2] & 0xff) << 16) |
                                        ((uint32_t)c[4 * k + 3] << 24)
                                  : (uint32_t)(c[2 * k] & 0xffff) | ((uint32_t)c[2 * k + 1] << 16);
        __builtin_memcpy(p, w, sizeof(w));
    }
}

// Codes from sums z + R in units of 2^-16: the upper halves of the sums, or their lower bytes, side by side.  PAST: past the caches
template <bool PAST, typename G, int N>
__device__ __forceinline__ void store_upper(G *p, const uint32_t (&t)[N])
{
    uint32_t w[N * sizeof(G) / 4];
#pragma unroll
    for (int k = 0; k < (int)(N * sizeof(G) / 4); ++k) {
        if constexpr (sizeof(G) == 2) {
            w[k] = __builtin_amdgcn_perm(t[2 * k + 1], t[2 * k], 0x07060302u);
        } else {
            const uint32_t lo = __builtin_amdgcn_perm(t[4 * k + 1], t[4 * k], 0x0c0c0602u), hi = __builtin_amdgcn_perm(t[4 * k + 3], t[4 * k + 2], 0x0c0c0602u);
            w[k] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        }
    }
    if constexpr (PAST) {
        typedef uint32_t vec __attribute__((ext_vector_type(N * sizeof(G) / 4), aligned(1)));
        vec v;
        __builtin_memcpy(&v, w, sizeof(w));
        __builtin_nontemporal_store(v, reinterpret_cast<vec *>(p));
    } else {
        __builtin_memcpy(p, w, sizeof(w));
    }
}

}  // namespace adapt
