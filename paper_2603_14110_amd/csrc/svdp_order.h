// The order of logits as whole numbers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace svdp {

// A word that grows with the value: NaN above all, -0 equal to 0; and one that then falls with the index.
__device__ __forceinline__ uint32_t best_order(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t best_key(float v, uint32_t index)
{
    return ((uint64_t)best_order(v) << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, m);
        v = o > v ? o : v;
    }
    return v;
}
__device__ __forceinline__ int best_index(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }

}  // namespace svdp
