// What the attention kernels of latent caches share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ngc_device.h"

namespace ngc {

// A word that nobody writes during the launch, at a wave-uniform address: through the scalar unit.
__device__ __forceinline__ int32_t constant_word(const int32_t *p)
{
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>((uintptr_t)p);
}

// A value that is not finite would reach rows that do not see it, through a product with a weight of 0.  Where some of a tile's
// pairs are masked such values become 0 in the operand (this: four of them; whether there was one), and are added by
// themselves to the rows that see them.
__device__ __forceinline__ bool take_out_odd(u32x2 &x)
{
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if ((x[e] & 0x7F80u) == 0x7F80u) { odd = true; x[e] &= 0xFFFF0000u; }
        if ((x[e] & 0x7F800000u) == 0x7F800000u) { odd = true; x[e] &= 0xFFFFu; }
    }
    return odd;
}

__device__ __forceinline__ bool has_odd(u32x2 x) { return take_out_odd(x); }

}  // namespace ngc
