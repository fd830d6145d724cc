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

// 16 bytes per lane from `base` (uniform) + offset straight into LDS, lane l to lds + 16 l (uniform), without the compiler's knowledge:
// of a load that it knows of it assumes that any transposing read may meet it, and waits for all that is on its way, the tiles that
// are asked for ahead included.  Here nothing waits but wait_for_loads(); no register is written.  (A barrier behind the last reads
// of what the load overwrites, wait_for_loads() and a barrier before the first reads of what it brings are the caller's.)
__device__ __forceinline__ void start_load_to_lds16(const unsigned char *base, uint32_t offset, const unsigned char *lds)
{
    const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char *)lds;
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(at) : "memory");
}
// The same for 4 bytes per lane, lane l to lds + 4 l.
__device__ __forceinline__ void start_load_to_lds4(const unsigned char *base, uint32_t offset, const unsigned char *lds)
{
    const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char *)lds;
    __asm__ volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(offset), "s"(base), "s"(at) : "memory");
}
// Until at most N of this wave's loads are on their way, and no read of LDS.
template <int N>
__device__ __forceinline__ void wait_for_loads()
{
    __asm__ volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}
// Everything that this wave has asked for is there, and the compiler knows it.  Needed before a loop that uses what was loaded before it:
// the compiler would count, inside the loop, the loads that may still be on their way on its first turn, and wait for the tiles asked
// for ahead of it in their place, on every turn.
__device__ __forceinline__ void own_rows_loaded() { __builtin_amdgcn_s_waitcnt(0x0F70); }       // vmcnt(0)
// No access to LDS of this wave is on its way.
__device__ __forceinline__ void lds_accesses_done() { __asm__ volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }
__device__ __forceinline__ void workgroup_barrier()
{
    __asm__ volatile("s_barrier" : : : "memory");
}

// 16-byte piece p of row r of a tile in LDS stands at slot p ^ lds_swizzle<PIECES>(r) of its row.  LDS has 64 banks, and what reads
// together is (measured: pairs of lanes of one bank, one of them after the other)
//   reads of 16 bytes           lanes 0-3, 12-15, 20-23, 24-27, the other 16 of the lower half, and the same of the upper half;
//   transposing reads of 8      the lower half and the upper half.
// With row = lane % 32 and piece p, or row = lane % 16 and piece p + lane / 16, the first meet every bank once; so do the second
// with 4 rows of 64 bytes (32 columns) or 8 rows of 32 bytes (16 columns) a half.  Written with r = r3 r2 r1 r0: rows of 256 bytes
// and multiples r1 r0 (r2^r3) r3, of 128 bytes without r0, of 64 without r1 r0, which count the rows of a line of banks there.
template <int PIECES>
__device__ __forceinline__ int lds_swizzle(int r)
{
    const int low = ((r >> 2) ^ (r >> 3)) % 2 * 2 + (r >> 3) % 2;
    return PIECES >= 16 ? r % 4 * 4 + low : PIECES == 8 ? (r >> 1) % 2 * 4 + low : low;
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
// 1 where a value is not finite, 0 where it is.
__device__ __forceinline__ u32x2 odd_ones(u32x2 x)
{
    u32x2 ones;
#pragma unroll
    for (int e = 0; e < 2; ++e) ones[e] = ((x[e] & 0x7F80u) == 0x7F80u ? 0x3F80u : 0u) | ((x[e] & 0x7F800000u) == 0x7F800000u ? 0x3F800000u : 0u);
    return ones;
}

}  // namespace ngc
