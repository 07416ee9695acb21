// The matrix-core kernel of attention over an uncompressed cache (cache_attend.hip): bf16, 128 channels.
#pragma once

#include "cache.h"

namespace xkv {
namespace cache_tile {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(8))) float f32x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// 16 B per lane from base + off into LDS at lds_base + lane * 16 (base and lds_base are wave-uniform); see copy16_global_to_lds.
__device__ __forceinline__ void copy16_to_lds(const void *base, uint32_t off, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_base), "v"(off), "s"(base) : "memory", "m0");
}

// The same for rows that are read once: past the caches.
__device__ __forceinline__ void copy16_to_lds_once(const void *base, uint32_t off, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(lds_base), "v"(off), "s"(base) : "memory", "m0");
}

// Waits for LDS reads alone: what they read may be overwritten after it (and none of them is moved behind it).
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// Both halves of a wavefront see the other's value as well: max or sum of lanes l and l + 32, in both.
__device__ __forceinline__ void halves(float x, float &lo, float &hi)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}

// The same for rows of 16 lanes: l and l + 16 of either half.
__device__ __forceinline__ void quarters(float x, float &lo, float &hi)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}

__device__ __forceinline__ f32x8_t eight(const f32x16_t &c, int j)
{
    f32x8_t x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = c[8 * j + e];
    return x;
}

__device__ __forceinline__ float sum8(const f32x8_t &p, float sum)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += p[e];
    return sum;
}

// Eight weights as operands of two products: their upper 16 bits (one instruction for two weights), and what is left of each, rounded.
// Together they hold a weight to 2^-15.  2^-22 of a weight more is left of each, so that it is not zero, which infinite values must not be
// multiplied with.
__device__ __forceinline__ bf16x8_t upper8(const f32x8_t &p)
{
    u32x4_t x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_perm(__float_as_uint(p[2 * e + 1]), __float_as_uint(p[2 * e]), 0x07060302u);
    return __builtin_bit_cast(bf16x8_t, x);
}
__device__ __forceinline__ bf16x8_t lower8(const f32x8_t &p)
{
    f32x8_t x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(p[e], 1.0f + 0x1p-22f, -__uint_as_float(__float_as_uint(p[e]) & 0xFFFF0000u));
    return __builtin_convertvector(x, bf16x8_t);
}

}  // namespace cache_tile
}  // namespace xkv
