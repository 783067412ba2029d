// Device helpers of the kernels on the paged cache: vector types, E4M3 conversions, a block's exponent,
// and the search for the sequence of a work item.
#ifndef EPARA_CACHE_DEVICE_H
#define EPARA_CACHE_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "epara.h"
#include "epara_cache.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
#define EPARA_GLOBAL __attribute__((address_space(1)))

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
// two fp32 -> two bf16 (round to nearest even, in hardware), low half first
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2bf));
}

// Four fp32 -> four E4M3 codes, low byte first, round to nearest even; no saturation: |x| > 464 gives a NaN code.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true));
}
__device__ __forceinline__ float clamp448(float x) { return __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }

// The smallest e in [-96, 120] with amax <= 448 * 2^e; 448 = 1.75 * 2^8.
__device__ __forceinline__ int block_exponent(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -96 ? -96 : e > 120 ? 120 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }     // -126 <= e <= 127

// Mask of the first n bytes of a word (n <= 0: none, n >= 4: all).
__device__ __forceinline__ int low_bytes(int n) { return n >= 4 ? -1 : n <= 0 ? 0 : (1 << (8 * n)) - 1; }

// The sequence of work item `item`: the last one whose running sum is <= item (sequences without work are skipped by the rule itself).
// 64 sums are looked at in one step: up to 64 sequences take one trip to memory, up to 4096 two.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ first, int n, int item, int lane)
{
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const int sum = at < n ? first[lo + at] : 0x7fffffff;
        const int before = (__builtin_popcountll(__ballot(sum <= item)) - 1) * step;     // sums never decrease and first[0] = 0
        lo += before;
        n = n - before < step ? n - before : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace

#endif
