// The 8-bit form of a page: e4m3 bytes, and for the keys and for the values of every KV head a scale that is a power of two.
#pragma once

#include "chess_internal.h"

namespace chess {

typedef __attribute__((ext_vector_type(2))) float f32x2;

// Exponents of a scale.  The largest: 448 2^119 is below the largest bf16 value's double, so that every stored value is finite in fp32; with the
// smallest, values below 2^-74 become 0.
constexpr int kScaleMin = -64, kScaleMax = 119;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// 16 bytes that no one reads again soon: kOnce, as a stream that does not stay in the caches.
template <bool kOnce>
__device__ __forceinline__ uint4 load_16(const uint8_t* p)
{
    if constexpr (!kOnce) return *reinterpret_cast<const uint4*>(p);
    const u32x4 v = __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4*)p);
    return make_uint4(v.x, v.y, v.z, v.w);
}

// 2^e for e in the range of normal numbers.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

}  // namespace chess
