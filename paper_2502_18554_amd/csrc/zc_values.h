// Values of the three floating types that the layer calls read and write, by fours.  gfx950 only.
#pragma once

#include "zc_common.h"

namespace zc {

// Four consecutive values in memory at their own alignment only: global memory takes wide accesses at any address.
struct __attribute__((packed, aligned(4))) F32Four { float v[4]; };
struct __attribute__((packed, aligned(2))) B16Four { __bf16 v[4]; };
struct __attribute__((packed, aligned(2))) H16Four { _Float16 v[4]; };

template <int TYPE> struct ValueOf;
template <> struct ValueOf<ZC_F32> { using One = float; using Four = F32Four; };
template <> struct ValueOf<ZC_BF16> { using One = __bf16; using Four = B16Four; };
template <> struct ValueOf<ZC_F16> { using One = _Float16; using Four = H16Four; };

__host__ __device__ constexpr u32 value_bytes(int type) { return type == ZC_F32 ? 4u : 2u; }

// Stores of a type that is known at run time only (the same for the whole grid).  Rounded to nearest, ties to even.
__device__ inline void store_value(void* base, int type, u64 i, float v) {
  if (type == ZC_F32) static_cast<float*>(base)[i] = v;
  else if (type == ZC_BF16) static_cast<__bf16*>(base)[i] = __bf16(v);
  else static_cast<_Float16*>(base)[i] = _Float16(v);
}
__device__ inline float load_value(const void* base, int type, u64 i) {
  if (type == ZC_F32) return static_cast<const float*>(base)[i];
  if (type == ZC_BF16) return float(static_cast<const __bf16*>(base)[i]);
  return float(static_cast<const _Float16*>(base)[i]);
}

template <int TYPE>
__device__ inline void store_four(void* base, u64 i, const float (&v)[4]) {
  using One = typename ValueOf<TYPE>::One;
  typename ValueOf<TYPE>::Four f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f.v[j] = One(v[j]);
  *reinterpret_cast<typename ValueOf<TYPE>::Four*>(static_cast<One*>(base) + i) = f;
}
__device__ inline void store_four(void* base, int type, u64 i, const float (&v)[4]) {
  if (type == ZC_F32) store_four<ZC_F32>(base, i, v);
  else if (type == ZC_BF16) store_four<ZC_BF16>(base, i, v);
  else store_four<ZC_F16>(base, i, v);
}

// 2^(exponent - 127) for exponents 1 .. 254.
__device__ inline float power_of_two(u32 exponent) { return __uint_as_float(exponent << 23); }
__device__ inline u32 exponent_field(float magnitude) { return __float_as_uint(magnitude) >> 23; }

// What a scale byte stands for: 2^(s - 127), not a number for 255.  (Written so that it takes no branch.)
__device__ inline float scale_value(u32 s) {
  const u32 bits = max(s << 23, 0x00400000u);
  return __uint_as_float(s == 255u ? 0x7fc00000u : bits);
}
// Of a block that has a scale: what its values are divided by.  (Of one that has none anything: its codes are zeros, see codes_if.)
__device__ inline float divisor_value(u32 s) { return __uint_as_float(max(s << 23, 0x00400000u)); }
__device__ inline u32 codes_if(u32 s, u32 codes) { return codes & (s == 255u ? 0u : ~0u); }

}  // namespace zc
