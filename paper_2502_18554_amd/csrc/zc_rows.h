// Rows of values of three types, by pieces of eight, and sums over the lanes that share a row.  gfx950 only.
#pragma once

#include "zc_values.h"

namespace zc {

// Eight consecutive values as they lie in memory, at their own alignment: 32 bytes or 16.
template <bool WIDE> struct RawEight;
template <> struct RawEight<true> { u32 w[8]; };
template <> struct RawEight<false> { u32 w[4]; };
struct __attribute__((packed, aligned(4))) F32EightAt { u32 w[8]; };
struct __attribute__((packed, aligned(2))) B16EightAt { u32 w[4]; };

struct __attribute__((packed, aligned(4))) W4At { u32 w[4]; };
struct __attribute__((packed, aligned(4))) W2At { u32 w[2]; };
struct __attribute__((packed, aligned(2))) H4At { u32 w[2]; };
struct __attribute__((packed, aligned(2))) H2At { u32 w; };

// The first `left` of them (8 and more: all, 0 and less: none); zeros behind.  The end of a row comes by four, two and one: few instructions, for kernels that run for a few us wait for
// instructions that they have not seen yet.
template <bool WIDE>
__device__ inline RawEight<WIDE> load_eight(const void* base, u64 at, i32 left) {
  RawEight<WIDE> r = {};
  if (left >= 8) {
    if constexpr (WIDE) {
      const F32EightAt v = *reinterpret_cast<const F32EightAt*>(static_cast<const float*>(base) + at);
#pragma unroll
      for (int j = 0; j < 8; ++j) r.w[j] = v.w[j];
    } else {
      const B16EightAt v = *reinterpret_cast<const B16EightAt*>(static_cast<const u16*>(base) + at);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[j] = v.w[j];
    }
  } else if (left > 0) {
    const bool four = left & 4, two = left & 2, one = left & 1;
    if constexpr (WIDE) {
      const u32* const from = static_cast<const u32*>(base) + at;
      u32 a0 = 0, a1 = 0, a2 = 0, a3 = 0, b0 = 0, b1 = 0, c = 0;
      if (four) {
        const W4At v = *reinterpret_cast<const W4At*>(from);
        a0 = v.w[0], a1 = v.w[1], a2 = v.w[2], a3 = v.w[3];
      }
      if (two) {
        const W2At v = *reinterpret_cast<const W2At*>(from + (left & 4));
        b0 = v.w[0], b1 = v.w[1];
      }
      if (one) c = from[left & 6];
      const u32 n0 = two ? b0 : c, n1 = b1, n2 = two ? c : 0u;
      r.w[0] = four ? a0 : n0;
      r.w[1] = four ? a1 : n1;
      r.w[2] = four ? a2 : n2;
      r.w[3] = a3;
      r.w[4] = four ? n0 : 0u;
      r.w[5] = four ? n1 : 0u;
      r.w[6] = four ? n2 : 0u;
    } else {
      const u16* const from = static_cast<const u16*>(base) + at;
      u32 a0 = 0, a1 = 0, b = 0, c = 0;
      if (four) {
        const H4At v = *reinterpret_cast<const H4At*>(from);
        a0 = v.w[0], a1 = v.w[1];
      }
      if (two) b = reinterpret_cast<const H2At*>(from + (left & 4))->w;
      if (one) c = from[left & 6];
      const u32 n0 = two ? b : c, n1 = two ? c : 0u;
      r.w[0] = four ? a0 : n0;
      r.w[1] = four ? a1 : n1;
      r.w[2] = four ? n0 : 0u;
      r.w[3] = four ? n1 : 0u;
    }
  }
  return r;
}

// As numbers.  (Which 16-bit type it is, is the same for the whole grid.)
template <bool WIDE>
__device__ inline void numbers_of(const RawEight<WIDE>& r, int type, float (&v)[8]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r.w[j]);
  } else if (type == ZC_BF16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = float(__builtin_bit_cast(_Float16, u16(r.w[j / 2] >> (16 * (j & 1)))));
  }
}

// Two numbers, each rounded once, as a word.
template <typename ONE>
__device__ inline u32 word_of_two(float low, float high) {
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef ONE Pair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u32, __builtin_convertvector((Two{low, high}), Pair));
}

// Eight numbers, each rounded once.
template <bool WIDE>
__device__ inline RawEight<WIDE> rounded_eight(int type, const float (&v)[8]) {
  RawEight<WIDE> r;
  if constexpr (WIDE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j] = __float_as_uint(v[j]);
  } else if (type == ZC_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) r.w[j] = word_of_two<__bf16>(v[2 * j], v[2 * j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r.w[j] = word_of_two<_Float16>(v[2 * j], v[2 * j + 1]);
  }
  return r;
}
template <bool WIDE>
__device__ inline void store_raw_eight(void* base, u64 at, i32 left, const RawEight<WIDE>& r) {
  if (left >= 8) {
    if constexpr (WIDE) {
      F32EightAt v;
#pragma unroll
      for (int j = 0; j < 8; ++j) v.w[j] = r.w[j];
      *reinterpret_cast<F32EightAt*>(static_cast<float*>(base) + at) = v;
    } else {
      B16EightAt v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v.w[j] = r.w[j];
      *reinterpret_cast<B16EightAt*>(static_cast<u16*>(base) + at) = v;
    }
  } else if (left > 0) {
    const bool four = left & 4, two = left & 2;
    if constexpr (WIDE) {
      u32* const to = static_cast<u32*>(base) + at;
      if (four) *reinterpret_cast<W4At*>(to) = W4At{{r.w[0], r.w[1], r.w[2], r.w[3]}};
      u32 n0 = r.w[0], n1 = r.w[1], n2 = r.w[2];
      if (four) n0 = r.w[4], n1 = r.w[5], n2 = r.w[6];
      if (two) {
        *reinterpret_cast<W2At*>(to + (left & 4)) = W2At{{n0, n1}};
        n0 = n2;
      }
      if (left & 1) to[left & 6] = n0;
    } else {
      u16* const to = static_cast<u16*>(base) + at;
      if (four) *reinterpret_cast<H4At*>(to) = H4At{{r.w[0], r.w[1]}};
      u32 n0 = r.w[0], n1 = r.w[1];
      if (four) n0 = r.w[2], n1 = r.w[3];
      if (two) {
        reinterpret_cast<H2At*>(to + (left & 4))->w = n0;
        n0 = n1;
      }
      if (left & 1) to[left & 6] = u16(n0);
    }
  }
}
template <bool WIDE>
__device__ inline void store_eight(void* base, int type, u64 at, i32 left, const float (&v)[8]) {
  store_raw_eight<WIDE>(base, at, left, rounded_eight<WIDE>(type, v));
}

// Of a type that is known at run time only.
__device__ inline void load_numbers(const void* base, int type, u64 at, i32 left, float (&v)[8]) {
  if (type == ZC_F32) numbers_of<true>(load_eight<true>(base, at, left), type, v);
  else numbers_of<false>(load_eight<false>(base, at, left), type, v);
}
__device__ inline void store_numbers(void* base, int type, u64 at, i32 left, const float (&v)[8]) {
  if (type == ZC_F32) store_eight<true>(base, type, at, left, v);
  else store_eight<false>(base, type, at, left, v);
}

// P pieces of a row, `apart` values from one to the next: all of them are asked for before the first is looked at, also where the type is known at run time only.
template <bool WIDE, int P>
__device__ inline void load_pieces_of(const void* base, int type, u64 at, u64 apart, const i32 (&left)[P], float (&v)[P][8]) {
  RawEight<WIDE> raw[P];
#pragma unroll
  for (int p = 0; p < P; ++p) raw[p] = load_eight<WIDE>(base, at + p * apart, left[p]);
#pragma unroll
  for (int p = 0; p < P; ++p) numbers_of<WIDE>(raw[p], type, v[p]);
}
template <int P>
__device__ inline void load_pieces(const void* base, int type, u64 at, u64 apart, const i32 (&left)[P], float (&v)[P][8]) {
  if (type == ZC_F32) load_pieces_of<true, P>(base, type, at, apart, left, v);
  else load_pieces_of<false, P>(base, type, at, apart, left, v);
}

// How many of a row's values there are from a piece's first on, 8 at most.
__device__ inline i32 left_of(u64 cols, u64 col) { return col >= cols ? 0 : i32(cols - col < 8 ? cols - col : 8); }

// Sums over 16 neighbouring lanes, over a wave; every lane has them, the same bits in all.
__device__ inline float swapped(float x, u32 o) { return x + __uint_as_float(o); }
__device__ inline float sum_of_16(float x) {
  x = swapped(x, dpp_mov<kDppQuadSwap1>(__float_as_uint(x)));
  x = swapped(x, dpp_mov<kDppQuadSwap2>(__float_as_uint(x)));
  x = swapped(x, dpp_mov<kDppRowHalfMirror>(__float_as_uint(x)));
  return swapped(x, dpp_mov<kDppRowMirror>(__float_as_uint(x)));
}
__device__ inline float sum_of_wave(float x) {
  x = sum_of_16(x);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace zc
