// One AdamW step over many tensors in one launch, with first and second moments in 32 bits or in 8.
//
// For every value (all steps in binary32, each rounded by itself, except that the quotient is a product with the reciprocal instruction's result, within
// three units in the last place, and the root, where it is not stored, is the instruction's, within one; c.* come from binary64 on the host):
//   g = grad x scale;  m' = b1 m + (1 - b1) g;  v' = b2 v + ((1 - b2) g) g;  r = sqrt(v')
//   p' = p (1 - lr decay) - (lr / (1 - b1^t)) (m' / (r / sqrt(1 - b2^t) + eps))
// In 8 bits a state holds m and r (the root: half the exponent range of v) as e4m3 codes, 32 values a block, the stream
// format's own block, with one power of two a block for a scale.  The largest magnitude of a block lands in [128, 256) of the format's 448,
// so that nothing saturates, rounding up included; scaling by powers of two is exact, so that a state that no gradient touches only decays.
// A value is 3 bits of fraction: by nearest rounding a second moment that changes by less than 6 % a step never
// moves, which with b2 = 0.999 is nearly always.  So rounding is by default up or down with the probability that keeps the
// mean, from 16 hashed bits per value and state (seed, step, place in the state).
//
// States in 32 bits: bound by memory (50 M values of 32 bits, gradients and copies of 16, 273 us, 5.1 TB/s, what a copy reaches; 4 groups of four values a lane, all of
// whose loads are on their way before the first is used; 9 M values of 16 bits with gradients likewise 30.4 us, 6.5 TB/s, partly from the last cache).  In 8 bits with weights of 32 bits as
// well (67 M values 205 us, 5.3 TB/s), with weights of 16 bits by arithmetic (9 M values 24.8 us, 3.7 TB/s, 92 vector instructions a value, 85 % of their issue time; the kind of rounding is
// asked for at every value, and the hash's place costs a multiplication that an addition could be).  The tensors' table travels in the kernel's arguments, so that a step of
// 110 tensors is one launch that nothing has to be copied for: 24 tensors of 1000 values 2.5 us.
#pragma once

#include "zc_values.h"

namespace zc {

constexpr int kAdamwThreads = 256;
constexpr int kAdamwFours = 4;                                       // a lane's groups of four values
constexpr u32 kAdamwTile = kAdamwThreads * 4 * kAdamwFours;
constexpr int kAdamwTensors = 110;                                   // of one launch: their table travels in the kernel's arguments
constexpr u64 kAdamwMost = u64(1) << 31;                             // values of an entry: a longer tensor has several

struct AdamwScalars {
  float b1, c1, b2, c2;          // c = 1 - b
  float keep;                    // 1 - lr decay
  float rate;                    // lr / (1 - b1^t)
  float root;                    // 1 / sqrt(1 - b2^t)
  float eps;
};

struct AdamwArgs {
  AdamwScalars c;
  u32 tensors;
  int copy_type;
  u8* state;
  u64 blocks;                    // of the whole state
  const float* grad_scale;
  u32 key;
  u32 stochastic;
  u32 first_tile[kAdamwTensors];
  u32 first_block[kAdamwTensors];          // in the state
  u32 n[kAdamwTensors];
  void* param[kAdamwTensors];
  const void* grad[kAdamwTensors];
  void* copy[kAdamwTensors];
};
static_assert(sizeof(AdamwArgs) <= 4096);

// Scrambles a word: the method of xxHash32's last mixing (Y. Collet: shifts by 15, 13 and 16 with a multiplication behind the first two), with other odd multipliers, the
// fractional parts of sqrt 2 and sqrt 3.  Places are spread by that hash's first prime, 0x9E3779B1, next to 2^32 over the golden ratio (multiplicative hashing, Knuth).
__host__ __device__ inline u32 mixed_word(u32 z) {
  z ^= z >> 15;
  z *= 0x6A09E667u;
  z ^= z >> 13;
  z *= 0xBB67AE85u;
  return z ^ (z >> 16);
}
__host__ inline u32 adamw_key(u64 seed, u64 step) {
  return mixed_word(mixed_word(mixed_word(u32(seed)) + u32(seed >> 32)) + u32(step));
}

// Offsets of the parts of a state of `blocks` blocks: m | v in 32 bits; m codes | r codes | m scales | r scales in 8.
__host__ __device__ inline u64 adamw_second(u64 blocks, int bits) { return blocks * kBlockValues * (bits / 8); }
__host__ __device__ inline u64 adamw_scales(u64 blocks) { return 2 * blocks * kBlockValues; }
__host__ __device__ inline u64 adamw_bytes(u64 blocks, int bits) {
  return bits == 32 ? 2 * adamw_second(blocks, 32) : adamw_scales(blocks) + 2 * pad16(blocks);
}

// Largest magnitude of a lane's four values, and of 8 neighbouring lanes (in pairs, in fours and with the mirrored half of the eight), as bits without their sign,
// shifted up by one: every NaN counts as more than infinity.
__device__ inline u32 top_of_four(const float (&x)[4]) {
  u32 t = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) t = max(t, __float_as_uint(x[j]) << 1);
  return t;
}
__device__ inline u32 top_of_eight(u32 x) {
  x = max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, true)));
  x = max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xf, 0xf, true)));
  return max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xf, 0xf, true)));
}

// Scale byte of a block in 8 bits, from the largest magnitude.
__device__ inline u32 adamw_scale(u32 top) {
  const u32 e = top >> 24;
  return e == 255u ? 255u : max(e, 7u) - 7u;
}

// A magnitude scaled into the range of e4m3, on that format's grid: quanta of 2^-3 of the binade, of 2^-9 below 2^-6.
__device__ inline float nearest_on_grid(float y) {
  const u32 e = max(exponent_field(y), 121u);
  return rintf(y * power_of_two(257u - e)) * power_of_two(e - 3u);
}
// Up when the 16 random bits and the way from the grid's lower neighbour reach the upper one: floor(y / quantum + random / 65536) quanta.  The last place that stays of a
// binary32 is its bit 20, so that is a sum of integers, except below 2^-6, where the quanta no longer shrink.
__device__ inline float random_on_grid(float y, u32 random16) {
  const u32 bits = __float_as_uint(y) + (random16 << 4);
  const float low = floorf(__builtin_fmaf(float(random16), 0x1p-16f, y * 0x1p9f)) * 0x1p-9f;
  return y < 0x1p-6f ? low : __uint_as_float(bits & 0xfff00000u);
}

__device__ inline u32 four_codes(const float (&v)[4]) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return u32(__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true));
}
__device__ inline void values_of_codes(u32 codes, float scale, float (&v)[4]) {
  const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), false);
  const auto high = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), true);
  v[0] = low[0] * scale;
  v[1] = low[1] * scale;
  v[2] = high[0] * scale;
  v[3] = high[1] * scale;
}

// The root to within a unit in the last place.  The instruction takes subnormal numbers for zeros: small ones are scaled by 2^32.  (1 M values of 32 bits 5.3 us; by the
// correctly rounded root 5.8, by the instruction alone 5.2; 50 M 240, 242 and 240.)
__device__ inline float root_of(float x) {
  const bool small = x < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(x * (small ? 0x1p32f : 1.0f)) * (small ? 0x1p-16f : 1.0f);
}

// Four values as they lie in memory, and as numbers.
template <int TYPE>
__device__ inline typename ValueOf<TYPE>::Four load_raw(const void* base, u32 i) {
  using One = typename ValueOf<TYPE>::One;
  return *reinterpret_cast<const typename ValueOf<TYPE>::Four*>(static_cast<const One*>(base) + i);
}
template <int TYPE>
__device__ inline void load_some(const void* base, u32 i, u32 n, typename ValueOf<TYPE>::Four& to) {
  using One = typename ValueOf<TYPE>::One;
#pragma unroll
  for (u32 j = 0; j < 4; ++j)
    if (i + j < n) to.v[j] = static_cast<const One*>(base)[i + j];
}

// A state's share of a lane.
template <int BITS> struct AdamwHeld;
template <> struct AdamwHeld<32> {
  f32x4_t m, v;
  __device__ void load(const AdamwArgs& a, u64 at) {
    m = *reinterpret_cast<const f32x4_t*>(a.state + 4 * at);
    v = *reinterpret_cast<const f32x4_t*>(a.state + adamw_second(a.blocks, 32) + 4 * at);
  }
};
template <> struct AdamwHeld<8> {
  u32 m, r, m_scale, r_scale;
  __device__ void load(const AdamwArgs& a, u64 at) {
    const u8* const scales = a.state + adamw_scales(a.blocks) + at / kBlockValues;
    m = *reinterpret_cast<const u32*>(a.state + at);
    r = *reinterpret_cast<const u32*>(a.state + adamw_second(a.blocks, 8) + at);
    m_scale = scales[0];
    r_scale = scales[pad16(a.blocks)];
  }
};

struct AdamwEntry {
  void* param;
  const void* grad;
  void* copy;
  u32 n, tile_at;
  u64 state_at;
};

// A workgroup's tile of an entry.  WHOLE: every value of it exists.  All loads come before the first use of one.
template <int P, int G, int BITS, bool WHOLE>
__device__ __forceinline__ void adamw_tile(const AdamwArgs& a, const AdamwEntry& x, float scale) {
  const AdamwScalars c = a.c;
  const u32 padded = (x.n + kBlockValues - 1u) & ~u32(kBlockValues - 1);
  typename ValueOf<P>::Four raw_p[kAdamwFours] = {};
  typename ValueOf<G>::Four raw_g[kAdamwFours] = {};
  AdamwHeld<BITS> held[kAdamwFours] = {};
#pragma unroll
  for (int u = 0; u < kAdamwFours; ++u) {
    const u32 i = x.tile_at + u32(u) * (kAdamwThreads * 4) + threadIdx.x * 4u;
    if (WHOLE || i + 4 <= x.n) {
      raw_p[u] = load_raw<P>(x.param, i);
      raw_g[u] = load_raw<G>(x.grad, i);
    }
    if (WHOLE || i < padded) held[u].load(a, x.state_at + i);
  }
  if (!WHOLE && (x.n & 3u)) {                                        // (one lane of the last tile)
#pragma unroll
    for (int u = 0; u < kAdamwFours; ++u) {
      const u32 i = x.tile_at + u32(u) * (kAdamwThreads * 4) + threadIdx.x * 4u;
      if (i < x.n && i + 4 > x.n) {
        load_some<P>(x.param, i, x.n, raw_p[u]);
        load_some<G>(x.grad, i, x.n, raw_g[u]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kAdamwFours; ++u) {
    const u32 i = x.tile_at + u32(u) * (kAdamwThreads * 4) + threadIdx.x * 4u;
    if (!WHOLE && x.tile_at + u32(u) * (kAdamwThreads * 4) >= padded) break;
    const u64 s = x.state_at + i, block = s / kBlockValues;
    float p[4], g[4], m[4], v[4], r[4];
    if constexpr (BITS == 32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = held[u].m[j], v[j] = held[u].v[j];
    } else {
      values_of_codes(held[u].m, scale_value(held[u].m_scale), m);
      values_of_codes(held[u].r, scale_value(held[u].r_scale), v);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = v[j] * v[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p[j] = float(raw_p[u].v[j]);
      g[j] = float(raw_g[u].v[j]) * scale;
      m[j] = m[j] * c.b1 + g[j] * c.c1;
      v[j] = v[j] * c.b2 + (g[j] * c.c2) * g[j];
      r[j] = BITS == 8 ? sqrtf(v[j]) : root_of(v[j]);
      p[j] = p[j] * c.keep - (m[j] * __builtin_amdgcn_rcpf(r[j] * c.root + c.eps)) * c.rate;
    }
    if (WHOLE || i + 4 <= x.n) {
      store_four<P>(x.param, i, p);
      if (x.copy) store_four(x.copy, a.copy_type, i, p);
    } else if (i < x.n) {
#pragma unroll
      for (u32 j = 0; j < 4; ++j)
        if (i + j < x.n) {
          store_value(x.param, P, i + j, p[j]);
          if (x.copy) store_value(x.copy, a.copy_type, i + j, p[j]);
        }
    }
    if constexpr (BITS == 32) {
      if (WHOLE || i < padded) {
        *reinterpret_cast<f32x4_t*>(a.state + 4 * s) = f32x4_t{m[0], m[1], m[2], m[3]};
        *reinterpret_cast<f32x4_t*>(a.state + adamw_second(a.blocks, 32) + 4 * s) = f32x4_t{v[0], v[1], v[2], v[3]};
      }
    } else {
      const u32 sm = adamw_scale(top_of_eight(top_of_four(m))), sr = adamw_scale(top_of_eight(top_of_four(r)));
      float cm[4], cr[4];
      const float up_m = power_of_two(254u - min(sm, 253u)), up_r = power_of_two(254u - min(sr, 253u));
      const u32 place = u32(s) * 0x9E3779B1u + a.key;
#pragma unroll
      for (u32 j = 0; j < 4; ++j) {
        const float ym = fabsf(m[j]) * up_m, yr = r[j] * up_r;
        if (a.stochastic) {
          const u32 z = mixed_word(place + j * 0x9E3779B1u);
          cm[j] = random_on_grid(ym, z & 0xffffu);
          cr[j] = random_on_grid(yr, z >> 16);
        } else {
          cm[j] = nearest_on_grid(ym);
          cr[j] = nearest_on_grid(yr);
        }
        cm[j] = copysignf(cm[j], m[j]);
        cr[j] = fmaxf(cr[j], r[j] > 0.0f ? 0x1p-9f : 0.0f);          // (a denominator never becomes none)
      }
      if (WHOLE || i < padded) {
        u8* const scales = a.state + adamw_scales(a.blocks) + block;
        *reinterpret_cast<u32*>(a.state + s) = codes_if(sm, four_codes(cm));
        *reinterpret_cast<u32*>(a.state + adamw_second(a.blocks, 8) + s) = codes_if(sr, four_codes(cr));
        if ((threadIdx.x & 7u) == 0) {
          scales[0] = u8(sm);
          scales[pad16(a.blocks)] = u8(sr);
        }
      }
    }
  }
}

template <int P, int G, int BITS>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a) {
  float scale = 1.0f;
  if (a.grad_scale) scale = *a.grad_scale;
  // The entry that the workgroup's tile lies in: the last one that begins at or before it.
  const u32 lane = threadIdx.x & 63u;
  u32 t = 0;
  for (u32 i = 0; i < a.tensors; i += 64)
    t += u32(__popcll(__ballot(i + lane < a.tensors && a.first_tile[i + lane] <= blockIdx.x)));
  t = u32(__builtin_amdgcn_readfirstlane(int(t))) - 1u;
  if (!(fabsf(scale) <= 3.402823466e38f)) return;                    // (not a number or infinite: no step)
  const AdamwEntry x = {a.param[t], a.grad[t], a.copy[t], a.n[t], (blockIdx.x - a.first_tile[t]) * kAdamwTile, u64(a.first_block[t]) * kBlockValues};
  if (x.tile_at + kAdamwTile <= x.n) adamw_tile<P, G, BITS, true>(a, x, scale);
  else adamw_tile<P, G, BITS, false>(a, x, scale);
}

}  // namespace zc
