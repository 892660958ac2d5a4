// One AdamW step over many tensors in one launch, with first and second moments in 32 bits or in 8.
//
// For every value (all steps in binary32, each rounded by itself; c.* come from binary64 on the host):
//   g = grad x scale;  m' = b1 m + (1 - b1) g;  v' = b2 v + ((1 - b2) g) g;  r = sqrt(v')
//   p' = p (1 - lr decay) - (lr / (1 - b1^t)) (m' / (r / sqrt(1 - b2^t) + eps))
// In 8 bits a state holds m and r (the root: half the exponent range of v) as e4m3 codes, 32 values a block, the stream
// format's own block, with one power of two a block for a scale.  The largest magnitude of a block lands in [128, 256) of the format's 448,
// so that nothing saturates, rounding up included; scaling by powers of two is exact, so that a state that no gradient touches only decays.
// A value is 3 bits of fraction: by nearest rounding a second moment that changes by less than 6 % a step never
// moves, which with b2 = 0.999 is nearly always.  So rounding is by default up or down with the probability that keeps the
// mean, from 16 hashed bits per value and state (seed, step, place in the state).
#pragma once

#include "zc_values.h"

namespace zc {

constexpr int kAdamwThreads = 256;
constexpr int kAdamwFours = 4;                                       // a lane's groups of four values
constexpr u32 kAdamwTile = kAdamwThreads * 4 * kAdamwFours;
constexpr int kAdamwTensors = 80;                                    // of one launch: their table travels in the kernel's arguments

struct AdamwScalars {
  float b1, c1, b2, c2;          // c = 1 - b
  float keep;                    // 1 - lr decay
  float rate;                    // lr / (1 - b1^t)
  float root;                    // 1 / sqrt(1 - b2^t)
  float eps;
};

struct AdamwTensor {
  void* param;
  const void* grad;
  void* copy;
  u64 n;
  u32 first_block;               // in the state
};

struct AdamwArgs {
  u32 first_tile[kAdamwTensors];
  AdamwTensor tensor[kAdamwTensors];
  AdamwScalars c;
  u32 tensors;
  int copy_type;
  u8* state;
  u64 blocks;                    // of the whole state
  const float* grad_scale;
  u32 key;
  u32 stochastic;
};
static_assert(sizeof(AdamwArgs) <= 4096);

// Scrambles a word (odd multipliers from the fractional parts of sqrt 2 and sqrt 3, folded by shifts).
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

template <int TYPE>
__device__ inline void load_four(const void* base, u64 i, u64 n, float (&v)[4]) {
  using One = typename ValueOf<TYPE>::One;
  const One* const p = static_cast<const One*>(base) + i;
  if (i + 4 <= n) {
    const typename ValueOf<TYPE>::Four f = *reinterpret_cast<const typename ValueOf<TYPE>::Four*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = float(f.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < n ? float(p[j]) : 0.0f;
  }
}

// Largest magnitude as bits (every NaN counts as more than infinity): of a lane's four values, and of 8 neighbouring lanes, in pairs, in fours
// and with the mirrored half of the eight.
__device__ inline u32 top_of_four(const float (&x)[4]) {
  u32 t = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) t = max(t, __float_as_uint(x[j]) & 0x7fffffffu);
  return t;
}
__device__ inline u32 top_of_eight(u32 x) {
  x = max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, true)));
  x = max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xf, 0xf, true)));
  return max(x, u32(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xf, 0xf, true)));
}

// Scale byte of a block in 8 bits, from the largest magnitude.
__device__ inline u32 adamw_scale(u32 top) {
  const u32 e = top >> 23;
  return e == 255u ? 255u : e > 7u ? e - 7u : 0u;
}

// A magnitude scaled into the range of e4m3, on that format's grid: quanta of 2^-3 of the binade, of 2^-9 below 2^-6.
__device__ inline float on_grid(float y, u32 random16, bool stochastic) {
  const u32 e = max(exponent_field(y), 121u);
  const float t = y * power_of_two(257u - e);
  const float k = stochastic ? floorf(t + float(random16) * 0x1p-16f) : rintf(t);
  return k * power_of_two(e - 3u);
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

template <int P, int G, int BITS>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a) {
  float scale = 1.0f;
  if (a.grad_scale) {
    scale = *a.grad_scale;
    if (!(fabsf(scale) <= 3.402823466e38f)) return;                  // (not a number or infinite: no step)
  }
  // The tensor that the workgroup's tile lies in: the last one that begins at or before it.
  const u32 lane = threadIdx.x & 63u;
  u32 t = 0;
  for (u32 i = 0; i < a.tensors; i += 64)
    t += u32(__popcll(__ballot(i + lane < a.tensors && a.first_tile[i + lane] <= blockIdx.x)));
  t = u32(__builtin_amdgcn_readfirstlane(int(t))) - 1u;
  const AdamwTensor x = a.tensor[t];
  const u64 tile_at = u64(blockIdx.x - a.first_tile[t]) * kAdamwTile;
  const u64 padded = num_blocks(x.n) * kBlockValues;
  const u64 state_at = u64(x.first_block) * kBlockValues;
  const AdamwScalars c = a.c;
#pragma unroll
  for (int u = 0; u < kAdamwFours; ++u) {
    const u64 i = tile_at + u64(u) * (kAdamwThreads * 4) + threadIdx.x * 4u;
    const bool here = i < padded;
    const u64 s = state_at + i, block = s / kBlockValues;
    float p[4], g[4], m[4], v[4], r[4];
    load_four<P>(x.param, i, x.n, p);
    load_four<G>(x.grad, i, x.n, g);
    if (BITS == 32) {
      const float* const ms = reinterpret_cast<const float*>(a.state);
      const float* const vs = reinterpret_cast<const float*>(a.state + adamw_second(a.blocks, 32));
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = here ? ms[s + j] : 0.0f, v[j] = here ? vs[s + j] : 0.0f;
    } else {
      const u8* const scales = a.state + adamw_scales(a.blocks);
      const u32 mc = here ? *reinterpret_cast<const u32*>(a.state + s) : 0u;
      const u32 rc = here ? *reinterpret_cast<const u32*>(a.state + adamw_second(a.blocks, 8) + s) : 0u;
      values_of_codes(mc, scale_value(here ? scales[block] : 0u), m);
      values_of_codes(rc, scale_value(here ? scales[pad16(a.blocks) + block] : 0u), v);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = v[j] * v[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float gs = a.grad_scale ? g[j] * scale : g[j];
      m[j] = m[j] * c.b1 + gs * c.c1;
      v[j] = v[j] * c.b2 + (gs * c.c2) * gs;
      r[j] = sqrtf(v[j]);
      p[j] = p[j] * c.keep - (m[j] / (r[j] * c.root + c.eps)) * c.rate;
    }
    if (i + 4 <= x.n) {
      store_four<P>(x.param, i, p);
      if (x.copy) store_four(x.copy, a.copy_type, i, p);
    } else {
      for (int j = 0; j < 4; ++j)
        if (i + j < x.n) {
          store_value(x.param, P, i + j, p[j]);
          if (x.copy) store_value(x.copy, a.copy_type, i + j, p[j]);
        }
    }
    if (BITS == 32) {
      float* const ms = reinterpret_cast<float*>(a.state);
      float* const vs = reinterpret_cast<float*>(a.state + adamw_second(a.blocks, 32));
      if (here) {
#pragma unroll
        for (int j = 0; j < 4; ++j) ms[s + j] = m[j], vs[s + j] = v[j];
      }
    } else {
      u8* const scales = a.state + adamw_scales(a.blocks);
      const u32 sm = adamw_scale(top_of_eight(top_of_four(m))), sr = adamw_scale(top_of_eight(top_of_four(r)));
      float cm[4], cr[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32 z = mixed_word(u32(s + j) * 0x9E3779B1u + a.key);
        cm[j] = copysignf(on_grid(fabsf(m[j]) * power_of_two(254u - min(sm, 253u)), z & 0xffffu, a.stochastic), m[j]);
        cr[j] = on_grid(r[j] * power_of_two(254u - min(sr, 253u)), z >> 16, a.stochastic);
        if (r[j] > 0.0f) cr[j] = fmaxf(cr[j], 0x1p-9f);              // (a denominator never becomes none)
      }
      if (here) {
        *reinterpret_cast<u32*>(a.state + s) = sm == 255u ? 0u : four_codes(cm);
        *reinterpret_cast<u32*>(a.state + adamw_second(a.blocks, 8) + s) = sr == 255u ? 0u : four_codes(cr);
        if ((lane & 7u) == 0) {
          scales[block] = u8(sm);
          scales[pad16(a.blocks) + block] = u8(sr);
        }
      }
    }
  }
}

}  // namespace zc
