// Products of few rows (up to 32) with many: serving, a token or some at a time.  What bounds them is reading b once.
//
// A workgroup makes all rows' results of 16 CG columns; its waves take turns along k, by spans of 16 blocks, and add up in LDS in the end, wave by wave, so that
// a sum's order depends on the sizes only.  A wave reads four blocks (64 bytes) of 16 rows of b with one load, and keeps the loads of a span in flight.
// Rows of a come as they are held, or as values: then a lane quantises the block that it brings to the instruction, in registers: some 60 operations for every four
// loads, hidden behind them, where a launch of its own for that takes longer than the product.
#pragma once

#include "zc_mx_product.h"

namespace zc {

constexpr u32 kFewRows = 32, kFewWaves = 8, kSpanOfBlocks = 16;
constexpr int kHeldRows = -1;                    // the type of rows that are held in 4 bits

struct MxFewArgs {
  MxProductArgs p;               // (without a where the rows come as values)
  const void* x;
  u64 x_stride, k;
};

// A block of a row of values as codes, and its scale byte.
template <int TYPE>
__device__ inline u32x4_t mx_block_of_values(const MxFewArgs& a, u64 row, u64 block, u32& scale_byte) {
  using One = typename ValueOf<TYPE>::One;
  using Pack = MxPack<TYPE>;
  constexpr u32 WORDS = TYPE == ZC_F32 ? 32 : 16;
  const One* const p = static_cast<const One*>(a.x) + row * a.x_stride + kBlockValues * block;
  u32 w[WORDS];
  if (kBlockValues * (block + 1) <= a.k) {
#pragma unroll
    for (u32 i = 0; i < WORDS / 4; ++i) {
      const MxSixteen s = reinterpret_cast<const MxSixteen*>(p)[i];
#pragma unroll
      for (u32 j = 0; j < 4; ++j) w[4 * i + j] = s.w[j];
    }
  } else {
    const u32 count = u32(a.k - kBlockValues * block);
#pragma unroll
    for (u32 i = 0; i < WORDS; ++i) {
      if constexpr (TYPE == ZC_F32) {
        w[i] = i < count ? __float_as_uint(p[i]) : 0u;
      } else {
        w[i] = 2 * i < count ? u32(__builtin_bit_cast(u16, p[2 * i])) : 0u;
        if (2 * i + 1 < count) w[i] |= u32(__builtin_bit_cast(u16, p[2 * i + 1])) << 16;
      }
    }
  }
  u32 top = 0;
#pragma unroll
  for (u32 i = 0; i < WORDS; ++i) top = TYPE == ZC_F32 ? max(top, w[i] & 0x7fffffffu) : max_pairs(top, w[i] & 0x7fff7fffu);
  scale_byte = mx_scale(Pack::top_value(top));
  const float scale = scale_value(scale_byte);
  u32x4_t codes;
#pragma unroll
  for (u32 q = 0; q < 4; ++q) {
    u32 eight[WORDS / 4];
#pragma unroll
    for (u32 j = 0; j < WORDS / 4; ++j) eight[j] = w[WORDS / 4 * q + j];
    codes[q] = scale_byte == 255u ? 0u : mx_codes<TYPE>(eight, scale);
  }
  return codes;
}

// The scale bytes of a span of a row, those behind the last block as zeros.
__device__ inline u32x4_t mx_span_scales(const u8* row, u32 first, u32 blocks) {
  u32x4_t w = {0, 0, 0, 0};
  if (first + kSpanOfBlocks <= blocks) {
    struct __attribute__((packed, aligned(4))) Words { u32 w[4]; };
    const Words s = *reinterpret_cast<const Words*>(row + first);
    w = u32x4_t{s.w[0], s.w[1], s.w[2], s.w[3]};
  } else {
#pragma unroll
    for (u32 j = 0; j < 4; ++j) {
      const u32 at = first + 4 * j;
      if (at >= blocks) break;
      w[j] = *reinterpret_cast<const u32*>(row + at);
      if (at + 4 > blocks) w[j] &= (1u << (8 * (blocks - at))) - 1u;
    }
  }
  return w;
}

template <int RG, int CG, int X>
__global__ __launch_bounds__(64 * kFewWaves) void mx_few_kernel(MxFewArgs a) {
  __shared__ f32x4_t parts[kFewWaves * RG * CG * 64];
  const u32 lane = threadIdx.x & 63u, wave = u32(__builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6))), waves = blockDim.x >> 6, in16 = lane & 15u, part = lane >> 4;
  const u64 col0 = u64(blockIdx.x) * (16 * CG);
  const u8* rows_b[CG];
  const u8* scales_b[CG];
#pragma unroll
  for (int c = 0; c < CG; ++c) {
    const u64 col = min(col0 + 16 * c + in16, a.p.n - 1);                      // (columns behind the last one: any, nobody looks at them)
    rows_b[c] = a.p.b + col * a.p.b_stride;
    scales_b[c] = a.p.b_scales + col * a.p.b_scales_stride;
  }
  f32x4_t sum[RG][CG];
#pragma unroll
  for (int r = 0; r < RG; ++r)
#pragma unroll
    for (int c = 0; c < CG; ++c) sum[r][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  for (u32 first = kSpanOfBlocks * wave; first < a.p.blocks; first += kSpanOfBlocks * waves) {
    u32x4_t b[CG][4], sb[CG], sa[RG];
#pragma unroll
    for (int c = 0; c < CG; ++c) {
#pragma unroll
      for (u32 t = 0; t < 4; ++t) {
        const u32 block = first + 4 * t + part;
        b[c][t] = *reinterpret_cast<const u32x4_t*>(rows_b[c] + kMxBytes * (block < a.p.blocks ? block : 0u));
      }
      sb[c] = mx_span_scales(scales_b[c], first, a.p.blocks);
    }
    if constexpr (X == kHeldRows) {
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        sa[r] = u32x4_t{0, 0, 0, 0};
        if (16 * r + in16 < a.p.m) sa[r] = mx_span_scales(a.p.a_scales + (16 * r + in16) * a.p.a_scales_stride, first, a.p.blocks);
      }
    }
#pragma unroll
    for (u32 t = 0; t < 4; ++t) {
      const u32 block = first + 4 * t + part;
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        const u64 row = 16 * r + in16;
        u32x4_t x = {0, 0, 0, 0};
        u32 scale_x = 0;
        if (row < a.p.m && block < a.p.blocks) {
          if constexpr (X == kHeldRows) {
            x = *reinterpret_cast<const u32x4_t*>(a.p.a + row * a.p.a_stride + kMxBytes * block);
            scale_x = sa[r][t] >> (8 * part);
          } else {
            x = mx_block_of_values<X>(a, row, block, scale_x);
          }
        }
#pragma unroll
        for (int c = 0; c < CG; ++c)
          sum[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(b[c][t]), mx_operand(x), sum[r][c], kMxFp4, kMxFp4, 0, int(sb[c][t] >> (8 * part)), 0, int(scale_x));
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RG; ++r)
#pragma unroll
    for (int c = 0; c < CG; ++c) parts[(wave * RG * CG + r * CG + c) * 64 + lane] = sum[r][c];
  __syncthreads();
  for (u32 i = threadIdx.x; i < RG * CG * 64; i += blockDim.x) {
    const u32 group = i >> 6, r = group / CG, c = group % CG;
    f32x4_t s = parts[i];
    for (u32 w = 1; w < waves; ++w) s += parts[w * RG * CG * 64 + i];
    float v[4] = {s[0], s[1], s[2], s[3]};
    const u64 row = 16 * r + in16, col = col0 + 16 * c + 4 * part;
    if (row < a.p.m && col < a.p.n) mx_finish(a.p, row, col, v);
  }
}

}  // namespace zc
