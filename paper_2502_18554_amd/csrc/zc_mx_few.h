// Products of few rows (up to 32) with many: serving, a token or some at a time.  What bounds them is reading b once.
//
// A workgroup makes all rows' results of 16 CG columns; its waves take turns along k, by spans of 16 blocks, and add up in LDS in the end, wave by wave, so that
// a sum's order depends on the sizes only.  A wave reads four blocks (64 bytes) of 16 rows of b with one load.
// Rows of a come as they are held, or (up to 8) as values: then a lane quantises the block that it brings to the instruction, in registers, some 60 operations a block,
// where a launch of its own for that takes half as long as the product.
// Bound by loads that wait for each other, more than by their bytes.  The source asks for all loads of a span ahead of the first use; compiled, they come in rounds, in 60 registers of the
// 256 that a lane could have: of a row of 16-bit values the four steps one after the other, each loaded, waited for and quantised, then the scales and two loads of b, then the other two: seven
// rounds a span; of 32 held rows by 64 columns, in 120 registers, seven waits for all that is on its way.
// 1 row x 4096 x 4096 4.3 us, held 3.3 (9 MB at 2.7 TB/s; some 2 of it are a launch's); 24 held rows x 16384 x 4096 10.9 us (36 MB at 3.4 TB/s).
#pragma once

#include "zc_mx_product.h"

namespace zc {

constexpr u64 kMostFewStride = u64(1) << 24;     // (8 rows of values are less than 2^32 bytes)
constexpr u32 kFewRows = 32, kFewValueRows = 8, kFewWaves = 8, kSpanOfBlocks = 16;
constexpr int kHeldRows = -1;                    // the type of rows that are held in 4 bits

struct MxFewArgs {
  MxProductArgs p;               // (without a where the rows come as values)
  const void* x;
  u64 x_stride, k;
  u32 steps;                     // of four blocks that a wave takes in turn where the rows come as values: 4 (a span), 2 or 1
};

// What a lane brings of a: a block of a row as it comes, and then as codes with its scale byte.
template <int X>
struct MxRaw {
  static constexpr u32 WORDS = X == ZC_F32 ? 32 : 16;
  u32 w[WORDS];
};
template <>
struct MxRaw<kHeldRows> {
  u32x4_t codes;
};

// The values of a block at `at` (bytes from the first row's begin; a lane that has none is beyond the buffer, where all is zero); of the last, incomplete block of a row
// its `count` values one by one.
template <int TYPE>
__device__ inline void mx_load_values(__amdgpu_buffer_rsrc_t from, u32 at, MxRaw<TYPE>& to) {
#pragma unroll
  for (u32 i = 0; i < MxRaw<TYPE>::WORDS / 4; ++i) {
    const u32x4_t s = __builtin_amdgcn_raw_buffer_load_b128(from, at == ~0u ? at : at + 16 * i, 0, 0);
#pragma unroll
    for (u32 j = 0; j < 4; ++j) to.w[4 * i + j] = s[j];
  }
}
template <int TYPE>
__device__ inline void mx_load_some_values(__amdgpu_buffer_rsrc_t from, u32 at, u32 count, MxRaw<TYPE>& to) {
#pragma unroll
  for (u32 i = 0; i < MxRaw<TYPE>::WORDS; ++i) {
    if constexpr (TYPE == ZC_F32) {
      to.w[i] = __builtin_amdgcn_raw_buffer_load_b32(from, at == ~0u || i >= count ? ~0u : at + 4 * i, 0, 0);
    } else {
      const u32 low = __builtin_amdgcn_raw_buffer_load_b16(from, at == ~0u || 2 * i >= count ? ~0u : at + 4 * i, 0, 0);
      const u32 high = __builtin_amdgcn_raw_buffer_load_b16(from, at == ~0u || 2 * i + 1 >= count ? ~0u : at + 4 * i + 2, 0, 0);
      to.w[i] = (low & 0xffffu) | high << 16;
    }
  }
}

template <int TYPE>
__device__ inline u32x4_t mx_block_of_values(const MxRaw<TYPE>& raw, u32& scale_byte) {
  using Pack = MxPack<TYPE>;
  constexpr u32 WORDS = MxRaw<TYPE>::WORDS;
  const u32 (&w)[WORDS] = raw.w;
  u32 top = 0;
#pragma unroll
  for (u32 i = 0; i < WORDS; ++i) top = TYPE == ZC_F32 ? max(top, w[i] & 0x7fffffffu) : max_pairs(top, w[i] & 0x7fff7fffu);
  scale_byte = mx_scale(Pack::top_value(top));
  const float scale = divisor_value(scale_byte);
  u32x4_t codes;
#pragma unroll
  for (u32 q = 0; q < 4; ++q) {
    u32 eight[WORDS / 4];
#pragma unroll
    for (u32 j = 0; j < WORDS / 4; ++j) eight[j] = w[WORDS / 4 * q + j];
    codes[q] = codes_if(scale_byte, mx_codes<TYPE>(eight, scale));
  }
  return codes;
}

// The scale bytes of a span of a row, those behind the last block as zeros.
template <bool WHOLE>
__device__ inline u32x4_t mx_span_scales(const u8* row, u32 first, u32 blocks) {
  u32x4_t w = {0, 0, 0, 0};
  if (WHOLE || first + kSpanOfBlocks <= blocks) {
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

// WHOLE: rows are whole spans, and every wave takes them as such: no step, block or value is missing anywhere.
template <int RG, int CG, int X, bool WHOLE>
__global__ __launch_bounds__(64 * kFewWaves) void mx_few_kernel(MxFewArgs a) {
  // Steps whose values of a are asked for together: as many as leave room for b's.
  constexpr u32 AHEAD = X == kHeldRows ? 4 : 64 / (RG * (X == ZC_F32 ? 32 : 16));
  constexpr bool SPANS = WHOLE || X == kHeldRows;       // a wave takes whole spans
  __shared__ f32x4_t parts[kFewWaves * RG * CG * 64];
  const u32 lane = threadIdx.x & 63u, wave = u32(__builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6))), in16 = lane & 15u, part = lane >> 4;
  const u64 col0 = u64(blockIdx.x) * (16 * CG);
  const u8* rows_b[CG];
  const u8* scales_b[CG];
#pragma unroll
  for (int c = 0; c < CG; ++c) {
    const u64 col = min(col0 + 16 * c + in16, a.p.n - 1);                      // (columns behind the last one: any, nobody looks at them)
    rows_b[c] = a.p.b + col * a.p.b_stride;
    scales_b[c] = a.p.b_scales + col * a.p.b_scales_stride;
  }
  __amdgpu_buffer_rsrc_t values;
  u32 row_bytes = 0, last_count = 0;                                            // (values of a row's last block, where it is incomplete)
  if constexpr (X != kHeldRows) {
    constexpr u32 BYTES = sizeof(typename ValueOf<X>::One);
    row_bytes = u32(a.x_stride) * BYTES;
    last_count = u32(a.k) % kBlockValues;
    values = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(a.x), 0, (u32(a.p.m) - 1u) * row_bytes + u32(a.k) * BYTES, 0x00027000);
  }
  f32x4_t sum[RG][CG];
#pragma unroll
  for (int r = 0; r < RG; ++r)
#pragma unroll
    for (int c = 0; c < CG; ++c) sum[r][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  for (u32 turn = wave * (SPANS ? 4u : a.steps); 4 * turn < a.p.blocks; turn += kFewWaves * (SPANS ? 4u : a.steps)) {
    const u32 first = turn / 4 * kSpanOfBlocks, t0 = SPANS ? 0u : turn & 3u, t1 = SPANS ? 4u : t0 + a.steps;             // the span, and the steps of it that are this wave's
    u32x4_t b[CG][4], sb[CG], sa[RG];
    MxRaw<X> x[RG][AHEAD];
    const auto load_x = [&](u32 from) {
#pragma unroll
      for (u32 t = from; t < from + AHEAD; ++t) {
        if (t < t0 || t >= t1) continue;
        const u32 block = first + 4 * t + part;
#pragma unroll
        for (int r = 0; r < RG; ++r) {
          const u32 row = 16 * r + in16;
          if constexpr (X == kHeldRows) {               // (rows and blocks that there are none of: any, with scale bytes of zero)
            x[r][t - from].codes = *reinterpret_cast<const u32x4_t*>(a.p.a + min(row, u32(a.p.m) - 1u) * a.p.a_stride + kMxBytes * (WHOLE || block < a.p.blocks ? block : 0u));
          } else {
            const u32 at = row < a.p.m && (WHOLE || block < a.p.blocks) ? row * row_bytes + block * u32(kBlockValues * sizeof(typename ValueOf<X>::One)) : ~0u;
            if (!WHOLE && last_count && first + 4 * t + 4 >= a.p.blocks) mx_load_some_values<X>(values, at, block + 1 < a.p.blocks ? kBlockValues : last_count, x[r][t - from]);
            else mx_load_values<X>(values, at, x[r][t - from]);
          }
        }
      }
    };
    load_x(0);
    if constexpr (X == kHeldRows) {
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        sa[r] = mx_span_scales<WHOLE>(a.p.a_scales + min(16u * r + in16, u32(a.p.m) - 1u) * a.p.a_scales_stride, first, a.p.blocks);
      }
    }
#pragma unroll
    for (int c = 0; c < CG; ++c) sb[c] = mx_span_scales<WHOLE>(scales_b[c], first, a.p.blocks);
#pragma unroll
    for (u32 t = 0; t < 4; ++t) {
      const u32 block = first + 4 * t + part;
      if (t < t0 || t >= t1) continue;
#pragma unroll
      for (int c = 0; c < CG; ++c) b[c][t] = *reinterpret_cast<const u32x4_t*>(rows_b[c] + kMxBytes * (WHOLE || block < a.p.blocks ? block : 0u));
    }
#pragma unroll
    for (u32 from = 0; from < 4; from += AHEAD) {
      u32x4_t codes[RG][AHEAD];
      u32 scale_a[RG][AHEAD];
#pragma unroll
      for (u32 t = from; t < from + AHEAD; ++t)
#pragma unroll
        for (int r = 0; r < RG; ++r) {
          if (t < t0 || t >= t1) continue;
          if constexpr (X == kHeldRows) codes[r][t - from] = x[r][t - from].codes, scale_a[r][t - from] = sa[r][t] >> (8 * part);
          else codes[r][t - from] = mx_block_of_values<X>(x[r][t - from], scale_a[r][t - from]);
        }
      if (from + AHEAD < 4) load_x(from + AHEAD);
#pragma unroll
      for (u32 t = from; t < from + AHEAD; ++t) {
        if (t < t0 || t >= t1) continue;
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
          for (int c = 0; c < CG; ++c)
            sum[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(b[c][t]), mx_operand(codes[r][t - from]), sum[r][c], kMxFp4, kMxFp4, 0,
                                                                         int(sb[c][t] >> (8 * part)), 0, int(scale_a[r][t - from]));
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RG; ++r)
#pragma unroll
    for (int c = 0; c < CG; ++c) parts[(wave * RG * CG + r * CG + c) * 64 + lane] = sum[r][c];
  __syncthreads();
  for (u32 i = threadIdx.x; i < RG * CG * 64; i += 64 * kFewWaves) {
    const u32 group = i >> 6, r = group / CG, c = group % CG;
    f32x4_t s = parts[i];
#pragma unroll
    for (u32 w = 1; w < kFewWaves; ++w) s += parts[w * RG * CG * 64 + i];
    float v[4] = {s[0], s[1], s[2], s[3]};
    const u64 row = 16 * r + in16, col = col0 + 16 * c + 4 * part;
    if (row < a.p.m && col < a.p.n) mx_finish(a.p, row, col, v);
  }
}

}  // namespace zc
