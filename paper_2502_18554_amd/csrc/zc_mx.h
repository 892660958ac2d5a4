// 4-bit blocks: 32 values as e2m1 codes with a power of two for a scale (one byte, e8m0), and back.
//
// The scale puts the largest magnitude of a block into [4, 8) of the codes' 0 .. 6: exponent field minus 2; a block with a value
// that is not finite has scale byte 255 and stands for 32 NaNs.  Codes are rounded half to even; what lies above 6 becomes 6.
#pragma once

#include "zc_values.h"

namespace zc {

constexpr u32 kMxBytes = kBlockValues / 2;          // of a block's codes: one lane's share of a matrix instruction

__device__ inline u32 mx_scale(u32 top) {
  const u32 e = top >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// Eight values (scaled by the block's power of two in the conversion) as eight codes, the first one lowest.
__device__ inline u32 mx_codes(const float (&v)[8], float scale) {
  u32 w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

__device__ inline void mx_values(u32 codes, float scale, float (&v)[8]) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

struct MxHeld {                 // a matrix held in 4 bits
  u8* codes;
  u8* scales;
  u64 codes_stride, scales_stride;
};

struct MxQuantizeArgs {
  const void* in;
  u64 rows, cols, stride;
  int type;
  MxHeld held, held_t;          // null codes: not wanted
};

// One thread a block: along a row, or down a column for the transposed matrix.
__device__ inline void mx_quantize_block(const MxQuantizeArgs& a, u64 row, u64 col, u64 row_step, u64 col_step, u64 count, u8* codes, u8* scale) {
  float v[32];
  u32 top = 0;
#pragma unroll
  for (u32 j = 0; j < 32; ++j) {
    v[j] = j < count ? load_value(a.in, a.type, (row + j * row_step) * a.stride + col + j * col_step) : 0.0f;
    top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  }
  const u32 s = mx_scale(top);
  *scale = u8(s);
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float part[8] = {v[8 * i], v[8 * i + 1], v[8 * i + 2], v[8 * i + 3], v[8 * i + 4], v[8 * i + 5], v[8 * i + 6], v[8 * i + 7]};
    w[i] = s == 255u ? 0u : mx_codes(part, scale_value(s));
  }
  *reinterpret_cast<u32x4_t*>(codes) = w;
}

__global__ __launch_bounds__(256) void mx_quantize_kernel(MxQuantizeArgs a) {
  const u64 i = u64(blockIdx.x) * 256 + threadIdx.x;
  const u64 across = num_blocks(a.cols), down = num_blocks(a.rows);
  if (a.held.codes && i < a.rows * across) {
    const u64 r = i / across, b = i % across;
    mx_quantize_block(a, r, 32 * b, 0, 1, a.cols - 32 * b, a.held.codes + r * a.held.codes_stride + kMxBytes * b, a.held.scales + r * a.held.scales_stride + b);
  }
  if (a.held_t.codes && i < a.cols * down) {
    const u64 b = i / a.cols, col = i % a.cols;
    mx_quantize_block(a, 32 * b, col, 1, 0, a.rows - 32 * b, a.held_t.codes + col * a.held_t.codes_stride + kMxBytes * b,
                      a.held_t.scales + col * a.held_t.scales_stride + b);
  }
}

struct MxDequantizeArgs {
  MxHeld held;
  u64 rows, cols, stride;
  void* out;
  int type;
};

__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxDequantizeArgs a) {
  const u64 i = u64(blockIdx.x) * 256 + threadIdx.x;
  const u64 across = num_blocks(a.cols);
  if (i >= a.rows * across) return;
  const u64 r = i / across, b = i % across;
  const u32x4_t w = *reinterpret_cast<const u32x4_t*>(a.held.codes + r * a.held.codes_stride + kMxBytes * b);
  const float scale = scale_value(a.held.scales[r * a.held.scales_stride + b]);
  const u64 count = a.cols - 32 * b;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float v[8];
    mx_values(w[q], scale, v);
#pragma unroll
    for (u32 j = 0; j < 8; ++j)
      if (8 * q + j < count) store_value(a.out, a.type, r * a.stride + 32 * b + 8 * q + j, v[j]);
  }
}

}  // namespace zc
