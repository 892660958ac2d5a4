// Products of matrices held in 4 bits, both along their rows: out[i][j] (+)= sum over k of a[i][k] b[j][k], + bias[j].
//
// The matrix instructions take a block as it lies in memory: a lane's operand is the 16 bytes of one block with its scale byte, and they
// scale, multiply and add in binary32.  Sums are rounded once, to the output's type.
#pragma once

#include "zc_mx.h"

namespace zc {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct MxProductArgs {
  const u8 *a, *a_scales, *b, *b_scales;
  u64 a_stride, a_scales_stride, b_stride, b_scales_stride;
  u64 m, n;
  u32 blocks;                    // of a row
  const float* bias;
  void* out;
  u64 out_stride;
  int out_type;
  u32 add;
};

constexpr int kMxFp4 = 4;        // the instructions' number for e2m1

__device__ inline i32x8_t mx_operand(u32x4_t w) { return i32x8_t{int(w[0]), int(w[1]), int(w[2]), int(w[3]), 0, 0, 0, 0}; }

// One result, or four neighbouring ones of a row.
__device__ inline void mx_finish(const MxProductArgs& a, u64 row, u64 col, const f32x4_t& sum) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (col + j >= a.n) break;
    const u64 at = row * a.out_stride + col + j;
    float v = sum[j];
    if (a.bias) v += a.bias[col + j];
    if (a.add) v += load_value(a.out, a.out_type, at);
    store_value(a.out, a.out_type, at, v);
  }
}

// A wave makes 16 x 16 results.  The rows of b go in as the instruction's first operand, so that a lane ends with four neighbouring results of one row.
__global__ __launch_bounds__(64) void mx_product_kernel(MxProductArgs a) {
  const u32 lane = threadIdx.x, part = lane >> 4;
  const u64 col0 = u64(blockIdx.x) * 16, row0 = u64(blockIdx.y) * 16;
  const u64 row = row0 + (lane & 15u), col = col0 + (lane & 15u);
  f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (u32 k = 0; k < a.blocks; k += 4) {
    const u32 block = k + part;
    u32x4_t wa = {0, 0, 0, 0}, wb = {0, 0, 0, 0};
    u32 sa = 0, sb = 0;
    if (row < a.m && block < a.blocks) {
      wa = *reinterpret_cast<const u32x4_t*>(a.a + row * a.a_stride + kMxBytes * block);
      sa = a.a_scales[row * a.a_scales_stride + block];
    }
    if (col < a.n && block < a.blocks) {
      wb = *reinterpret_cast<const u32x4_t*>(a.b + col * a.b_stride + kMxBytes * block);
      sb = a.b_scales[col * a.b_scales_stride + block];
    }
    sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(wb), mx_operand(wa), sum, kMxFp4, kMxFp4, 0, int(sb), 0, int(sa));
  }
  if (row < a.m) mx_finish(a, row, col0 + 4 * part, sum);
}

}  // namespace zc
