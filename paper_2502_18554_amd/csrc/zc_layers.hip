// C ABI of the calls around the collective: the optimiser's step over many tensors, and layers held in 4-bit blocks.
// Argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "zc_adamw.h"
#include "zc_mx.h"
#include "zc_mx_few.h"
#include "zc_mx_product.h"

using namespace zc;

namespace {

bool aligned(const void* p, u64 to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool type_valid(int type) { return type == ZC_F32 || type == ZC_BF16 || type == ZC_F16; }
int launched() { return hipGetLastError() == hipSuccess ? ZC_OK : ZC_ERR_HIP; }
constexpr u64 kMostGroups = 0xffffffu;             // of 256 threads: a grid has less than 2^32 threads
constexpr u64 kMostTiles = 0x7fffffffu;            // that a persistent grid counts
constexpr u64 kMostCols = u64(1) << 28;            // of a product's one launch, with the same limit

template <int P, int G>
void launch_adamw(const AdamwArgs& a, u32 tiles, int bits, hipStream_t stream) {
  if (bits == 32) hipLaunchKernelGGL((adamw_kernel<P, G, 32>), dim3(tiles), dim3(kAdamwThreads), 0, stream, a);
  else hipLaunchKernelGGL((adamw_kernel<P, G, 8>), dim3(tiles), dim3(kAdamwThreads), 0, stream, a);
}
template <int P>
void launch_adamw(const AdamwArgs& a, u32 tiles, int bits, int grad_type, hipStream_t stream) {
  if (grad_type == ZC_F32) launch_adamw<P, ZC_F32>(a, tiles, bits, stream);
  else if (grad_type == ZC_BF16) launch_adamw<P, ZC_BF16>(a, tiles, bits, stream);
  else launch_adamw<P, ZC_F16>(a, tiles, bits, stream);
}
void launch_adamw(const AdamwArgs& a, u32 tiles, int bits, int param_type, int grad_type, hipStream_t stream) {
  if (param_type == ZC_F32) launch_adamw<ZC_F32>(a, tiles, bits, grad_type, stream);
  else if (param_type == ZC_BF16) launch_adamw<ZC_BF16>(a, tiles, bits, grad_type, stream);
  else launch_adamw<ZC_F16>(a, tiles, bits, grad_type, stream);
}

// Blocks of the tensors' state, or ~0 where sizes are out of range.
u64 state_blocks(const size_t* n, int k) {
  u64 blocks = 0;
  for (int i = 0; i < k; ++i) {
    if (n[i] > (u64(1) << 36)) return ~u64(0);
    blocks += num_blocks(n[i]);
  }
  return blocks <= 0xffffffffu ? blocks : ~u64(0);
}

bool held_valid(const void* codes, const void* scales, u64 rows, u64 cols, u64 codes_stride, u64 scales_stride) {
  const u64 blocks = num_blocks(cols);
  if (codes_stride % 16 || scales_stride % 4 || codes_stride > (u64(1) << 32) || scales_stride > (u64(1) << 32)) return false;
  if (codes_stride < kMxBytes * blocks || scales_stride < blocks) return false;
  return rows == 0 || cols == 0 || (codes && scales && aligned(codes, 16) && aligned(scales, 4));
}
bool matrix_valid(const void* p, int type, u64 rows, u64 cols, u64 stride) {
  return type_valid(type) && stride >= cols && stride <= (u64(1) << 32) && (rows == 0 || cols == 0 || (p && aligned(p, value_bytes(type))));
}
bool sizes_valid(u64 rows, u64 cols) { return rows <= 0x7fffffffu && cols <= 0x7fffffffu; }
bool product_valid(u64 m, u64 n, u64 k) { return sizes_valid(m, k) && sizes_valid(n, k) && ((m + 63) / 64) * ((n + 63) / 64) <= kMostTiles; }

template <int T, int TYPE>
void launch_tiles(const MxProductArgs& a, hipStream_t stream) {
  const u64 down = (a.m + mx_tile_rows(T) - 1) / mx_tile_rows(T), across = (a.n + mx_tile_rows(T) - 1) / mx_tile_rows(T);
  const u64 at_once = 256 * (T == 4 ? 1 : T == 2 ? 2 : 4);            // workgroups that the GPU holds
  hipLaunchKernelGGL((mx_tile_kernel<T, T, TYPE>), dim3(u32(down * across < at_once ? down * across : at_once)), dim3(256), 0, stream, a, u32(down), u32(across));
}

// Few rows: as many columns a workgroup as leave a workgroup for every CU (24 rows x 16384 x 4096 11.0 us by 64 columns, 14.3 by 16; x 8192 x 4096 7.1 by 32, 8.5 by 16; a
// row x 8192 x 4096 5.7 and 5.3).  Where rows of values are short, every wave takes a part of a span, so that all of them share the quantising (1 x 4096 x 1000 4.1 us, 4.8
// by spans); of held rows a wave takes whole spans (1 x 4096 x 1024 2.4 us, 2.9 by parts).
template <int RG, int CG, int X>
int launch_few(MxFewArgs a, hipStream_t stream) {
  const u64 groups = (a.p.n + 16 * CG - 1) / (16 * CG), steps = (a.p.blocks + 3) / 4;
  a.steps = X == kHeldRows || steps >= 4 * kFewWaves ? 4 : steps >= 2 * kFewWaves ? 2 : 1;
  const bool whole = a.steps == 4 && a.p.blocks % kSpanOfBlocks == 0 && (X == kHeldRows || a.k % kBlockValues == 0);
  if (whole) hipLaunchKernelGGL((mx_few_kernel<RG, CG, X, true>), dim3(u32(groups)), dim3(64 * kFewWaves), 0, stream, a);
  else hipLaunchKernelGGL((mx_few_kernel<RG, CG, X, false>), dim3(u32(groups)), dim3(64 * kFewWaves), 0, stream, a);
  return launched();
}
template <int RG, int X>
int launch_few(const MxFewArgs& a, hipStream_t stream) {
  if (a.p.n >= 4 * 16 * 256) return launch_few<RG, 4, X>(a, stream);
  if (a.p.n >= 2 * 16 * 256) return launch_few<RG, 2, X>(a, stream);
  return launch_few<RG, 1, X>(a, stream);
}
template <int T>
void launch_tiles(const MxProductArgs& a, hipStream_t stream) {
  if (a.out_type == ZC_F32) launch_tiles<T, ZC_F32>(a, stream);
  else if (a.out_type == ZC_BF16) launch_tiles<T, ZC_BF16>(a, stream);
  else launch_tiles<T, ZC_F16>(a, stream);
}

// Calls `launch` for the columns of a product, kMostCols at a time.
template <typename F>
int by_columns(const MxProductArgs& a, const F& launch) {
  for (u64 at = 0; at < a.n; at += kMostCols) {
    MxProductArgs part = a;
    part.n = a.n - at < kMostCols ? a.n - at : kMostCols;
    part.b += at * a.b_stride;
    part.b_scales += at * a.b_scales_stride;
    if (a.bias) part.bias += at;
    part.out = static_cast<u8*>(a.out) + at * value_bytes(a.out_type);
    const int st = launch(part);
    if (st != ZC_OK) return st;
  }
  return ZC_OK;
}

int product_launch(const MxProductArgs& a, hipStream_t stream) {
  if (a.m <= kFewRows) {
    const MxFewArgs few{a, nullptr, 0, 0, 0};
    return a.m <= 16 ? launch_few<1, kHeldRows>(few, stream) : launch_few<2, kHeldRows>(few, stream);
  }
  if (a.blocks > 0 && a.a_stride <= kMostTileStride && a.b_stride <= kMostTileStride && a.a_scales_stride <= kMostTileStride && a.b_scales_stride <= kMostTileStride) {
    // The size of tile that takes the least time, in us, by what a turn of all CUs has been measured to take: a tile's begin and end, and 4096 values along k.
    // (4096 x 4096 x 4096 by tiles of 256, 128 and 64: 39, 43 and 63 us; 1024 x 4096 x 4096: 26, 14 and 19; 333 x 1531 x 1000: 18, 7.4 and 4.6.)
    const double along = double(a.blocks) / 128;
    const auto turns = [&](u64 rows) { return double(((a.m + rows - 1) / rows * ((a.n + rows - 1) / rows) + 255) / 256); };
    const double large = turns(256) * (14.8 + 25.0 * along), middle = 3.0 + turns(128) * (2.6 + 8.9 * along), small = 3.0 + turns(64) * (0.6 + 3.4 * along);
    if (large <= middle && large <= small) launch_tiles<4>(a, stream);
    else if (middle <= small) launch_tiles<2>(a, stream);
    else launch_tiles<1>(a, stream);
    return launched();
  }
  const u64 down = (a.m + 15) / 16, across = (a.n + 15) / 16;
  for (u64 at = 0; at < down; at += 65535) {                        // (a grid's second extent)
    MxProductArgs part = a;
    part.m = a.m - 16 * at;
    part.a += 16 * at * a.a_stride;
    part.a_scales += 16 * at * a.a_scales_stride;
    part.out = static_cast<u8*>(a.out) + 16 * at * a.out_stride * value_bytes(a.out_type);
    const u64 left = down - at;
    hipLaunchKernelGGL(mx_product_kernel, dim3(u32(across), u32(left < 65535 ? left : 65535)), dim3(64), 0, stream, part);
  }
  return launched();
}
int product(const MxProductArgs& a, hipStream_t stream) {
  if (a.m == 0 || a.n == 0) return ZC_OK;
  return by_columns(a, [&](const MxProductArgs& part) { return product_launch(part, stream); });
}

MxHeld from_block(MxHeld h, u64 row, u64 block) {
  if (!h.codes) return h;
  h.codes += row * h.codes_stride + kMxBytes * block;
  h.scales += row * h.scales_stride + block;
  return h;
}

template <int TYPE>
int launch_quantize(const MxQuantizeArgs& a, hipStream_t stream) {
  const bool by_columns = a.held_t.codes;
  const u64 rows = mx_quantize_rows(by_columns), cols = mx_quantize_cols(TYPE, by_columns);
  // Pieces of whole tiles, as many as a grid counts (long thin matrices have more: 2^30 values of 32 bits down the columns of one row are 2^24 tiles).
  const u64 most_cols = kMostGroups * cols;
  for (u64 col = 0; col < a.cols; col += most_cols) {
    const u64 now = a.cols - col < most_cols ? a.cols - col : most_cols, across = (now + cols - 1) / cols, most_rows = kMostGroups / across * rows;
    for (u64 row = 0; row < a.rows; row += most_rows) {
      MxQuantizeArgs part = a;
      part.rows = a.rows - row < most_rows ? a.rows - row : most_rows;
      part.cols = now;
      part.in = static_cast<const u8*>(a.in) + (row * a.stride + col) * value_bytes(TYPE);
      part.held = from_block(a.held, row, col / kBlockValues);
      part.held_t = from_block(a.held_t, col, row / kBlockValues);
      const u32 tiles = u32((part.rows + rows - 1) / rows * across);
      if (a.held.codes && a.held_t.codes) hipLaunchKernelGGL((mx_quantize_kernel<TYPE, true, true>), dim3(tiles), dim3(256), 0, stream, part, u32(across));
      else if (a.held.codes) hipLaunchKernelGGL((mx_quantize_kernel<TYPE, true, false>), dim3(tiles), dim3(256), 0, stream, part, u32(across));
      else hipLaunchKernelGGL((mx_quantize_kernel<TYPE, false, true>), dim3(tiles), dim3(256), 0, stream, part, u32(across));
    }
  }
  return launched();
}
int quantize(const MxQuantizeArgs& a, hipStream_t stream) {
  if (a.rows == 0 || a.cols == 0) return ZC_OK;
  return a.type == ZC_F32 ? launch_quantize<ZC_F32>(a, stream) : a.type == ZC_BF16 ? launch_quantize<ZC_BF16>(a, stream) : launch_quantize<ZC_F16>(a, stream);
}

template <int TYPE>
void launch_dequantize(const MxDequantizeArgs& a, u32 across, u32 pieces, hipStream_t stream) {
  const u32 inverse = u32(((u64(1) << 32) + across - 1) / across);
  // Four pieces a thread where the GPU is full and a piece is a single store (4096 x 4096 in 16 bits 7.8 us, 8.5 by one; 8192 x 8192 in 32 bits 75 us by four, 60 by one;
  // 777 x 2048 in 16 bits 3.3 by four, 2.4 by one).
  if (TYPE == ZC_F32 || pieces <= 8 * 256 * 256) hipLaunchKernelGGL((mx_dequantize_kernel<TYPE, 1>), dim3((pieces + 255) / 256), dim3(256), 0, stream, a, across, inverse, pieces);
  else if constexpr (TYPE != ZC_F32) hipLaunchKernelGGL((mx_dequantize_kernel<TYPE, 4>), dim3((pieces + 1023) / 1024), dim3(256), 0, stream, a, across, inverse, pieces);
}
void dequantize(const MxDequantizeArgs& a, u32 across, u32 pieces, hipStream_t stream) {
  if (a.type == ZC_F32) launch_dequantize<ZC_F32>(a, across, pieces, stream);
  else if (a.type == ZC_BF16) launch_dequantize<ZC_BF16>(a, across, pieces, stream);
  else launch_dequantize<ZC_F16>(a, across, pieces, stream);
}

}  // namespace

extern "C" {

size_t zc_adamw_state_bytes(const size_t* n, int k, int state_bits) {
  if (k < 0 || (k > 0 && !n) || (state_bits != 8 && state_bits != 32)) return 0;
  const u64 blocks = state_blocks(n, k);
  return blocks == ~u64(0) ? 0 : size_t(adamw_bytes(blocks, state_bits));
}

int zc_adamw(int k, const size_t* n, void* const* d_params, int param_type, const void* const* d_grads, int grad_type,
             void* const* d_copies, int copy_type, void* d_state, size_t state_bytes, int state_bits, uint64_t step, double lr, double beta1,
             double beta2, double eps, double weight_decay, const float* d_grad_scale, uint64_t seed, void* hip_stream) {
  if (k < 0 || (k > 0 && (!n || !d_params || !d_grads)) || !type_valid(param_type) || !type_valid(grad_type)) return ZC_ERR_ARG;
  if ((d_copies && !type_valid(copy_type)) || (state_bits != 8 && state_bits != 32) || step == 0) return ZC_ERR_ARG;
  if (!(std::isfinite(lr) && lr >= 0 && beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && std::isfinite(eps) && eps >= 0 &&
        std::isfinite(weight_decay) && weight_decay >= 0))
    return ZC_ERR_ARG;
  const u64 blocks = state_blocks(n, k);
  if (blocks == ~u64(0) || state_bytes < adamw_bytes(blocks, state_bits) || (blocks && !d_state) || !aligned(d_state, 16)) return ZC_ERR_ARG;
  if (!aligned(d_grad_scale, 4)) return ZC_ERR_ARG;
  for (int i = 0; i < k; ++i) {
    if (n[i] == 0) continue;
    if (!d_params[i] || !d_grads[i] || !aligned(d_params[i], value_bytes(param_type)) || !aligned(d_grads[i], value_bytes(grad_type))) return ZC_ERR_ARG;
    if (d_copies && !aligned(d_copies[i], value_bytes(copy_type))) return ZC_ERR_ARG;
  }
  AdamwArgs a = {};
  a.c.b1 = float(beta1);
  a.c.c1 = float(1 - beta1);
  a.c.b2 = float(beta2);
  a.c.c2 = float(1 - beta2);
  a.c.keep = float(1 - lr * weight_decay);
  // The reciprocal instruction takes subnormal numbers for zeros and makes none.  A denominator is eps, or at least a root, 2^-75, and at most 2^91 and eps: where eps lets it
  // be subnormal, or so large that its reciprocal is, it is scaled by a power of two (exactly), which the last factor takes out again.
  const float eps32 = float(eps);
  const double scaled = eps32 > 0 && eps32 < 0x1p-126f ? 0x1p24 : eps32 >= 0x1p96f ? 0x1p-32 : 1;
  a.c.rate = float(lr / (1 - std::pow(beta1, double(step))) * scaled);
  a.c.root = float(1 / std::sqrt(1 - std::pow(beta2, double(step))) * scaled);
  a.c.eps = float(double(eps32) * scaled);
  a.copy_type = copy_type;
  a.state = static_cast<u8*>(d_state);
  a.blocks = blocks;
  a.grad_scale = d_grad_scale;
  a.key = adamw_key(seed, step);
  a.stochastic = seed != 0;
  u32 tiles = 0;
  u64 block = 0;
  const auto go = [&] {
    launch_adamw(a, tiles, state_bits, param_type, grad_type, static_cast<hipStream_t>(hip_stream));
    a.tensors = tiles = 0;
  };
  for (int i = 0; i < k; ++i) {
    for (u64 at = 0; at < n[i]; at += kAdamwMost) {
      const u64 now = n[i] - at < kAdamwMost ? n[i] - at : kAdamwMost;
      const u32 own = u32((now + kAdamwTile - 1) / kAdamwTile);
      if (a.tensors == kAdamwTensors || u64(tiles) + own > kMostGroups) go();
      a.first_tile[a.tensors] = tiles;
      a.first_block[a.tensors] = u32(block);
      a.n[a.tensors] = u32(now);
      a.param[a.tensors] = static_cast<u8*>(d_params[i]) + at * value_bytes(param_type);
      a.grad[a.tensors] = static_cast<const u8*>(d_grads[i]) + at * value_bytes(grad_type);
      a.copy[a.tensors] = d_copies && d_copies[i] ? static_cast<u8*>(d_copies[i]) + at * value_bytes(copy_type) : nullptr;
      ++a.tensors;
      tiles += own;
      block += num_blocks(now);
    }
  }
  if (!a.tensors) return ZC_OK;                                      // (no values at all)
  go();
  return launched();
}

size_t zc_mx_codes_stride(size_t cols) { return kMxBytes * num_blocks(cols); }
size_t zc_mx_scales_stride(size_t cols) { return 4 * ((num_blocks(cols) + 3) / 4); }

size_t zc_mx_workspace_bytes(size_t m, size_t n, size_t k) {
  (void)n;
  return pad16(m * zc_mx_codes_stride(k)) + pad16(m * zc_mx_scales_stride(k));
}

int zc_mx_quantize(const void* d_in, int type, size_t rows, size_t cols, size_t stride, void* d_codes, size_t codes_stride, void* d_scales,
                   size_t scales_stride, void* d_codes_t, size_t codes_t_stride, void* d_scales_t, size_t scales_t_stride, void* hip_stream) {
  if (!sizes_valid(rows, cols) || !matrix_valid(d_in, type, rows, cols, stride)) return ZC_ERR_ARG;
  if ((!d_codes) != (!d_scales) || (!d_codes_t) != (!d_scales_t) || (!d_codes && !d_codes_t && rows && cols)) return ZC_ERR_ARG;
  if (d_codes && !held_valid(d_codes, d_scales, rows, cols, codes_stride, scales_stride)) return ZC_ERR_ARG;
  if (d_codes_t && !held_valid(d_codes_t, d_scales_t, cols, rows, codes_t_stride, scales_t_stride)) return ZC_ERR_ARG;
  MxQuantizeArgs a;
  a.in = d_in;
  a.rows = rows, a.cols = cols, a.stride = stride;
  a.type = type;
  a.held = {static_cast<u8*>(d_codes), static_cast<u8*>(d_scales), codes_stride, scales_stride};
  a.held_t = {static_cast<u8*>(d_codes_t), static_cast<u8*>(d_scales_t), codes_t_stride, scales_t_stride};
  return quantize(a, static_cast<hipStream_t>(hip_stream));
}

int zc_mx_dequantize(const void* d_codes, size_t codes_stride, const void* d_scales, size_t scales_stride, size_t rows, size_t cols, void* d_out,
                     int type, size_t stride, void* hip_stream) {
  if (!sizes_valid(rows, cols) || !matrix_valid(d_out, type, rows, cols, stride)) return ZC_ERR_ARG;
  if (!held_valid(d_codes, d_scales, rows, cols, codes_stride, scales_stride)) return ZC_ERR_ARG;
  if (rows == 0 || cols == 0) return ZC_OK;
  const u32 across = u32((cols + 7) / 8);
  const u64 most = 0xf0000000u / across;                            // rows whose pieces, and those of the last workgroup and row behind them, are counted in 32 bits
  for (u64 at = 0; at < rows; at += most) {
    const u64 now = rows - at < most ? rows - at : most;
    MxDequantizeArgs a;
    a.held = {static_cast<u8*>(const_cast<void*>(d_codes)) + at * codes_stride, static_cast<u8*>(const_cast<void*>(d_scales)) + at * scales_stride, codes_stride, scales_stride};
    a.rows = now, a.cols = cols, a.stride = stride;
    a.out = static_cast<u8*>(d_out) + at * stride * value_bytes(type);
    a.type = type;
    const u32 pieces = u32(now * across);
    dequantize(a, across, pieces, static_cast<hipStream_t>(hip_stream));
  }
  return launched();
}

int zc_mx_product(const void* d_a, size_t a_stride, const void* d_a_scales, size_t a_scales_stride, const void* d_b, size_t b_stride,
                  const void* d_b_scales, size_t b_scales_stride, size_t m, size_t n, size_t k, const float* d_bias, void* d_out, int out_type,
                  size_t out_stride, unsigned flags, void* d_ws, size_t ws_bytes, void* hip_stream) {
  if (!product_valid(m, n, k) || (flags & ~ZC_MX_ADD) || !matrix_valid(d_out, out_type, m, n, out_stride)) return ZC_ERR_ARG;
  if (!held_valid(d_a, d_a_scales, m, k, a_stride, a_scales_stride) || !held_valid(d_b, d_b_scales, n, k, b_stride, b_scales_stride)) return ZC_ERR_ARG;
  if (!aligned(d_bias, 4) || !aligned(d_ws, 16)) return ZC_ERR_ARG;
  (void)ws_bytes;
  MxProductArgs a;
  a.a = static_cast<const u8*>(d_a), a.a_scales = static_cast<const u8*>(d_a_scales);
  a.b = static_cast<const u8*>(d_b), a.b_scales = static_cast<const u8*>(d_b_scales);
  a.a_stride = a_stride, a.a_scales_stride = a_scales_stride, a.b_stride = b_stride, a.b_scales_stride = b_scales_stride;
  a.m = m, a.n = n;
  a.blocks = u32(num_blocks(k));
  a.bias = d_bias;
  a.out = d_out;
  a.out_stride = out_stride;
  a.out_type = out_type;
  a.add = flags & ZC_MX_ADD;
  return product(a, static_cast<hipStream_t>(hip_stream));
}

int zc_mx_linear(const void* d_x, int x_type, size_t x_stride, const void* d_w, size_t w_stride, const void* d_w_scales, size_t w_scales_stride,
                 size_t m, size_t n, size_t k, const float* d_bias, void* d_out, int out_type, size_t out_stride, unsigned flags, void* d_ws,
                 size_t ws_bytes, void* hip_stream) {
  if (!sizes_valid(m, k) || !matrix_valid(d_x, x_type, m, k, x_stride)) return ZC_ERR_ARG;
  if (ws_bytes < zc_mx_workspace_bytes(m, n, k) || !aligned(d_ws, 16) || (!d_ws && m && k)) return ZC_ERR_ARG;
  const u64 codes_stride = zc_mx_codes_stride(k), scales_stride = zc_mx_scales_stride(k), codes_bytes = pad16(m * codes_stride);
  u8* const codes = static_cast<u8*>(d_ws);
  u8* const scales = codes + codes_bytes;
  // (the product's own checks come first: nothing is launched by a call that is refused)
  if (!product_valid(m, n, k) || (flags & ~ZC_MX_ADD) || !matrix_valid(d_out, out_type, m, n, out_stride) || !aligned(d_bias, 4) ||
      !held_valid(d_w, d_w_scales, n, k, w_stride, w_scales_stride))
    return ZC_ERR_ARG;
  if (m == 0 || n == 0) return ZC_OK;
  MxProductArgs a;
  a.a = codes, a.a_scales = scales;
  a.b = static_cast<const u8*>(d_w), a.b_scales = static_cast<const u8*>(d_w_scales);
  a.a_stride = codes_stride, a.a_scales_stride = scales_stride, a.b_stride = w_stride, a.b_scales_stride = w_scales_stride;
  a.m = m, a.n = n;
  a.blocks = u32(num_blocks(k));
  a.bias = d_bias;
  a.out = d_out;
  a.out_stride = out_stride;
  a.out_type = out_type;
  a.add = flags & ZC_MX_ADD;
  hipStream_t const stream = static_cast<hipStream_t>(hip_stream);
  // Up to 8 rows are quantised by the product's own waves, each of which does so again for its 16 CG columns; more rows take longer so than a launch of their own.
  // (In this kernel against both, GPU time: 4096 x 4096 by 1, 8 and 16 rows 4.3, 5.6 and 6.8 us against 5.4, 5.9 and 6.3; 16384 x 4096 by 1, 8, 16 and 32 rows
  // 9.9, 10.5, 11.6 and 16.8 against 10.3, 10.5, 10.9 and 13.1.  8 rows by two launches cost the caller's thread another 2.5 us besides.)
  if (m <= kFewValueRows && x_stride <= kMostFewStride) {
    return by_columns(a, [&](const MxProductArgs& part) {
      const MxFewArgs few{part, d_x, x_stride, k, 0};
      return x_type == ZC_F32 ? launch_few<1, ZC_F32>(few, stream) : x_type == ZC_BF16 ? launch_few<1, ZC_BF16>(few, stream) : launch_few<1, ZC_F16>(few, stream);
    });
  }
  const int st = zc_mx_quantize(d_x, x_type, m, k, x_stride, codes, codes_stride, scales, scales_stride, nullptr, 0, nullptr, 0, hip_stream);
  return st != ZC_OK ? st : product(a, stream);
}

}  // extern "C"
