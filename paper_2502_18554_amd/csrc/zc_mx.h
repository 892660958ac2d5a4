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

// Values of a type by the 16 bytes, as they lie in memory.
template <int TYPE> struct MxPack;
template <> struct MxPack<ZC_F32> {
  static constexpr u32 kValues = 4;
  static __device__ u32 top(u32x4_t w) {
    const u32x4_t m = w & 0x7fffffffu;
    return max(max(m[0], m[1]), max(m[2], m[3]));
  }
  static __device__ u32 top_value(u32 top) { return top; }                  // the largest magnitude in binary32, from what top() gave
};
// Magnitudes of two 16-bit values compared side by side.
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
__device__ inline u32 max_pairs(u32 a, u32 b) {
  return __builtin_bit_cast(u32, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}
template <> struct MxPack<ZC_BF16> {
  static constexpr u32 kValues = 8;
  static __device__ u32 top(u32x4_t w) {
    const u32x4_t m = w & 0x7fff7fffu;
    return max_pairs(max_pairs(m[0], m[1]), max_pairs(m[2], m[3]));
  }
  static __device__ u32 top_value(u32 top) { return max(top << 16, top & 0xffff0000u); }
};
template <> struct MxPack<ZC_F16> {
  static constexpr u32 kValues = 8;
  static __device__ u32 top(u32x4_t w) { return MxPack<ZC_BF16>::top(w); }
  static __device__ u32 top_value(u32 top) {
    const u16 high = u16(max(top & 0xffffu, top >> 16));
    return __float_as_uint(float(__builtin_bit_cast(_Float16, high)));
  }
};

// Eight values, in the order of their words, as eight codes, the first one lowest; the conversion divides by the block's power of two.
template <int TYPE>
__device__ inline u32 mx_codes(const u32 (&w)[TYPE == ZC_F32 ? 8 : 4], float scale) {
  u32 c = 0;
  if constexpr (TYPE == ZC_F32) {
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[4]), __uint_as_float(w[5]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[6]), __uint_as_float(w[7]), scale, 3);
  } else if constexpr (TYPE == ZC_BF16) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(pair, w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(pair, w[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(pair, w[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(pair, w[3]), scale, 3);
  } else {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(pair, w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(pair, w[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(pair, w[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(pair, w[3]), scale, 3);
  }
  return c;
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

// A workgroup takes 32 KiB.  A thread holds 32 bytes of each of four rows and makes the blocks along them with its neighbours, two or four threads a block.  For the
// blocks down the columns the tile (128 rows of 256 bytes) goes through LDS: wave w takes rows 32 w .. 32 w + 31, a lane one column (of 32 bits) or two (of 16).  Memory
// sees every value once, whichever of the two are wanted.  Along the rows alone a tile is 32 rows of 1024 bytes, so that it writes whole lines of codes: of lines
// that two workgroups share, each half goes to memory by itself (8192 x 8192 in 16 bits 30 us, by 256 bytes 34; 8000 x 8001 31 and 42; of 2048 bytes 30 and 29, and
// 16384 x 16384 123 for 119).
// Tiles follow each other along the rows in the order of the workgroups: neighbours are read at the same time.  (Runs of tiles for each XCD, along the rows or down the
// columns, were slower by 5 to 20 %.)
// Bound by memory: 8192 x 8192 in 16 bits, again and again on inputs that no cache holds, along the rows 30 us (170 MB, 5.6 TB/s), along both axes 50 us (205 MB, 4.1 TB/s), on an
// input in the last cache 26 and 39; right behind kernels that wrote as much or more, 38 to 45 and 68.  Down the columns a lane writes 16 bytes and a byte of lines of its own: of both axes
// 100 MB are written for 71 (tiles of 256 rows, which write whole lines of codes there too, took as long, and small matrices 20 % longer); 24 x 4096 2.3 us, a launch.
__host__ __device__ constexpr u32 mx_tile_bytes(bool down) { return down ? 256 : 1024; }
__host__ __device__ constexpr u32 mx_quantize_rows(bool down) { return 32768 / mx_tile_bytes(down); }
__host__ __device__ constexpr u32 mx_quantize_cols(int type, bool down) { return mx_tile_bytes(down) / (type == ZC_F32 ? 4 : 2); }
constexpr u32 kMxTileBytes = mx_tile_bytes(true);

struct __attribute__((packed, aligned(2))) MxSixteen { u32 w[4]; };

// What a tile's loads have to look after: nothing, as the matrix has all of it; the matrix's end; rows of less than 16 bytes.
enum MxEdge { kWholeTile, kEdgeTile, kNarrowTile };

// 16 bytes of a row from a column on.  Those that the row's end cuts off are the row's last 16, which mx_cut then moves down: loads of single values took up to twice as
// long (333 x 1000 in 16 bits along the rows 2.9 us, 6.1 so).
template <int TYPE, MxEdge EDGE>
__device__ __forceinline__ u32x4_t mx_load_sixteen(const typename ValueOf<TYPE>::One* row, u64 col, u64 cols) {
  constexpr u32 K = MxPack<TYPE>::kValues;
  if constexpr (EDGE != kNarrowTile) {
    const MxSixteen s = *reinterpret_cast<const MxSixteen*>(row + (EDGE == kWholeTile ? col : min(col, cols - K)));
    return u32x4_t{s.w[0], s.w[1], s.w[2], s.w[3]};
  } else {
    u32x4_t w = {0, 0, 0, 0};
#pragma unroll
    for (u32 j = 0; j < K; ++j) {
      const auto one = row[min(u64(j), cols - 1)];
      const bool there = col == 0 && j < cols;
      if constexpr (TYPE == ZC_F32) w[j] = there ? __float_as_uint(one) : 0u;
      else w[j / 2] |= (there ? u32(__builtin_bit_cast(u16, one)) : 0u) << (16 * (j & 1u));
    }
    return w;
  }
}
template <int TYPE>
__device__ __forceinline__ u32x4_t mx_cut(u32x4_t w, int left) {                            // (left: the row's values from the column on)
  constexpr int K = MxPack<TYPE>::kValues;
  const u32 by = u32(K - max(min(left, K), 0));          // values to move
  const u32 words = TYPE == ZC_F32 ? by : by / 2;
  if (TYPE != ZC_F32 && by % 2) w = u32x4_t{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
  if (words & 1u) w = u32x4_t{w[1], w[2], w[3], 0};
  if (words & 2u) w = u32x4_t{w[2], w[3], 0, 0};
  if (words & 4u) w = u32x4_t{0, 0, 0, 0};
  return w;
}

// (Nothing is asked about between the loads, so that all of them are on their way together.)
template <int TYPE, bool ALONG, bool DOWN, MxEdge EDGE>
__device__ __forceinline__ void mx_quantize_tile(const MxQuantizeArgs& a, u64 row0, u64 col0, u32x4_t* tile) {
  using One = typename ValueOf<TYPE>::One;
  using Pack = MxPack<TYPE>;
  constexpr bool WHOLE = EDGE == kWholeTile;
  constexpr u32 N = 2 * Pack::kValues, LANES = kBlockValues / N;          // values of a thread, of a row; threads of a block
  constexpr u32 PARTS = mx_tile_bytes(DOWN) / 32, ROWS = 256 / PARTS;     // threads of a row; rows at a time
  const u32 tid = threadIdx.x, part = tid % PARTS, own_row = tid / PARTS;
  const u64 col = col0 + part * N;
  u32x4_t w[4][2];
#pragma unroll
  for (u32 i = 0; i < 4; ++i) {
    const u64 row = row0 + ROWS * i + own_row;
    const One* const p = static_cast<const One*>(a.in) + (WHOLE ? row : min(row, a.rows - 1)) * a.stride;
#pragma unroll
    for (u32 h = 0; h < 2; ++h) w[i][h] = mx_load_sixteen<TYPE, EDGE>(p, col + Pack::kValues * h, a.cols);
  }
  if (!WHOLE) {
    const int left = int(max(min(i64(a.cols) - i64(col), i64(1024)), i64(0)));
    if (EDGE == kEdgeTile && col0 + PARTS * N > a.cols) {
#pragma unroll
      for (u32 i = 0; i < 4; ++i)
#pragma unroll
        for (u32 h = 0; h < 2; ++h) w[i][h] = mx_cut<TYPE>(w[i][h], left - int(Pack::kValues * h));
    }
#pragma unroll
    for (u32 i = 0; i < 4; ++i)
#pragma unroll
      for (u32 h = 0; h < 2; ++h) {
        if (row0 + ROWS * i + own_row >= a.rows) w[i][h] = u32x4_t{0, 0, 0, 0};
      }
  }
  if (DOWN) {
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      tile[(ROWS * i + own_row) * 16 + part * 2] = w[i][0];
      tile[(ROWS * i + own_row) * 16 + part * 2 + 1] = w[i][1];
    }
  }
  if (ALONG) {
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const u64 row = row0 + ROWS * i + own_row;
      u32 top = Pack::top_value(TYPE == ZC_F32 ? max(Pack::top(w[i][0]), Pack::top(w[i][1])) : max_pairs(Pack::top(w[i][0]), Pack::top(w[i][1])));
      top = max(top, u32(__builtin_amdgcn_update_dpp(0, int(top), 0xB1, 0xf, 0xf, true)));                    // quad_perm 1 0 3 2
      if (LANES == 4) top = max(top, u32(__builtin_amdgcn_update_dpp(0, int(top), 0x4E, 0xf, 0xf, true)));    // quad_perm 2 3 0 1
      const u32 s = mx_scale(top);
      const float scale = divisor_value(s);
      const u64 block = col / kBlockValues;
      if (WHOLE || (row < a.rows && block * kBlockValues < a.cols)) {
        u8* const codes = a.held.codes + row * a.held.codes_stride + col / 2;
        if constexpr (TYPE == ZC_F32) {
          const u32 eight[8] = {w[i][0][0], w[i][0][1], w[i][0][2], w[i][0][3], w[i][1][0], w[i][1][1], w[i][1][2], w[i][1][3]};
          *reinterpret_cast<u32*>(codes) = codes_if(s, mx_codes<TYPE>(eight, scale));
        } else {
          const u32 low[4] = {w[i][0][0], w[i][0][1], w[i][0][2], w[i][0][3]}, high[4] = {w[i][1][0], w[i][1][1], w[i][1][2], w[i][1][3]};
          *reinterpret_cast<u32x2_t*>(codes) = u32x2_t{codes_if(s, mx_codes<TYPE>(low, scale)), codes_if(s, mx_codes<TYPE>(high, scale))};
        }
        if (part % LANES == 0) a.held.scales[row * a.held.scales_stride + block] = u8(s);
      }
    }
  }
  if (!DOWN) return;
  __syncthreads();
  const u32 lane = tid & 63u, wave = tid >> 6;
  const u64 block = row0 / kBlockValues + wave;
  if (!WHOLE && block * kBlockValues >= a.rows) return;
  const u32* const words = reinterpret_cast<const u32*>(tile) + wave * (32 * kMxTileBytes / 4) + lane;
  u32 v[32];
  u32 top = 0;
#pragma unroll
  for (u32 r = 0; r < 32; ++r) {
    v[r] = words[r * (kMxTileBytes / 4)];
    top = TYPE == ZC_F32 ? max(top, v[r] & 0x7fffffffu) : max_pairs(top, v[r] & 0x7fff7fffu);
  }
#pragma unroll
  for (u32 h = 0; h < (TYPE == ZC_F32 ? 1u : 2u); ++h) {
    const u64 c = col0 + (TYPE == ZC_F32 ? lane : 2 * lane + h);
    if (!WHOLE && c >= a.cols) break;
    const u32 s = mx_scale(TYPE == ZC_F32 ? top : Pack::top_value(h ? top >> 16 : top & 0xffffu));
    const float scale = divisor_value(s);
    u32x4_t codes;
#pragma unroll
    for (u32 q = 0; q < 4; ++q) {
      if constexpr (TYPE == ZC_F32) {
        const u32 eight[8] = {v[8 * q], v[8 * q + 1], v[8 * q + 2], v[8 * q + 3], v[8 * q + 4], v[8 * q + 5], v[8 * q + 6], v[8 * q + 7]};
        codes[q] = codes_if(s, mx_codes<TYPE>(eight, scale));
      } else {
        u32 four[4];                                    // two rows' values of the column side by side
#pragma unroll
        for (u32 j = 0; j < 4; ++j) four[j] = __builtin_amdgcn_perm(v[8 * q + 2 * j + 1], v[8 * q + 2 * j], h ? 0x07060302u : 0x05040100u);
        codes[q] = codes_if(s, mx_codes<TYPE>(four, scale));
      }
    }
    *reinterpret_cast<u32x4_t*>(a.held_t.codes + c * a.held_t.codes_stride + kMxBytes * block) = codes;
    a.held_t.scales[c * a.held_t.scales_stride + block] = u8(s);
  }
}

template <int TYPE, bool ALONG, bool DOWN>
__global__ __launch_bounds__(256) void mx_quantize_kernel(MxQuantizeArgs a, u32 tiles_across) {
  constexpr u32 ROWS = mx_quantize_rows(DOWN), COLS = mx_quantize_cols(TYPE, DOWN);
  __shared__ u32x4_t tile[DOWN ? ROWS * kMxTileBytes / 16 : 1];
  const u32 down = blockIdx.x / tiles_across;
  const u64 row0 = u64(down) * ROWS, col0 = u64(blockIdx.x - down * tiles_across) * COLS;
  if (row0 + ROWS <= a.rows && col0 + COLS <= a.cols) mx_quantize_tile<TYPE, ALONG, DOWN, kWholeTile>(a, row0, col0, tile);
  else if (a.cols >= MxPack<TYPE>::kValues) mx_quantize_tile<TYPE, ALONG, DOWN, kEdgeTile>(a, row0, col0, tile);
  else mx_quantize_tile<TYPE, ALONG, DOWN, kNarrowTile>(a, row0, col0, tile);
}

struct MxDequantizeArgs {
  MxHeld held;
  u64 rows, cols, stride;
  void* out;
  int type;
};

// Four bytes of codes a thread and step: eight values, so that a wave's stores follow each other.  Pieces of eight are counted through the rows, `across` of them a
// row; a quotient by it is a product with `inverse` (2^32 / across rounded up), one too large at most.  A thread asks for all of its pieces before it writes the first.  Bound by
// what it writes: 8192 x 8192 to 16 bits 25.8 us (6.6 TB/s, partly from the last cache), to 32 bits 60 us (5.1 TB/s); 77 x 1001 2.0 us, a launch.
template <int TYPE, u32 PIECES>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxDequantizeArgs a, u32 across, u32 inverse, u32 pieces) {
  using One = typename ValueOf<TYPE>::One;
  const u32 first = blockIdx.x * PIECES * 256u + threadIdx.x;
  u32 rows[PIECES], parts[PIECES], words[PIECES], scales[PIECES];
#pragma unroll
  for (u32 u = 0; u < PIECES; ++u) {
    const u32 i = min(first + 256u * u, pieces - 1u);
    u32 row = across == 1 ? i : __umulhi(i, inverse);
    if (row * across > i) --row;
    rows[u] = row;
    parts[u] = i - row * across;
    words[u] = *reinterpret_cast<const u32*>(a.held.codes + row * a.held.codes_stride + 4 * u64(parts[u]));
    scales[u] = a.held.scales[row * a.held.scales_stride + parts[u] / 4];
  }
#pragma unroll
  for (u32 u = 0; u < PIECES; ++u) {
    if (first + 256u * u >= pieces) return;
    float v[8];
    mx_values(words[u], scale_value(scales[u]), v);
    const u64 col = 8 * u64(parts[u]);
    One* const to = static_cast<One*>(a.out) + rows[u] * a.stride + col;
    if (col + 8 <= a.cols) {
      struct __attribute__((packed, aligned(2))) Eight { One one[8]; } eight;
#pragma unroll
      for (u32 j = 0; j < 8; ++j) eight.one[j] = One(v[j]);
      *reinterpret_cast<Eight*>(to) = eight;
    } else {
#pragma unroll
      for (u32 j = 0; j < 8; ++j)
        if (col + j < a.cols) to[j] = One(v[j]);
    }
  }
}

}  // namespace zc
