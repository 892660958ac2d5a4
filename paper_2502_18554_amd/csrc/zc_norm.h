// Layer norm over the rows of a matrix, and its gradients.
//
// Of a row x of n values, in binary32:  mean = sum x / n,  d = 1 / sqrt(sum (x - mean)^2 / n + eps),  y = (x - mean) d w + b.
// With h = dy w and z = (x - mean) d:  dx = d (h - sum h / n - z sum (h z) / n),  dw = sum over rows of dy z,  db = sum over rows of dy.
//
// Bound by memory: a row is read once and stays in registers.  T lanes share a row, P pieces of eight values each.  The sums of a row need one exchange between
// its waves: every wave makes the sum of its values and the squares around its own mean, and the waves' squares are brought to the row's mean by
// sum (x - mean)^2 = sum over waves of [sum (x - mean_w)^2 + n_w (mean_w - mean)^2], in which no large numbers are subtracted: what the means' own roundings leave in d, relative
// to it, is no more than what they leave in (x - mean) d.
// Workgroups take rows in turn and ask for the next one before they work on this one; weights stay in registers for all of them, and so do the backward pass's sums down
// the columns, which a workgroup writes once.  A second launch adds the workgroups' sums in their order, so that equal calls give equal results.
//
// How many lanes share a row grows with its length, so that a lane has 8 to 32 values: 16 up to 128 values, a wave up to 2048, 256 up to 8192, 512 up to 16384.  Measured: 16384 rows of 4096 values,
// 32 bits to 16 with statistics, 80 us (5.0 TB/s, a copy's rate); their gradients, dx added to 32 bits, 169 us (5.6 TB/s) and 5 us for the workgroups' sums.  512 rows of 16384 values of 16 bits
// 11.6, 18 and 6.5 us: a row for each of 256 workgroups and one more, so that little is on its way at once; a row of 4096 values 3.2 us, 333 of 1001 4.7, 6 and 3.8: latency.
// Longer rows are read three times: 4096 of 32768 values of 16 bits 173 us (3.1 TB/s of what has to be read and written; 16384 values in registers 44, 6.1), their gradients 306.
#pragma once

#include "zc_rows.h"

namespace zc {

struct NormArgs {
  const void* x;
  const void* w;                 // both of w_type, both may be missing
  const void* b;
  void* out;
  float* stats;                  // means, then d's; may be missing
  u64 rows, cols, x_stride, out_stride;
  float eps;
  int x_type, w_type, out_type;
};

struct NormBackwardArgs {
  const void* dy;
  const void* x;
  const float* stats;
  const void* w;
  void* dx;                      // may be missing
  float* partial;                // [workgroup][dw, db][cols]; missing where neither is wanted
  float* row_sums;               // of the long way: [row][2]
  u64 rows, cols, dy_stride, x_stride, dx_stride;
  int dy_type, x_type, w_type, dx_type;
  u32 add;
};

template <int T>
constexpr int norm_threads() { return T < 256 ? 256 : T; }

// (sum, squares around it) or two sums of T lanes, from every wave's.  `parity` changes from row to row: one barrier a row is enough, since nobody writes a
// place again before everybody has passed the barrier behind its last reading.
template <int T>
struct NormExchange {
  float2 slot[2][T < 64 ? 1 : T / 64];
};

// How many values of a row a wave (or 16 lanes) has.
template <int T, int P>
__device__ inline u32 values_of_lanes(u64 cols, u32 t0) {
  constexpr u32 LANES = T < 64 ? T : 64;
  u32 n = 0;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const u64 first = u64(8) * (u32(p) * T + t0);
    n += cols > first ? u32(cols - first < 8 * LANES ? cols - first : 8 * LANES) : 0u;
  }
  return n;
}

template <int T, int P, bool X32>
__global__ __launch_bounds__(norm_threads<T>()) void norm_kernel(NormArgs a) {
  constexpr u32 ROWS = u32(norm_threads<T>()) / T;
  __shared__ NormExchange<T> exchange;
  const u32 t = threadIdx.x % T, group = threadIdx.x / T;
  const u32 mine = values_of_lanes<T, P>(a.cols, T < 64 ? 0u : t & ~63u);
  const float per_mine = mine ? 1.0f / float(mine) : 0.0f, per_row = 1.0f / float(a.cols);
  // A lane brings one of the waves' sums together with the others': how many values that wave has.
  const u32 of_wave = t & 15u;
  const float its = T > 64 && of_wave < T / 64 ? float(values_of_lanes<T, P>(a.cols, 64 * of_wave)) : 0.0f, per_its = its > 0.0f ? 1.0f / its : 0.0f;
  i32 left[P];
  float w[P][8], b[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const u64 col = u64(8) * (u32(p) * T + t);
    left[p] = left_of(a.cols, col);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[p][j] = 1.0f, b[p][j] = 0.0f;
  }
  const u64 step = u64(gridDim.x) * ROWS;
  u64 row = u64(blockIdx.x) * ROWS + group;
  RawEight<X32> next[P];
  const auto ask = [&](u64 r) {
#pragma unroll
    for (int p = 0; p < P; ++p) next[p] = load_eight<X32>(a.x, r * a.x_stride + u64(8) * (u32(p) * T + t), r < a.rows ? left[p] : 0);
  };
  ask(row);
  if (a.w) load_pieces<P>(a.w, a.w_type, 8 * t, 8 * T, left, w);
  if (a.b) load_pieces<P>(a.b, a.w_type, 8 * t, 8 * T, left, b);
  u32 parity = 0;
  for (u64 first = u64(blockIdx.x) * ROWS; first < a.rows; first += step, row += step) {       // (the same for all threads)
    float x[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) numbers_of<X32>(next[p], a.x_type, x[p]);
    ask(row + step);
    float sum = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += x[p][j];          // (zeros where there are no values)
    sum = T < 64 ? sum_of_16(sum) : sum_of_wave(sum);
    float mean = sum * per_mine, squares = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if (left[p] >= 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) squares = __builtin_fmaf(x[p][j] - mean, x[p][j] - mean, squares);
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j) squares = j < left[p] ? __builtin_fmaf(x[p][j] - mean, x[p][j] - mean, squares) : squares;
      }
    }
    squares = T < 64 ? sum_of_16(squares) : sum_of_wave(squares);
    if constexpr (T > 64) {
      if ((t & 63u) == 0) exchange.slot[parity][t >> 6] = make_float2(sum, squares);
      __syncthreads();
      const float2 of = of_wave < T / 64 ? exchange.slot[parity][of_wave] : make_float2(0.0f, 0.0f);
      mean = sum_of_16(of.x) * per_row;
      const float off = its > 0.0f ? of.x * per_its - mean : 0.0f;       // (of a lane without a wave it would be the mean, whose square may pass binary32)
      squares = sum_of_16(__builtin_fmaf(off * off, its, of.y));
      parity ^= 1u;
    }
    const float d = 1.0f / sqrtf(__builtin_fmaf(squares, per_row, a.eps));
    if (row < a.rows) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf((x[p][j] - mean) * d, w[p][j], b[p][j]);
        store_numbers(a.out, a.out_type, row * a.out_stride + u64(8) * (u32(p) * T + t), left[p], y);
      }
      if (a.stats && t == 0) {
        a.stats[row] = mean;
        a.stats[a.rows + row] = d;
      }
    }
  }
}

template <int T, int P, bool X32, bool DY32>
__global__ __launch_bounds__(norm_threads<T>()) void norm_backward_kernel(NormBackwardArgs a) {
  constexpr u32 W = u32(norm_threads<T>()), ROWS = W / T;
  // In LDS: the rows' sums, and behind the rows the groups' sums down the columns.
  __shared__ union { NormExchange<T> exchange; float columns[ROWS > 1 ? ROWS : 1][ROWS > 1 ? 8 * P * T : 1]; } lds;
  const u32 t = threadIdx.x % T, group = threadIdx.x / T;
  const float per_row = 1.0f / float(a.cols);
  i32 left[P];
  float w[P][8], dw[P][8], db[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const u64 col = u64(8) * (u32(p) * T + t);
    left[p] = left_of(a.cols, col);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[p][j] = 1.0f, dw[p][j] = 0.0f, db[p][j] = 0.0f;
  }
  const u64 step = u64(gridDim.x) * ROWS;
  u64 row = u64(blockIdx.x) * ROWS + group;
  // (Two rows of 32-bit values of this length do not fit into the registers of two waves.)
  constexpr bool AHEAD = !(T == 512 && (X32 || DY32));
  constexpr bool CHOOSE = T <= 64;
  RawEight<X32> next_x[P];
  RawEight<DY32> next_dy[P];
  float next_mean, next_d;
  const auto ask = [&](u64 r) {
    const bool there = r < a.rows;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const u64 col = u64(8) * (u32(p) * T + t);
      next_x[p] = load_eight<X32>(a.x, r * a.x_stride + col, there ? left[p] : 0);
      next_dy[p] = load_eight<DY32>(a.dy, r * a.dy_stride + col, there ? left[p] : 0);
    }
    next_mean = there ? a.stats[r] : 0.0f;
    next_d = there ? a.stats[a.rows + r] : 0.0f;
  };
  if constexpr (P <= 2) {
    if (a.w) load_pieces<P>(a.w, a.w_type, 8 * t, 8 * T, left, w);
  } else if (a.w) {                                        // (one by one: the registers are full)
#pragma unroll
    for (int p = 0; p < P; ++p) load_numbers(a.w, a.w_type, u64(8) * (u32(p) * T + t), left[p], w[p]);
  }
  if (AHEAD) ask(row);
  u32 parity = 0;
  for (u64 first = u64(blockIdx.x) * ROWS; first < a.rows; first += step, row += step) {
    float z[P][8], dy[P][8];
    if (!AHEAD) ask(row);
    const float mean = next_mean, d = next_d;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      numbers_of<X32>(next_x[p], a.x_type, z[p]);
      numbers_of<DY32>(next_dy[p], a.dy_type, dy[p]);
    }
    // Where there are no values, h is 0 and z = -mean d, which has to be 0 where it passes binary32, since 0 x infinity is NaN.  Chosen value by value, or by a branch that ordinary rows pass by:
    // 65536 x 100 in 32 bits 21.6 us and 22.8, 333 x 1001 9.1 and 9.5; 4096 x 8190 121 and 112, 8192 x 2050 in 16 bits 44.7 and 43.7 (without either 21.5, 9.1, 116 and 42.5).
    if (!CHOOSE && !(fabsf(mean * d) < __builtin_inff())) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[p][j] = j < left[p] ? z[p][j] : mean;
    }
    if (AHEAD) ask(row + step);
    float old[P <= 2 ? P : 1][8];                          // what dx is added to
    if constexpr (P <= 2) if (a.dx && a.add && row < a.rows) load_pieces<P>(a.dx, a.dx_type, row * a.dx_stride + 8 * t, 8 * T, left, old);
    float one = 0.0f, two = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[p][j] = (z[p][j] - mean) * d;
        if (CHOOSE) z[p][j] = j < left[p] ? z[p][j] : 0.0f;
        const float h = dy[p][j] * w[p][j];                // (0 where there are no values)
        one += h;
        two = __builtin_fmaf(h, z[p][j], two);
        dw[p][j] = __builtin_fmaf(dy[p][j], z[p][j], dw[p][j]);
        db[p][j] += dy[p][j];
      }
    }
    one = T < 64 ? sum_of_16(one) : sum_of_wave(one);
    two = T < 64 ? sum_of_16(two) : sum_of_wave(two);
    if constexpr (T > 64) {
      if ((t & 63u) == 0) lds.exchange.slot[parity][t >> 6] = make_float2(one, two);
      __syncthreads();
      const u32 of_wave = t & 15u;
      const float2 of = of_wave < T / 64 ? lds.exchange.slot[parity][of_wave] : make_float2(0.0f, 0.0f);
      one = sum_of_16(of.x);
      two = sum_of_16(of.y);
      parity ^= 1u;
    }
    one *= per_row;
    two *= per_row;
    if (a.dx && row < a.rows) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const u64 at = row * a.dx_stride + u64(8) * (u32(p) * T + t);
        float v[8];
        if (P > 2 && a.add) load_numbers(a.dx, a.dx_type, at, left[p], old[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float g = d * (__builtin_fmaf(dy[p][j], w[p][j], -one) - z[p][j] * two);
          v[j] = a.add ? old[P <= 2 ? p : 0][j] + g : g;
        }
        store_numbers(a.dx, a.dx_type, at, left[p], v);
      }
    }
  }
  if (!a.partial) return;
  float* const to = a.partial + u64(blockIdx.x) * 2 * a.cols;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const u64 col = u64(8) * (u32(p) * T + t);
      store_eight<true>(to, ZC_F32, col, left[p], dw[p]);
      store_eight<true>(to, ZC_F32, a.cols + col, left[p], db[p]);
    }
  } else {
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) lds.columns[group][8 * (p * T + t) + j] = which ? db[p][j] : dw[p][j];
      __syncthreads();
      for (u32 col = threadIdx.x; col < a.cols; col += W) {
        float sum = 0.0f;
#pragma unroll
        for (u32 g = 0; g < ROWS; ++g) sum += lds.columns[g][col];
        to[which * a.cols + col] = sum;
      }
    }
  }
}

// The workgroups' sums down the columns, added in their order (16 strands of them, then these): 64 columns a workgroup.
struct NormColumnsArgs {
  const float* partial;
  void* to[2];                   // dw, db
  u64 cols;
  u32 groups;
  int type;
  u32 add;
};
constexpr u32 kNormStrands = 16;
__global__ __launch_bounds__(1024) void norm_columns_kernel(NormColumnsArgs a) {
  __shared__ float strand[kNormStrands][64];
  const u32 lane = threadIdx.x & 63u, s = threadIdx.x >> 6;
  const u64 col = u64(blockIdx.x) * 64 + lane;
  void* const to = a.to[blockIdx.y];
  if (!to) return;
  float sum = 0.0f;
  if (col < a.cols) {
    const float* from = a.partial + u64(blockIdx.y) * a.cols + col;
#pragma unroll 8
    for (u32 g = s; g < a.groups; g += kNormStrands) sum += from[u64(g) * 2 * a.cols];
  }
  strand[s][lane] = sum;
  __syncthreads();
  if (s || col >= a.cols) return;
  sum = 0.0f;
#pragma unroll
  for (u32 k = 0; k < kNormStrands; ++k) sum += strand[k][lane];
  if (a.add) sum += load_value(to, a.type, col);
  store_value(to, a.type, col, sum);
}

// ---- Rows of more values than a workgroup holds: read several times, from the caches where they fit there.

// A sum over the workgroup, the same in all threads.
__device__ inline float sum_of_1024(float x, float (&slot)[16]) {
  x = sum_of_wave(x);
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) slot[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.0f;
#pragma unroll
  for (int k = 0; k < 16; ++k) x += slot[k];
  return x;
}

__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float slot[16];
  const float per_row = 1.0f / float(a.cols);
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float sum = 0.0f, squares = 0.0f;
    for (u64 col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float x[8];
      load_numbers(a.x, a.x_type, row * a.x_stride + col, left_of(a.cols, col), x);
      sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    const float mean = sum_of_1024(sum, slot) * per_row;
    for (u64 col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float x[8];
      const i32 left = left_of(a.cols, col);
      load_numbers(a.x, a.x_type, row * a.x_stride + col, left, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) squares = j < left ? __builtin_fmaf(x[j] - mean, x[j] - mean, squares) : squares;
    }
    const float d = 1.0f / sqrtf(__builtin_fmaf(sum_of_1024(squares, slot), per_row, a.eps));
    for (u64 col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float x[8], w[8], b[8];
      const i32 left = left_of(a.cols, col);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 1.0f, b[j] = 0.0f;
      load_numbers(a.x, a.x_type, row * a.x_stride + col, left, x);
      if (a.w) load_numbers(a.w, a.w_type, col, left, w);
      if (a.b) load_numbers(a.b, a.w_type, col, left, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf((x[j] - mean) * d, w[j], b[j]);
      store_numbers(a.out, a.out_type, row * a.out_stride + col, left, x);
    }
    if (a.stats && threadIdx.x == 0) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = d;
    }
  }
}

// First launch: the two sums of every row.
__global__ __launch_bounds__(1024) void norm_long_sums_kernel(NormBackwardArgs a) {
  __shared__ float slot[16];
  const float per_row = 1.0f / float(a.cols);
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.stats[row], d = a.stats[a.rows + row];
    float one = 0.0f, two = 0.0f;
    for (u64 col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float x[8], dy[8], w[8];
      const i32 left = left_of(a.cols, col);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 1.0f;
      load_numbers(a.x, a.x_type, row * a.x_stride + col, left, x);
      load_numbers(a.dy, a.dy_type, row * a.dy_stride + col, left, dy);
      if (a.w) load_numbers(a.w, a.w_type, col, left, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float h = dy[j] * w[j];
        one += h;
        two = j < left ? __builtin_fmaf(h, (x[j] - mean) * d, two) : two;       // (-mean d may pass binary32)
      }
    }
    one = sum_of_1024(one, slot);
    two = sum_of_1024(two, slot);
    if (threadIdx.x == 0) {
      a.row_sums[2 * row] = one * per_row;
      a.row_sums[2 * row + 1] = two * per_row;
    }
  }
}
// Second launch: a workgroup has 2048 columns (blockIdx.x) of every gridDim.y-th row.
__global__ __launch_bounds__(256) void norm_long_backward_kernel(NormBackwardArgs a) {
  const u64 col = u64(blockIdx.x) * 2048 + 8 * threadIdx.x;
  const i32 left = left_of(a.cols, col);
  float w[8], dw[8] = {}, db[8] = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = 1.0f;
  if (a.w) load_numbers(a.w, a.w_type, col, left, w);
  for (u64 row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float mean = a.stats[row], d = a.stats[a.rows + row], one = a.row_sums[2 * row], two = a.row_sums[2 * row + 1];
    const u64 at = row * a.dx_stride + col;
    float x[8], dy[8], v[8];
    load_numbers(a.x, a.x_type, row * a.x_stride + col, left, x);
    load_numbers(a.dy, a.dy_type, row * a.dy_stride + col, left, dy);
    if (a.dx && a.add) load_numbers(a.dx, a.dx_type, at, left, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float z = (x[j] - mean) * d, g = d * (__builtin_fmaf(dy[j], w[j], -one) - z * two);
      dw[j] = __builtin_fmaf(dy[j], z, dw[j]);
      db[j] += dy[j];
      v[j] = a.add ? v[j] + g : g;
    }
    if (a.dx) store_numbers(a.dx, a.dx_type, at, left, v);
  }
  if (!a.partial) return;
  float* const to = a.partial + u64(blockIdx.y) * 2 * a.cols;
  store_eight<true>(to, ZC_F32, col, left, dw);
  store_eight<true>(to, ZC_F32, a.cols + col, left, db);
}

}  // namespace zc
