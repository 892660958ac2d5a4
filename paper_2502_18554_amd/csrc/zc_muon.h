// The optimiser's step for matrices: momentum, made nearly orthogonal by Newton-Schulz products, into the weights.
//
//   g = grad x scale;  m' = mu m + (1 - mu) g;  u = mu m' + (1 - mu) g, or m' itself
//   X = u / max(|u|, 1e-7) with the root of the sum of squares for |u|, turned where it has more rows than columns: r x c, r <= c
//   several times:  A = X X^T;  B = b A + c A A;  X = a X + B X        (a, b, c) = (3.4445, -4.7750, 2.0315)
//   p' = p (1 - lr decay) - lr factor X
// The polynomial a s + b s^3 + c s^5 takes the singular values s from (0, 1] towards 1: from 0.002 on they are between 0.68 and 1.21 after five times, and never above 1.21
// (Jordan et al., "Muon", 2024, from where the coefficients are).
//
// The products are the matrix instructions' in binary16, with sums in binary32.  X, A and B are kept times 2^12: their entries are at most 1.21, 1.5 and 2.9, so that
// nothing overflows, and typical ones (1 / sqrt(r c) at first, 2^-12 for 4096 x 4096) are far from the smallest normal one.  An operand of one binary16 number has 11 bits: each
// product's result is rounded by 2^-12 of itself, eight times less than bfloat16 would.  Where that is too much (weights in 32 bits), an operand is two binary16 numbers, 22 bits, and a product
// three of theirs: high high + high low + low high.
//
// A and B are symmetric: the tiles on and under the diagonal are computed and written twice.  X is kept as it is and turned, since the instructions take both operands along
// the sum: X X^T sums along the columns, B X along the rows.  All matrices of a list go through each product in one launch.
#pragma once

#include <utility>

#include "zc_rows.h"

namespace zc {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) u32 LdsWord;

constexpr int kMuonTensors = 64;                     // of one launch: their table travels in the kernel's arguments
constexpr u32 kMuonAlong = 128;                      // rows of X, A, B and of X turned are filled up with zeros to a multiple of so many values
constexpr float kMuonA = 3.4445f, kMuonB = -4.7750f, kMuonC = 2.0315f;
constexpr float kMuonScale = 4096.0f;

__host__ __device__ inline u64 muon_along(u64 n) { return (n + kMuonAlong - 1) / kMuonAlong * kMuonAlong; }

struct MuonTensor {
  u8* at;                        // in the workspace
  void* param;
  void* copy;
  const void* grad;
  float* m;
  u32 r, c;                      // r <= c
  u32 first;                     // of its tiles (or workgroups) in the launch
  float step;                    // lr factor
};
struct MuonArgs {
  MuonTensor t[kMuonTensors];
  u32 turned[(kMuonTensors + 31) / 32];
  u32 tensors;
  u32 count;                     // tiles (or workgroups) of the launch
  u32 planes;                    // 1 or 2
  u32 which;                     // of the two turned X
  const float* grad_scale;
  double* partial;               // [tensor][kMuonPartials]
  float keep, mu, rest;          // 1 - lr decay; mu, 1 - mu
  u32 nesterov;
  int param_type, grad_type, copy_type;
};
static_assert(sizeof(MuonArgs) <= 4096);
__device__ inline bool turned(const MuonArgs& a, u32 i) { return a.turned[i / 32] >> (i % 32) & 1u; }

// Places of a matrix's parts in its share of the workspace: X, X turned twice (one is read while the other is written), A, B; the low parts of two behind the high ones of each.
struct MuonParts {
  u64 row_x, row_t;                                  // values of a row of X; of X turned, A and B
  u64 plane_x, plane_t, plane_a;                     // bytes
  u64 x, t0, t1, a, b, bytes;
  __host__ __device__ MuonParts(u32 r, u32 c, u32 planes) {
    row_x = muon_along(c), row_t = muon_along(r);
    plane_x = 2 * r * row_x, plane_t = 2 * c * row_t, plane_a = 2 * r * row_t;
    x = 0;
    t0 = x + planes * plane_x;
    t1 = t0 + planes * plane_t;
    a = t1 + planes * plane_t;
    b = a + planes * plane_a;
    bytes = b + planes * plane_a;
  }
};

// The matrix that a tile or workgroup belongs to.
__device__ inline u32 muon_tensor_of(const MuonArgs& a, u32 tile) {
  u32 i = 0;
  while (i + 1 < a.tensors && a.t[i + 1].first <= tile) ++i;
  return i;
}

// ---- Momentum, and the sum of u's squares: in 64 bits, by workgroups whose sums the next launch adds.
constexpr u32 kMuonPartials = 512;
constexpr u32 kMuonPiece = 2048;                     // values that a workgroup takes at a time
__host__ __device__ inline u32 muon_partials(u64 values) {
  const u64 pieces = (values + kMuonPiece - 1) / kMuonPiece;
  return u32(pieces < kMuonPartials ? pieces : kMuonPartials);
}

__device__ inline double sum_of_256(double x, double (&slot)[4]) {
#pragma unroll
  for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s, 64);
  if ((threadIdx.x & 63u) == 0) slot[threadIdx.x >> 6] = x;
  __syncthreads();
  return (slot[0] + slot[1]) + (slot[2] + slot[3]);
}

__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonArgs a) {
  __shared__ double slot[4];
  const float scale = a.grad_scale ? *a.grad_scale : 1.0f;
  if (!(fabsf(scale) < __builtin_inff())) return;
  const u32 i = muon_tensor_of(a, blockIdx.x), part = blockIdx.x - a.t[i].first;
  const u64 values = u64(a.t[i].r) * a.t[i].c;
  const u32 parts = muon_partials(values);
  double sum = 0.0;
  for (u64 at = u64(part) * kMuonPiece + 8 * threadIdx.x; at < values; at += u64(parts) * kMuonPiece) {
    const i32 left = left_of(values, at);
    float g[8], m[8];
    load_numbers(a.t[i].grad, a.grad_type, at, left, g);
    load_numbers(a.t[i].m, ZC_F32, at, left, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[j] = a.rest * (g[j] * scale);
      m[j] = __builtin_fmaf(a.mu, m[j], g[j]);
      const double u = a.nesterov ? __builtin_fmaf(a.mu, m[j], g[j]) : m[j];
      sum = __builtin_fma(u, u, sum);
    }
    store_numbers(a.t[i].m, ZC_F32, at, left, m);
  }
  sum = sum_of_256(sum, slot);
  if (threadIdx.x == 0) a.partial[u64(i) * kMuonPartials + part] = sum;
}

// The parts of a value in binary16.
__device__ inline void halves_of(float v, u32 planes, _Float16& high, _Float16& low) {
  high = _Float16(v);
  low = planes > 1 ? _Float16(v - float(high)) : _Float16(0.0f);
}

// ---- X, as it is and turned, from m' and the gradient: tiles of 64 x 64 of the matrix as it lies in memory.
__global__ __launch_bounds__(256) void muon_begin_kernel(MuonArgs a) {
  __shared__ double slot[4];
  __shared__ float tile[64][65];
  const float scale = a.grad_scale ? *a.grad_scale : 1.0f;
  const u32 i = muon_tensor_of(a, blockIdx.x), r = a.t[i].r, c = a.t[i].c;
  const bool turn = turned(a, i);
  const u64 rows = turn ? c : r, cols = turn ? r : c;
  const MuonParts parts(r, c, a.planes);
  const u32 across = u32(muon_along(cols) / 64), t = blockIdx.x - a.t[i].first;
  const u64 row0 = u64(t / across) * 64, col0 = u64(t % across) * 64;
  const u32 n = muon_partials(rows * cols);
  double sum = 0.0;
  for (u32 k = threadIdx.x; k < n; k += 256) sum += a.partial[u64(i) * kMuonPartials + k];
  const double norm = __builtin_sqrt(sum_of_256(sum, slot));
  const float factor = float(4096.0 / (norm < 1e-7 ? 1e-7 : norm));
  // As it lies in memory: a thread has eight values of rows threadIdx.x / 8 and 32 more.
  const u64 plane = turn ? parts.plane_t : parts.plane_x, along = turn ? parts.row_t : parts.row_x, to = turn ? parts.t0 : parts.x;
#pragma unroll
  for (u32 h = 0; h < 2; ++h) {
    const u64 row = row0 + (threadIdx.x >> 3) + 32 * h, col = col0 + 8 * (threadIdx.x & 7u);
    const i32 left = row < rows ? left_of(cols, col) : 0;
    float m[8], g[8] = {};
    load_numbers(a.t[i].m, ZC_F32, row * cols + col, left, m);
    if (a.nesterov) load_numbers(a.t[i].grad, a.grad_type, row * cols + col, left, g);
    f16x8_t high, low;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = a.nesterov ? __builtin_fmaf(a.mu, m[j], a.rest * (g[j] * scale)) : m[j];
      const float x = j < left ? u * factor : 0.0f;
      tile[(threadIdx.x >> 3) + 32 * h][8 * (threadIdx.x & 7u) + j] = x;
      _Float16 one, two;
      halves_of(x, a.planes, one, two);
      high[j] = one, low[j] = two;
    }
    if (row < rows) {
      u8* const place = a.t[i].at + to + 2 * (row * along + col);
      *reinterpret_cast<f16x8_t*>(place) = high;
      if (a.planes > 1) *reinterpret_cast<f16x8_t*>(place + plane) = low;
    }
  }
  __syncthreads();
  const u64 plane_2 = turn ? parts.plane_x : parts.plane_t, along_2 = turn ? parts.row_x : parts.row_t, to_2 = turn ? parts.x : parts.t0;
#pragma unroll
  for (u32 h = 0; h < 2; ++h) {
    const u64 col = col0 + (threadIdx.x >> 3) + 32 * h, row = row0 + 8 * (threadIdx.x & 7u);
    f16x8_t high, low;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      _Float16 one, two;
      halves_of(tile[8 * (threadIdx.x & 7u) + j][(threadIdx.x >> 3) + 32 * h], a.planes, one, two);
      high[j] = one, low[j] = two;
    }
    if (col < cols && row < along_2) {
      u8* const place = a.t[i].at + to_2 + 2 * (col * along_2 + row);
      *reinterpret_cast<f16x8_t*>(place) = high;
      if (a.planes > 1) *reinterpret_cast<f16x8_t*>(place + plane_2) = low;
    }
  }
}

// Zeros behind the rows of A, B and the other X turned: the products write values only.  A thread has a row.
__global__ __launch_bounds__(256) void muon_zeros_kernel(MuonArgs a) {
  const u32 i = muon_tensor_of(a, blockIdx.x), r = a.t[i].r, c = a.t[i].c;
  const MuonParts parts(r, c, a.planes);
  const u32 row = (blockIdx.x - a.t[i].first) * 256 + threadIdx.x;
  for (u32 plane = 0; plane < a.planes; ++plane)
    for (u64 col = r; col < parts.row_t; ++col) {
      if (row < c) *reinterpret_cast<_Float16*>(a.t[i].at + parts.t1 + plane * parts.plane_t + 2 * (row * parts.row_t + col)) = _Float16(0.0f);
      if (row < r) {
        *reinterpret_cast<_Float16*>(a.t[i].at + parts.a + plane * parts.plane_a + 2 * (row * parts.row_t + col)) = _Float16(0.0f);
        *reinterpret_cast<_Float16*>(a.t[i].at + parts.b + plane * parts.plane_a + 2 * (row * parts.row_t + col)) = _Float16(0.0f);
      }
    }
}

// ---- The products.  Workgroups of 2 x 2 waves make tiles of 64 T x 64 T results, a wave 32 T x 32 T.
//
// A stage is 64 values (128 bytes) of every row of the tile, brought straight to LDS while the stage before is multiplied.  Rows follow each other in LDS, their eight
// 16-byte blocks exchanged by the row's number, so that 16 lanes that read LDS together find 64 different banks.  An instruction multiplies eight values of 32 rows with as many of 32
// columns from lanes 0 .. 31, eight others from lanes 32 .. 63: blocks t and 4 + t of the stage.  Which column of the tile a lane brings is free: it is chosen so that a lane ends with 16
// neighbouring results of a row.  The requests run two stages ahead, into the workgroup's next tile too.
enum { kMuonGram, kMuonPoly, kMuonUpdate, kMuonFinish };       // kMuonFinish + the weights' type

// Rows of a tile as a buffer, seen from some bytes along them: rows behind the last one read as zeros.
struct MuonRows {
  u64 at;
  u32 bytes;
  __device__ void aim(const u8* base, u64 first, u64 rows, u64 stride, u32 most) {
    at = reinterpret_cast<u64>(base) + first * stride;
    bytes = u32(min(rows - first, u64(most)) * stride);
  }
  __device__ void move_on(u32 by) {
    at += by;
    bytes = bytes > by ? bytes - by : 0u;
  }
  __device__ __amdgpu_buffer_rsrc_t buffer() const {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u64(uniform(u32(at))) | u64(uniform(u32(at >> 32))) << 32), 0, int(uniform(bytes)), 0x00027000);
  }
};

// 16 bytes a lane to LDS, at `to` and on.  (Written out: of its own loads to LDS the compiler thinks that any read of LDS may have to wait for them.  m0 is reserved, so
// that it cannot be named among what is overwritten: nothing else in these kernels may use it.)
__device__ inline void muon_load_to_lds(__amdgpu_buffer_rsrc_t from, u32 to, u32 lane_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(lane_offset), "s"(from) : "memory");
}
// Keeps an instruction's sums at their place, in the matrix instructions' own registers where a wave has more of them than the others would hold.
template <int OF>
__device__ __forceinline__ void muon_hold(f32x16_t& sum) {
  if constexpr (OF > 4) asm volatile("" : "+a"(sum));
  else asm volatile("" : "+v"(sum));
}

// The tiles of a launch, and the operands of one.
template <int MODE>
struct MuonTiles {
  static constexpr bool kTriangle = MODE == kMuonGram || MODE == kMuonPoly;
  u32 first, end, step;                              // the workgroup's own
  __device__ explicit MuonTiles(u32 tiles) {         // every XCD has a run of neighbouring tiles (workgroups go round the eight XCDs)
    const u32 xcd = blockIdx.x & 7u, share = tiles >> 3, more = tiles & 7u, begin = xcd * share + min(xcd, more);
    first = begin + (blockIdx.x >> 3);
    end = begin + share + (xcd < more ? 1u : 0u);
    step = (gridDim.x + 7u - xcd) >> 3;
  }
  // Row and column of tile t of a matrix whose results are `down` x `across` tiles.
  __device__ static void place(u32 t, u32 down, u32 across, u32& row, u32& col) {
    if constexpr (kTriangle) {
      u32 i = u32((sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
      while (i * (i + 1) / 2 > t) --i;
      while ((i + 1) * (i + 2) / 2 <= t) ++i;
      row = uniform(i);
      col = uniform(t - i * (i + 1) / 2);
    } else {
      const u32 strip = t / (8u * across), rest = t - strip * 8u * across, high = min(8u, down - 8u * strip), c = rest / high;
      col = uniform(c);
      row = uniform(8u * strip + rest - c * high);
    }
  }
};

// Sixteen neighbouring values of a row of X, A or B as numbers, as far as there are any.
__device__ inline void sixteen_of(const u8* from, u64 plane, u32 planes, float (&v)[16]) {
#pragma unroll
  for (u32 h = 0; h < 2; ++h) {
    const f16x8_t high = *reinterpret_cast<const f16x8_t*>(from + 16 * h);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[8 * h + j] = float(high[j]);
    if (planes > 1) {
      const f16x8_t low = *reinterpret_cast<const f16x8_t*>(from + plane + 16 * h);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[8 * h + j] += float(low[j]);
    }
  }
}

template <int T, int MODE>
__global__ __launch_bounds__(256, T == 4 ? 1 : T == 2 ? 2 : 4) void muon_product_kernel(MuonArgs a) {
  constexpr u32 R = 64u * T, LOADS = 2 * R / 32;
  constexpr u32 AT_B = 2 * R * 128;
  __shared__ u32x4_t memory[2 * AT_B / 16];
  const u32 tid = threadIdx.x, lane = tid & 63u, wave = uniform(tid >> 6), half = lane >> 5, in32 = lane & 31u;
  const MuonTiles<MODE> tiles(a.count);
  if (tiles.first >= tiles.end) return;

  // What is asked for next: a tile's rows, and how far along them.
  u32 ask_tile = tiles.first, ask_pair = 0, ask_pairs = 0, ask_segment = 0;
  u32 ask_stride_a = 0, ask_stride_b = 0;
  MuonRows rows_a, rows_b;
  const u32 my_row = tid >> 3;
  const u32 block_a = 16u * ((tid ^ (my_row >> 1)) & 7u), block_b = 16u * ((tid ^ (((my_row >> 1) & 1u) | ((my_row >> 3) & 2u) | (my_row & 4u))) & 7u);
  const auto aim = [&] {
    const u32 i = muon_tensor_of(a, ask_tile), r = a.t[i].r, c = a.t[i].c;
    const MuonParts parts(r, c, a.planes);
    u32 row, col;
    const u32 down = (r + R - 1) / R, across = MODE == kMuonGram || MODE == kMuonPoly ? down : (c + R - 1) / R;
    MuonTiles<MODE>::place(ask_tile - a.t[i].first, down, across, row, col);
    const u8* const at = a.t[i].at;
    const u64 plane_a = MODE == kMuonGram ? parts.plane_x : parts.plane_a, plane_b = MODE == kMuonGram ? parts.plane_x : MODE == kMuonPoly ? parts.plane_a : parts.plane_t;
    const u8* const from_a = at + (MODE == kMuonGram ? parts.x : MODE == kMuonPoly ? parts.a : parts.b) + (ask_segment == 2 ? plane_a : 0);
    const u8* const from_b = at + (MODE == kMuonGram ? parts.x : MODE == kMuonPoly ? parts.a : a.which ? parts.t1 : parts.t0) + (ask_segment == 1 ? plane_b : 0);
    const u64 along = MODE == kMuonGram ? parts.row_x : parts.row_t;
    rows_a.aim(from_a, u64(row) * R, r, 2 * along, R);
    rows_b.aim(from_b, u64(col) * R, MODE == kMuonGram || MODE == kMuonPoly ? r : c, 2 * along, R);
    ask_stride_a = ask_stride_b = uniform(u32(2 * along));
    ask_pairs = uniform(u32(along / 128));
  };
  // (Behind the last tile there is nothing to ask for.)
  const auto next_pair = [&] {
    if (++ask_pair < ask_pairs) return;
    ask_pair = 0;
    if (a.planes > 1 && ++ask_segment < 3) {
      aim();
      return;
    }
    ask_segment = 0;
    ask_tile += tiles.step;
    if (ask_tile < tiles.end) aim();
    else rows_a.bytes = rows_b.bytes = 0;
  };
  const u32 lds0 = u32(reinterpret_cast<uintptr_t>((LdsWord*)&memory[0]));
  const auto ask = [&](u32 u, u32 i) {
    const u32 to = lds0 + wave * 1024u;
    if (i < R / 32) muon_load_to_lds(rows_a.buffer(), to + u * (R * 128u) + 4096u * i, (my_row + 32 * i) * ask_stride_a + block_a);
    else muon_load_to_lds(rows_b.buffer(), to + AT_B + u * (R * 128u) + 4096u * (i - R / 32), (my_row + 32 * (i - R / 32)) * ask_stride_b + block_b);
  };
  const auto next_stage = [&] {
    rows_a.move_on(128);
    rows_b.move_on(128);
  };

  const u32 wave_a = (wave >> 1) * 32u * T, wave_b = (wave & 1u) * 32u * T;
  const u32 lane_b = (in32 & 3u) + 16u * ((in32 >> 2) & 1u) + 4u * (in32 >> 3);
  u32x4_t fa[2][T], fb[2][T];                        // of this step and of the next one
  u32 at_a[4], at_b[4];                              // where a lane's block of step t is, in the first stage's place
#pragma unroll
  for (u32 t = 0; t < 4; ++t) {
    at_a[t] = lds0 + (wave_a + in32) * 128u + 16u * ((4 * half + t) ^ (in32 >> 1 & 7u));
    at_b[t] = lds0 + AT_B + (wave_b + lane_b) * 128u + 16u * ((4 * half + t) ^ (((lane_b >> 1) & 1u) | ((lane_b >> 3) & 2u) | (lane_b & 4u)));
  }
  typedef const __attribute__((address_space(3))) u32x4_t LdsBlock;
  const auto read = [&](u32 buffer, u32 t, u32 i) {
    if (i < T) fa[t & 1][i] = *reinterpret_cast<LdsBlock*>(at_a[t] + (buffer * R * 128u + 4096u * i));
    else fb[t & 1][i - T] = *reinterpret_cast<LdsBlock*>(at_b[t] + (buffer * R * 128u + 4096u * (i - T)));
  };

  constexpr u32 SLOTS = T * T, READS = 2 * T, EARLY = LOADS / 2;
  aim();
#pragma unroll
  for (u32 i = 0; i < LOADS; ++i) ask(0, i);
  next_stage();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (u32 i = 0; i < EARLY; ++i) ask(1, i);
#pragma unroll
  for (u32 i = 0; i < READS; ++i) read(0, 0, i);
  for (u32 tile = tiles.first; tile < tiles.end; tile += tiles.step) {
    const u32 ti = muon_tensor_of(a, tile), r = a.t[ti].r, c = a.t[ti].c;
    const MuonParts parts(r, c, a.planes);
    const u32 pairs = uniform(u32((MODE == kMuonGram ? parts.row_x : parts.row_t) / 128) * (a.planes > 1 ? 3u : 1u));
    f32x16_t sum[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[i][j][k] = 0.0f;
    for (u32 pair = 0; pair < pairs; ++pair) {
#pragma unroll
      for (u32 u = 0; u < 2; ++u) {
#pragma unroll
        for (u32 t = 0; t < 4; ++t) {
          if (t == 3) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
          }
#pragma unroll
          for (u32 slot = 0; slot < SLOTS; ++slot) {
#pragma unroll
            for (u32 i = 0; i < EARLY; ++i) {
              if (i * SLOTS / EARLY != slot) continue;
              if (t == 3) ask(u, i);
              if (t == 0) ask(u ^ 1u, EARLY + i);
            }
#pragma unroll
            for (u32 i = 0; i < READS; ++i)
              if (i * SLOTS / (2 * READS) == slot) read(t < 3 ? u : u ^ 1, (t + 1) & 3u, i);
            const u32 i = slot / T, j = slot % T;
            sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, fb[t & 1][j]), __builtin_bit_cast(f16x8_t, fa[t & 1][i]), sum[i][j], 0, 0, 0);
            muon_hold<T * T>(sum[i][j]);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (t == 0) next_stage();
          if (u == 0 && t == 0) next_pair();
        }
      }
    }
    // The results.
    u32 down, across;
    const u32 tiles_down = (r + R - 1) / R, tiles_across = MODE == kMuonGram || MODE == kMuonPoly ? tiles_down : (c + R - 1) / R;
    MuonTiles<MODE>::place(tile - a.t[ti].first, tiles_down, tiles_across, down, across);
    const u64 row0 = u64(down) * R + wave_a + in32, col0 = u64(across) * R + wave_b + 16 * half;
    const u64 cols = MODE == kMuonGram || MODE == kMuonPoly ? r : c;
    u8* const at = a.t[ti].at;
    const bool turn = MODE >= kMuonFinish && turned(a, ti);
    if (MODE >= kMuonFinish && a.grad_scale && !(fabsf(*a.grad_scale) < __builtin_inff())) continue;
    const auto write = [&](auto number) __attribute__((always_inline)) {
        constexpr int i = decltype(number)::value / T, j = decltype(number)::value % T;
        muon_hold<T * T>(sum[i][j]);
        const u64 row = row0 + 32 * i, col = col0 + 32 * j;
        const i32 left = row < r && col < cols ? i32(min(cols - col, u64(16))) : 0;
        if (left > 0) {
        // (Values behind the matrix's columns are zeros, there and in the workspace, whose rows go on to a multiple of 128.)
        float v[16], old[16];
        if constexpr (MODE == kMuonGram) {
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = sum[i][j][k] * (1.0f / kMuonScale);
        } else if constexpr (MODE == kMuonPoly) {
          sixteen_of(at + parts.a + 2 * (row * parts.row_t + col), parts.plane_a, a.planes, old);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = __builtin_fmaf(old[k], kMuonB, sum[i][j][k] * (kMuonC / kMuonScale));
        } else {
          sixteen_of(at + parts.x + 2 * (row * parts.row_x + col), parts.plane_x, a.planes, old);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = __builtin_fmaf(old[k], kMuonA, sum[i][j][k] * (1.0f / kMuonScale));
        }
        if constexpr (MODE >= kMuonFinish) {
          using One = typename ValueOf<MODE - kMuonFinish>::One;
          constexpr bool WIDE = MODE == kMuonFinish + ZC_F32;
          One* const param = static_cast<One*>(a.t[ti].param);
          void* const copy = a.t[ti].copy;
          const float step = a.t[ti].step * (1.0f / kMuonScale);
          if (turn) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              if (k < left) {
                const u64 place = (col + k) * r + row;
                v[k] = __builtin_fmaf(-step, v[k], float(param[place]) * a.keep);
                param[place] = One(v[k]);
                if (copy) store_value(copy, a.copy_type, place, v[k]);
              }
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float p[8];
              const u64 place = row * c + col + 8 * h;
              numbers_of<WIDE>(load_eight<WIDE>(param, place, left - 8 * h), MODE - kMuonFinish, p);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = __builtin_fmaf(-step, v[8 * h + k], p[k] * a.keep);
              store_eight<WIDE>(param, MODE - kMuonFinish, place, left - 8 * h, p);
              if (copy) store_numbers(copy, a.copy_type, place, left - 8 * h, p);
            }
          }
        } else {
          // As it is ...
          u8* const to = at + (MODE == kMuonGram ? parts.a + 2 * (row * parts.row_t + col) : MODE == kMuonPoly ? parts.b + 2 * (row * parts.row_t + col) : parts.x + 2 * (row * parts.row_x + col));
          const u64 plane = MODE == kMuonUpdate ? parts.plane_x : parts.plane_a;
          f16x8_t high[2], low[2];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            _Float16 one, two;
            halves_of(v[k], a.planes, one, two);
            high[k / 8][k % 8] = one, low[k / 8][k % 8] = two;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            *reinterpret_cast<f16x8_t*>(to + 16 * h) = high[h];
            if (a.planes > 1) *reinterpret_cast<f16x8_t*>(to + plane + 16 * h) = low[h];
          }
          // ... and turned: into the other half of a symmetric matrix (of a tile on the diagonal that is there already), or into the X turned that the next product reads.
          if (MODE == kMuonUpdate || down != across) {
            u8* const other = at + (MODE == kMuonGram ? parts.a : MODE == kMuonPoly ? parts.b : a.which ? parts.t0 : parts.t1);
            const u64 plane_2 = MODE == kMuonUpdate ? parts.plane_t : parts.plane_a;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              if (k < left) {
                u8* const place = other + 2 * ((col + k) * parts.row_t + row);
                *reinterpret_cast<_Float16*>(place) = high[k / 8][k % 8];
                if (a.planes > 1) *reinterpret_cast<_Float16*>(place + plane_2) = low[k / 8][k % 8];
              }
            }
          }
        }
        }
    };
    [&]<int... N>(std::integer_sequence<int, N...>) { (write(std::integral_constant<int, N>()), ...); }(std::make_integer_sequence<int, T * T>());
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the last requests, too, before the workgroup's LDS is given to another one)
}

}  // namespace zc
