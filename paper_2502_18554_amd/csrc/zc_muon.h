// The optimiser's step for matrices: momentum, made nearly orthogonal by Newton-Schulz products, into the weights.
//
//   g = grad x scale;  m' = mu m + (1 - mu) g;  u = mu m' + (1 - mu) g, or m' itself
//   X = u / max(|u|, 1e-7) with the root of the sum of squares for |u|, turned where it has more rows than columns: r x c, r <= c
//   several times:  A = X X^T;  B = a I + b A + c A A;  X = B X        (a, b, c) = (3.4445, -4.7750, 2.0315)
//   p' = p (1 - lr decay) - lr factor X
// The polynomial a s + b s^3 + c s^5 takes the singular values s from (0, 1] towards 1: from 0.002 on they are between 0.68 and 1.21 after five times, and never above 1.21
// (Jordan et al., "Muon", 2024, from where the coefficients are).
//
// The products are the matrix instructions' in binary16, with sums in binary32.  X, A and B are kept times 2^12: their entries are at most 1.21, 1.5 and 3.5, so that
// nothing overflows, and typical ones (1 / sqrt(r c) at first, 2^-12 for 4096 x 4096) are far from the smallest normal one.  An operand of one binary16 number has 11 bits: each
// product's result is rounded by at most 2^-11 of itself, an eighth of bfloat16's.  Where that is too much (weights in 32 bits), an operand is two binary16 numbers, 22 bits, and a product
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
  float step;                    // lr factor
  u32 turned;
};
struct MuonArgs {
  MuonTensor t[kMuonTensors];
  u32 first[kMuonTensors];       // of its tiles (or workgroups) in the launch, in ascending order
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

// The matrix that a tile or workgroup belongs to: a lane looks at one of them each, since a search one by one would wait for memory at each (24 matrices of 256 x 512: 4 us a launch).
static_assert(kMuonTensors == 64);
__device__ inline u32 muon_tensor_of(const MuonArgs& a, u32 tile) {
  const u32 lane = threadIdx.x & 63u;
  return u32(__popcll(__ballot(lane < a.tensors && a.first[lane] <= tile))) - 1;
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
  const u32 i = muon_tensor_of(a, blockIdx.x), part = blockIdx.x - a.first[i];
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
  const bool turn = a.t[i].turned;
  const u64 rows = turn ? c : r, cols = turn ? r : c;
  const MuonParts parts(r, c, a.planes);
  const u32 across = u32(muon_along(cols) / 64), t = blockIdx.x - a.first[i];
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

// Zeros behind the rows of A, B and the other X turned: the products write values only.  A thread has eight of the last 128 values of a row, as far as they are behind its end.
__global__ __launch_bounds__(256) void muon_zeros_kernel(MuonArgs a) {
  const u32 i = muon_tensor_of(a, blockIdx.x), r = a.t[i].r, c = a.t[i].c;
  const MuonParts parts(r, c, a.planes);
  const u64 row = u64(blockIdx.x - a.first[i]) * 16 + threadIdx.x / 16, col = parts.row_t - kMuonAlong + 8 * (threadIdx.x % 16);
  if (col + 8 <= r || row >= c) return;
  const u32 skip = col < r ? r - u32(col) : 0;
  const auto clear = [&](u64 from, u64 plane) {
    for (u32 k = 0; k < a.planes; ++k) {
      _Float16* const to = reinterpret_cast<_Float16*>(a.t[i].at + from + k * plane) + row * parts.row_t + col;
      if (skip == 0) *reinterpret_cast<f16x8_t*>(to) = f16x8_t{};
      else for (u32 j = skip; j < 8; ++j) to[j] = _Float16(0.0f);
    }
  };
  clear(parts.t1, parts.plane_t);
  if (row >= r) return;
  clear(parts.a, parts.plane_a);
  clear(parts.b, parts.plane_a);
}

// ---- The products.  Workgroups of 2 x 2 waves make tiles of 64 T x 64 T results, a wave 32 T x 32 T.
//
// A stage is KB values of every row of the tile, brought straight to LDS; S stages lie there, of which one is multiplied while the others are on their way.  Rows follow each
// other in LDS, their 16-byte blocks exchanged by the row's number, so that 16 lanes that read LDS together find 64 different banks.  An instruction multiplies eight values of 32 rows with as
// many of 32 columns from lanes 0 .. 31, eight others from lanes 32 .. 63.  Which column of the tile a lane brings is free: it is chosen so that a lane ends with 16
// neighbouring results of a row.  The requests run ahead into the workgroup's next tile too.
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

// Between two registers: 16 lanes 1 and 3 (of 0 .. 3) of the first with 16 lanes 0 and 2 of the second.
__device__ inline void swap_sixteens(u32& a, u32& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0], b = r[1];
}
// A lane has 16 neighbouring values of row l % 32 of 32 x 32, from column 16 (l / 32) on, in eight words of two.  In memory they are read and written so that four lanes have 64 bytes of a
// row: 16 bytes, number l / 16, of rows l % 16 and 16 + l % 16.
__device__ inline void sixteen_to_memory(u32 (&w)[8]) {
#pragma unroll
  for (int d = 0; d < 4; ++d) swap_sixteens(w[d], w[4 + d]);
}
struct MuonPlace {                                   // of a lane's two pieces
  u64 at[2];
  bool there[2];
};
__device__ inline void read_sixteen(const u8* from, const MuonPlace& place, u32 (&w)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const u32x4_t p = place.there[q] ? *reinterpret_cast<const u32x4_t*>(from + place.at[q]) : u32x4_t{};
#pragma unroll
    for (int d = 0; d < 4; ++d) w[4 * q + d] = p[d];
  }
}
__device__ inline float half_of(const u32 (&w)[8], int k) { return float(__builtin_bit_cast(_Float16, u16(w[k / 2] >> (16 * (k & 1))))); }
__device__ inline void write_sixteen(u8* to, const MuonPlace& place, u32 (&w)[8]) {
  sixteen_to_memory(w);
#pragma unroll
  for (int q = 0; q < 2; ++q)
    if (place.there[q]) *reinterpret_cast<u32x4_t*>(to + place.at[q]) = u32x4_t{w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]};
}
// The same values turned: four lanes exchange theirs so that each has four neighbouring rows of one column, 8 bytes, for four times four columns.
// `at`: of row 4 (l % 32 / 4), column 16 (l / 32) + l % 4, in the turned matrix; rows: how many from there; left: how many of the columns there are from the first on.
__device__ inline void write_turned(u8* at, u64 along, i32 rows, i32 left, u32 lane, const u32 (&w)[8]) {
  const bool upper = lane & 2u, odd = lane & 1u;
  const u32 give = odd ? 0x01000504u : 0x03020706u, first = odd ? 0x07060100u : 0x01000504u, second = odd ? 0x07060302u : 0x03020504u;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const u32 other = dpp_mov<kDppQuadSwap2>(upper ? w[2 * m] : w[2 * m + 1]);
    const u32 p = upper ? other : w[2 * m], r = upper ? w[2 * m + 1] : other;         // rows (lane & 1) and that + 2, two columns
    const u32 got = dpp_mov<kDppQuadSwap1>(__builtin_amdgcn_perm(p, r, give));
    const u32 one = __builtin_amdgcn_perm(p, got, first), two = __builtin_amdgcn_perm(r, got, second);
    if (4 * m + i32(lane & 3u) < left && rows > 0) {
      u8* const to = at + 2 * along * (4 * m);
      if (rows >= 4) {
        *reinterpret_cast<u32x2_t*>(to) = u32x2_t{one, two};
      } else {
        *reinterpret_cast<u16*>(to) = u16(one);
        if (rows > 1) *reinterpret_cast<u16*>(to + 2) = u16(one >> 16);
        if (rows > 2) *reinterpret_cast<u16*>(to + 4) = u16(two);
      }
    }
  }
}

// Waits for all but the last N requests (they come back in the order in which they were made), for LDS, and for the workgroup's other waves.
template <int N>
__device__ __forceinline__ void muon_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Waves that a SIMD holds of a kernel with tiles of 64 T and S stages of KB values in LDS: a workgroup has one on each.
constexpr u32 muon_lds_bytes(int T, int KB, int S) { return u32(S) * 2 * 64 * T * KB * 2; }
constexpr int muon_groups(int T, int KB, int S) { return T >= 3 ? 1 : int(163840u / muon_lds_bytes(T, KB, S)) < (T == 2 ? 2 : 4) ? int(163840u / muon_lds_bytes(T, KB, S)) : T == 2 ? 2 : 4; }

template <int T, int KB, int S, int MODE>
__global__ __launch_bounds__(256, T >= 3 ? 1 : muon_groups(T, KB, S) < 2 ? 2 : muon_groups(T, KB, S)) void muon_product_kernel(MuonArgs a) {
  constexpr u32 R = 64u * T, BLOCKS = KB / 8, ROW = 2 * KB, PLANE = R * ROW, STAGE = 2 * PLANE;      // bytes of a row, of an operand's rows, of a stage
  constexpr u32 APART = 4096 / ROW, LOADS = STAGE / 4096, STEPS = KB / 16;                           // rows between a thread's loads
  static_assert(KB == 64 || KB == 32);
  __shared__ u32x4_t memory[S * STAGE / 16];
  const u32 tid = threadIdx.x, lane = tid & 63u, wave = uniform(tid >> 6), half = lane >> 5, in32 = lane & 31u;
  const MuonTiles<MODE> tiles(a.count);
  if (tiles.first >= tiles.end) return;

  // What is asked for next: a tile's rows, and how far along them.
  u32 ask_tile = tiles.first, ask_stage = 0, ask_stages = 0, ask_segment = 0;
  u32 ask_stride = 0;
  MuonRows rows_a, rows_b;
  const u32 my_row = tid / BLOCKS;
  // Which block of a row is where: the place's number exchanged by what tells the rows apart that are read together.
  const auto key_a = [](u32 row) { return KB == 64 ? row >> 1 & 7u : row >> 2 & 3u; };
  const auto key_b = [](u32 row) { return KB == 64 ? (row >> 1 & 1u) | (row >> 3 & 2u) | (row & 4u) : (row >> 2 & 1u) | (row >> 3 & 2u); };
  const u32 block_a = 16u * ((tid ^ key_a(my_row)) & (BLOCKS - 1)), block_b = 16u * ((tid ^ key_b(my_row)) & (BLOCKS - 1));
  const auto aim = [&] {
    const u32 i = muon_tensor_of(a, ask_tile), r = a.t[i].r, c = a.t[i].c;
    const MuonParts parts(r, c, a.planes);
    u32 row, col;
    const u32 down = (r + R - 1) / R, across = MODE == kMuonGram || MODE == kMuonPoly ? down : (c + R - 1) / R;
    MuonTiles<MODE>::place(ask_tile - a.first[i], down, across, row, col);
    const u8* const at = a.t[i].at;
    const u64 plane_a = MODE == kMuonGram ? parts.plane_x : parts.plane_a, plane_b = MODE == kMuonGram ? parts.plane_x : MODE == kMuonPoly ? parts.plane_a : parts.plane_t;
    const u8* const from_a = at + (MODE == kMuonGram ? parts.x : MODE == kMuonPoly ? parts.a : parts.b) + (ask_segment == 2 ? plane_a : 0);
    const u8* const from_b = at + (MODE == kMuonGram ? parts.x : MODE == kMuonPoly ? parts.a : a.which ? parts.t1 : parts.t0) + (ask_segment == 1 ? plane_b : 0);
    const u64 along = MODE == kMuonGram ? parts.row_x : parts.row_t;
    rows_a.aim(from_a, u64(row) * R, r, 2 * along, R);
    rows_b.aim(from_b, u64(col) * R, MODE == kMuonGram || MODE == kMuonPoly ? r : c, 2 * along, R);
    ask_stride = uniform(u32(2 * along));
    ask_stages = uniform(u32(along / KB));
  };
  // (Behind the last tile there is nothing to ask for.)
  const auto next_stage = [&] {
    rows_a.move_on(ROW);
    rows_b.move_on(ROW);
    if (++ask_stage < ask_stages) return;
    ask_stage = 0;
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
  const auto ask = [&](u32 place, u32 i) {           // place: of the stage in LDS, in bytes
    const u32 to = lds0 + wave * 1024u + place + 4096u * i;
    if (i < LOADS / 2) muon_load_to_lds(rows_a.buffer(), to, (my_row + APART * i) * ask_stride + block_a);
    else muon_load_to_lds(rows_b.buffer(), to, (my_row + APART * (i - LOADS / 2)) * ask_stride + block_b);
  };

  const u32 wave_a = (wave >> 1) * 32u * T, wave_b = (wave & 1u) * 32u * T;
  const u32 lane_b = (in32 & 3u) + 16u * ((in32 >> 2) & 1u) + 4u * (in32 >> 3);
  // The blocks of this step and of the next one; in tiles of 64, where a step is one instruction, less than LDS takes to answer, those of this stage and of the next one.
  constexpr u32 AHEAD = T == 1 ? STEPS : 1;
  u32x4_t fa[2 * AHEAD][T], fb[2 * AHEAD][T];
  u32 at_a[STEPS], at_b[STEPS];                      // where a lane's block of step t is, in the first stage's place
#pragma unroll
  for (u32 t = 0; t < STEPS; ++t) {
    at_a[t] = lds0 + (wave_a + in32) * ROW + 16u * ((STEPS * half + t) ^ key_a(in32));
    at_b[t] = lds0 + PLANE + (wave_b + lane_b) * ROW + 16u * ((STEPS * half + t) ^ key_b(lane_b));
  }
  typedef const __attribute__((address_space(3))) u32x4_t LdsBlock;
  const auto read = [&](u32 to, u32 place, u32 t, u32 i) {
    if (i < T) fa[to][i] = *reinterpret_cast<LdsBlock*>(at_a[t] + place + 32 * ROW * i);
    else fb[to][i - T] = *reinterpret_cast<LdsBlock*>(at_b[t] + place + 32 * ROW * (i - T));
  };

  // The instructions of a step and what goes between them: in the first half the reads for the next step; in the last step of a stage, once everybody has read that stage,
  // half of the requests for the stage that takes its place, and the other half in the step behind it.
  constexpr u32 SLOTS = T * T, READS = 2 * T, EARLY = LOADS / 2;
  aim();
  const auto behind = [](u32 place) { return place + STAGE == S * STAGE ? 0u : place + STAGE; };
  u32 now = 0, free = 0;                             // the stage that is multiplied; the one that is asked for
#pragma unroll
  for (int s = 0; s + 1 < S; ++s) {
#pragma unroll
    for (u32 i = 0; i < LOADS; ++i) ask(free, i);
    next_stage();
    free = behind(free);
  }
  muon_wait<(S - 2) * int(LOADS)>();
#pragma unroll
  for (u32 i = 0; i < EARLY; ++i) ask(free, i);
#pragma unroll
  for (u32 t = 0; t < AHEAD; ++t)
#pragma unroll
    for (u32 i = 0; i < READS; ++i) read(t, 0, t, i);
  for (u32 tile = tiles.first; tile < tiles.end; tile += tiles.step) {
    const u32 ti = muon_tensor_of(a, tile), r = a.t[ti].r, c = a.t[ti].c;
    const MuonParts parts(r, c, a.planes);
    const u32 stages = uniform(u32((MODE == kMuonGram ? parts.row_x : parts.row_t) / KB) * (a.planes > 1 ? 3u : 1u));
    f32x16_t sum[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[i][j][k] = 0.0f;
    if constexpr (T == 1) {
      for (u32 pair = 0; pair < stages; pair += 2) {
#pragma unroll
        for (u32 u = 0; u < 2; ++u) {                  // (of an even number of stages)
          const u32 next = behind(now);
#pragma unroll
          for (u32 i = 0; i < EARLY; ++i) ask(free, EARLY + i);
          next_stage();
          muon_wait<(S - 2) * int(LOADS)>();
#pragma unroll
          for (u32 t = 0; t < STEPS; ++t)
#pragma unroll
            for (u32 i = 0; i < READS; ++i) read((u ^ 1) * STEPS + t, next, t, i);
#pragma unroll
          for (u32 i = 0; i < EARLY; ++i) ask(now, i);
#pragma unroll
          for (u32 t = 0; t < STEPS; ++t)
            sum[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, fb[u * STEPS + t][0]), __builtin_bit_cast(f16x8_t, fa[u * STEPS + t][0]), sum[0][0], 0, 0, 0);
          free = now;
          now = next;
        }
      }
    } else {
      for (u32 stage = 0; stage < stages; ++stage) {
        const u32 next = behind(now);
#pragma unroll
        for (u32 t = 0; t < STEPS; ++t) {
          if (t == STEPS - 1) muon_wait<(S - 2) * int(LOADS)>();
#pragma unroll
          for (u32 slot = 0; slot < SLOTS; ++slot) {
#pragma unroll
            for (u32 i = 0; i < EARLY; ++i) {
              if (i * SLOTS / EARLY != slot) continue;
              if (t == STEPS - 1) ask(now, i);
              if (t == 0) ask(free, EARLY + i);
            }
#pragma unroll
            for (u32 i = 0; i < READS; ++i)
              if (i * SLOTS / (2 * READS) == slot) read((t + 1) & 1, t + 1 < STEPS ? now : next, (t + 1) % STEPS, i);
            const u32 i = slot / T, j = slot % T;
            sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, fb[t & 1][j]), __builtin_bit_cast(f16x8_t, fa[t & 1][i]), sum[i][j], 0, 0, 0);
            muon_hold<T * T>(sum[i][j]);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (t == 0) next_stage();
        }
        free = now;
        now = next;
      }
    }
    // The results.
    u32 down, across;
    const u32 tiles_down = (r + R - 1) / R, tiles_across = MODE == kMuonGram || MODE == kMuonPoly ? tiles_down : (c + R - 1) / R;
    MuonTiles<MODE>::place(tile - a.first[ti], tiles_down, tiles_across, down, across);
    const u64 row0 = u64(down) * R + wave_a, col0 = u64(across) * R + wave_b;      // the wave's
    u8* const at = a.t[ti].at;
    if (MODE >= kMuonFinish && a.grad_scale && !(fabsf(*a.grad_scale) < __builtin_inff())) continue;
    // Where a lane's results of 32 x 32 are.
    constexpr bool OF_X = MODE != kMuonGram && MODE != kMuonPoly;
    const u64 along = OF_X ? parts.row_x : parts.row_t;
    const auto row_of = [&](int i) { return row0 + 32 * i + in32; };
    const auto col_of = [&](int j) { return col0 + 32 * j + 16 * half; };
    const auto place_of = [&](int i, int j) {
      MuonPlace place;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u64 of_row = row0 + 32 * i + 16 * q + (lane & 15u), of_col = col0 + 32 * j + 8 * (lane >> 4);
        place.at[q] = 2 * (of_row * along + of_col);
        place.there[q] = of_row < r && of_col < along;
      }
      return place;
    };
    // Rows of 32 x 32 one after the other: what is there already is asked for first, for the whole row.
    const auto row_of_blocks = [&](auto number) __attribute__((always_inline)) {
      constexpr int i = decltype(number)::value;
#pragma unroll
      for (int j = 0; j < T; ++j) muon_hold<T * T>(sum[i][j]);
      if constexpr (MODE >= kMuonFinish) {
        using One = typename ValueOf<MODE - kMuonFinish>::One;
        constexpr bool WIDE = MODE == kMuonFinish + ZC_F32;
        One* const param = static_cast<One*>(a.t[ti].param);
        void* const copy = a.t[ti].copy;
        const float step = -a.t[ti].step * (1.0f / (kMuonScale * kMuonScale));
        const u64 row = row_of(i);
        if (a.t[ti].turned) {
          One old[T][16];
#pragma unroll
          for (int j = 0; j < T; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) old[j][k] = row < r && col_of(j) + k < c ? param[(col_of(j) + k) * r + row] : One(0.0f);
#pragma unroll
          for (int j = 0; j < T; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float p = __builtin_fmaf(step, sum[i][j][k], float(old[j][k]) * a.keep);
              const u64 place = (col_of(j) + k) * r + row;
              if (row < r && col_of(j) + k < c) {
                param[place] = One(p);
                if (copy) store_value(copy, a.copy_type, place, p);
              }
            }
        } else {
          RawEight<WIDE> old[T][2];
          i32 left[T];
#pragma unroll
          for (int j = 0; j < T; ++j) {
            left[j] = row < r && col_of(j) < c ? i32(min(c - col_of(j), u64(16))) : 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) old[j][h] = load_eight<WIDE>(param, row * c + col_of(j) + 8 * h, left[j] - 8 * h);
          }
#pragma unroll
          for (int j = 0; j < T; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float p[8];
              const u64 place = row * c + col_of(j) + 8 * h;
              numbers_of<WIDE>(old[j][h], MODE - kMuonFinish, p);
#pragma unroll
              for (int k = 0; k < 8; ++k) p[k] = __builtin_fmaf(step, sum[i][j][8 * h + k], p[k] * a.keep);
              store_eight<WIDE>(param, MODE - kMuonFinish, place, left[j] - 8 * h, p);
              if (copy) store_numbers(copy, a.copy_type, place, left[j] - 8 * h, p);
            }
        }
      } else {
        // As it is, and turned: into the other half of a symmetric matrix (of a tile on the diagonal that is there already), or into the X turned that the next product reads.
        // (Values behind the matrix's columns are zeros, there and in the workspace, whose rows go on to a multiple of 128.)
        u8* const to = at + (MODE == kMuonGram ? parts.a : MODE == kMuonPoly ? parts.b : parts.x);
        u8* const other = at + (MODE == kMuonGram ? parts.a : MODE == kMuonPoly ? parts.b : a.which ? parts.t0 : parts.t1);
        const u64 row4 = row0 + 32 * i + (in32 & ~3u);
        const i32 rows4 = row4 < r ? i32(min(r - row4, u64(4))) : 0;
        u32 old[MODE == kMuonPoly ? T : 1][2][8];
        if constexpr (MODE == kMuonPoly) {
#pragma unroll
          for (int j = 0; j < T; ++j) {
            read_sixteen(at + parts.a, place_of(i, j), old[j][0]);
            if (a.planes > 1) read_sixteen(at + parts.a + parts.plane_a, place_of(i, j), old[j][1]);
          }
        }
#pragma unroll
        for (int j = 0; j < T; ++j) {
          const u64 col4 = col_of(j) + (lane & 3u);
          const i32 left4 = col_of(j) < (OF_X ? c : r) ? i32(min((OF_X ? c : r) - col_of(j), u64(16))) : 0;
          const MuonPlace place = place_of(i, j);
          float v[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = sum[i][j][k] * (MODE == kMuonPoly ? kMuonC / kMuonScale : 1.0f / kMuonScale);
          if constexpr (MODE == kMuonPoly) {
            sixteen_to_memory(old[j][0]);              // (the same exchange takes them back)
            if (a.planes > 1) sixteen_to_memory(old[j][1]);
            const i32 diagonal = i32(min(i64(row_of(i)) - i64(col_of(j)) + 64, i64(127))) - 64;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float x = half_of(old[j][0], k);
              if (a.planes > 1) x += half_of(old[j][1], k);
              v[k] = __builtin_fmaf(x, kMuonB, v[k]);
              if (k == diagonal) v[k] += kMuonA * kMuonScale;
            }
          }
          const auto both = [&](u32 (&w)[8], u64 plane, u64 plane_turned) __attribute__((always_inline)) {
            if (MODE == kMuonUpdate || down != across) write_turned(other + plane_turned + 2 * (col4 * parts.row_t + row4), parts.row_t, rows4, left4, lane, w);
            write_sixteen(to + plane, place, w);
          };
          u32 w[8];
#pragma unroll
          for (int d = 0; d < 8; ++d) w[d] = word_of_two<_Float16>(v[2 * d], v[2 * d + 1]);
          if (a.planes > 1) {
            u32 low[8];
#pragma unroll
            for (int d = 0; d < 8; ++d) low[d] = word_of_two<_Float16>(v[2 * d] - half_of(w, 2 * d), v[2 * d + 1] - half_of(w, 2 * d + 1));
            both(low, MODE == kMuonUpdate ? parts.plane_x : parts.plane_a, MODE == kMuonUpdate ? parts.plane_t : parts.plane_a);
          }
          both(w, 0, 0);
        }
      }
    };
    [&]<int... N>(std::integer_sequence<int, N...>) { (row_of_blocks(std::integral_constant<int, N>()), ...); }(std::make_integer_sequence<int, T>());
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the last requests, too, before the workgroup's LDS is given to another one)
}

}  // namespace zc
