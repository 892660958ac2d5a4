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
//
// Bound by the matrix instructions where the matrices are large: 4096 x 8192 takes 146, 84 and 247 us for the three products (138 GFLOP of the symmetric half, 69, 275: 0.94, 0.82 and 1.11 PFLOP/s,
// where a library's product of 8192^3 reaches 1.4), at 1.7 to 2.1 GHz.  What is between: the results' way to memory after the last instruction, as they are and turned, some 25 us a product,
// and tiles that do not fill the last turn of CUs.  24 matrices of 256 x 512 take 7, 6.5 and 11 us: a launch and the latencies of one tile
// (waves wait for 65, 65 and 46 % of their time, matrix instructions are busy for 3, 1 and 4 %).
#pragma once

#include <utility>

#include "zc_muon_ask.h"
#include "zc_rows.h"
#include "zc_to_lds.h"

namespace zc {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) u32 LdsWord;

constexpr int kMuonTensors = 64;                     // of one launch: their table travels in the kernel's arguments
constexpr float kMuonA = 3.4445f, kMuonB = -4.7750f, kMuonC = 2.0315f;
constexpr float kMuonScale = 4096.0f;

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
  // What the waves need first (they have it in registers when they start).  Where all matrices have one shape, what a tile needs to begin is here, and not behind two answers of memory.
  u32 count;                     // tiles (or workgroups) of the launch
  u32 each;                      // of a matrix, where all have one shape; 0 otherwise
  u32 r, c;                      // that shape
  u8* at;                        // the first matrix's share of the workspace, `bytes` before the next one's
  u64 bytes;
  u32 tensors;
  u32 planes;                    // 1 or 2
  u32 which;                     // of the two turned X
  const float* grad_scale;
  double* partial;               // [tensor][kMuonPartials]
  float keep, mu, rest;          // 1 - lr decay; mu, 1 - mu
  u32 nesterov;
  int param_type, grad_type, copy_type;
  u32 first[kMuonTensors];       // of its tiles (or workgroups) in the launch, in ascending order
  MuonTensor t[kMuonTensors];
};
static_assert(sizeof(MuonArgs) <= 4096);
// (The kernels read them where they lie: of a parameter that is used in many places, with an index, the compiler makes a copy in scratch memory.)

// The matrix that a tile or workgroup belongs to: a lane looks at one of them each, since a search one by one would wait for memory at each (24 matrices of 256 x 512: 4 us a launch).
static_assert(kMuonTensors == 64);
struct MuonOf {
  u32 i, r, c, first;            // the matrix, its shape and its first tile
  u8* at;
  __device__ MuonOf(const MuonArgs& a, u32 tile) {
    if (a.each) {
      i = tile / a.each;
      first = i * a.each;
      r = a.r, c = a.c;
      at = a.at + i * a.bytes;
    } else {
      const u32 lane = threadIdx.x & 63u;
      i = u32(__popcll(__ballot(lane < a.tensors && a.first[lane] <= tile))) - 1;
      first = a.first[i];
      r = a.t[i].r, c = a.t[i].c;
      at = a.t[i].at;
    }
  }
};

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

__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonArgs) {
  const MuonArgs& a = kernel_args<MuonArgs, 0>();
  __shared__ double slot[4];
  const float scale = a.grad_scale ? *a.grad_scale : 1.0f;
  if (!(fabsf(scale) < __builtin_inff())) return;
  const MuonOf of(a, blockIdx.x);
  const u32 i = of.i, part = blockIdx.x - of.first;
  const u64 values = u64(of.r) * of.c;
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
__global__ __launch_bounds__(256) void muon_begin_kernel(MuonArgs) {
  const MuonArgs& a = kernel_args<MuonArgs, 0>();
  __shared__ double slot[4];
  __shared__ float tile[64][65];
  const float scale = a.grad_scale ? *a.grad_scale : 1.0f;
  const MuonOf of(a, blockIdx.x);
  const u32 i = of.i, r = of.r, c = of.c;
  const bool turn = a.t[i].turned;
  const u64 rows = turn ? c : r, cols = turn ? r : c;
  const MuonParts parts(r, c, a.planes);
  const u32 across = u32(muon_along(cols) / 64), t = blockIdx.x - of.first;
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
      u8* const place = of.at + to + 2 * (row * along + col);
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
      u8* const place = of.at + to_2 + 2 * (col * along_2 + row);
      *reinterpret_cast<f16x8_t*>(place) = high;
      if (a.planes > 1) *reinterpret_cast<f16x8_t*>(place + plane_2) = low;
    }
  }
}

// Zeros behind the rows of A, B and the other X turned: the products write values only.  A thread has eight of the last 128 values of a row, as far as they are behind its end.
__global__ __launch_bounds__(256) void muon_zeros_kernel(MuonArgs) {
  const MuonArgs& a = kernel_args<MuonArgs, 0>();
  const MuonOf of(a, blockIdx.x);
  const u32 r = of.r, c = of.c;
  const MuonParts parts(r, c, a.planes);
  const u64 row = u64(blockIdx.x - of.first) * 16 + threadIdx.x / 16, col = parts.row_t - kMuonAlong + 8 * (threadIdx.x % 16);
  if (col + 8 <= r || row >= c) return;
  const u32 skip = col < r ? r - u32(col) : 0;
  const auto clear = [&](u64 from, u64 plane) {
    for (u32 k = 0; k < a.planes; ++k) {
      _Float16* const to = reinterpret_cast<_Float16*>(of.at + from + k * plane) + row * parts.row_t + col;
      if (skip == 0) *reinterpret_cast<f16x8_t*>(to) = f16x8_t{};
      else for (u32 j = skip; j < 8; ++j) to[j] = _Float16(0.0f);
    }
  };
  clear(parts.t1, parts.plane_t);
  if (row >= r) return;
  clear(parts.a, parts.plane_a);
  clear(parts.b, parts.plane_a);
}

// ---- The products.  Workgroups of 2 x 2 waves make tiles of 64 TM x 64 TN results, a wave 32 TM x 32 TN.
//
// A stage is 64 values (128 bytes) of every row of the tile, brought straight to LDS; S stages lie there, of which one is multiplied while the others are on their way.  Rows follow each
// other in LDS, their 16-byte blocks exchanged by the row's number, so that 16 lanes that read LDS together find 64 different banks.  An instruction multiplies eight values of 32 rows with as
// many of 32 columns from lanes 0 .. 31, eight others from lanes 32 .. 63.  Which column of the tile a lane brings is free: it is chosen so that a lane ends with 16
// neighbouring results of a row.  The requests run ahead into the workgroup's next tile too.

// Rows of a tile as a buffer: rows behind the last one read as zeros.
struct MuonRows : MuonSpan {
  __device__ __amdgpu_buffer_rsrc_t buffer() const {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u64(uniform(u32(at))) | u64(uniform(u32(at >> 32))) << 32), 0, int(uniform(bytes)), 0x00027000);
  }
};

// Keeps an instruction's sums at their place, in the matrix instructions' own registers where a wave is alone on its SIMD (the compiler has them there then).
template <bool OWN>
__device__ __forceinline__ void muon_hold(f32x16_t& sum) {
  if constexpr (OWN) asm volatile("" : "+a"(sum));
  else asm volatile("" : "+v"(sum));
}

// The workgroup's tiles.
template <int MODE>
struct MuonTiles : MuonShare {
  __device__ explicit MuonTiles(u32 tiles) : MuonShare(tiles, blockIdx.x, gridDim.x) {}
  __device__ static void place(u32 t, u32 down, u32 across, u32& row, u32& col) {
    const MuonPlace p = muon_place<muon_symmetric(MODE)>(t, down, across, muon_symmetric(MODE) ? u32(sqrtf(float(t) * (1.0f / 32.0f))) : 0u);
    row = uniform(p.row);
    col = uniform(p.col);
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
__device__ inline float half_of(const u32 (&w)[8], int k) { return float(__builtin_bit_cast(_Float16, u16(w[k / 2] >> (16 * (k & 1))))); }

// The same values turned: four lanes exchange theirs so that each has four neighbouring rows of one column, two words, for four times four columns.
struct MuonTurn {
  u32 give, first, second;                           // which bytes
  bool upper;
  __device__ explicit MuonTurn(u32 lane) {
    const bool odd = lane & 1u;
    upper = lane & 2u;
    give = odd ? 0x01000504u : 0x03020706u, first = odd ? 0x07060100u : 0x01000504u, second = odd ? 0x07060302u : 0x03020504u;
  }
  __device__ u32x2_t operator()(u32 low, u32 high) const {
    const u32 other = dpp_mov<kDppQuadSwap2>(upper ? low : high);
    const u32 p = upper ? other : low, r = upper ? high : other;              // rows (lane & 1) and that + 2, two columns
    const u32 got = dpp_mov<kDppQuadSwap1>(__builtin_amdgcn_perm(p, r, give));
    return u32x2_t{__builtin_amdgcn_perm(p, got, first), __builtin_amdgcn_perm(r, got, second)};
  }
};

// Workgroups that a CU holds of a kernel with tiles of 64 TM x 64 TN and S stages in LDS: a workgroup has a wave on each SIMD.
constexpr int muon_groups(int TM, int TN, int S) {
  const int by_lds = 20 / ((TM + TN) * S);           // (160 KiB, of which a stage takes 8 KiB (TM + TN))
  return TM * TN > 4 || by_lds < 2 ? 1 : by_lds < 4 ? 2 : 4;
}

// The results of a wave, 32 TM x 32 TN from (row0, col0) on.  mirrored: those of a symmetric matrix off its diagonal, which go to the other half as well.
template <int TM, int TN, int MODE, bool ALONE>
__device__ __forceinline__ void muon_results(const MuonArgs& a, const MuonOf& of, const MuonParts& parts, u64 row0, u64 col0, bool mirrored, f32x16_t (&sum)[TM][TN]) {
  u8* const at = of.at;
  const u32 r = of.r, c = of.c, lane = threadIdx.x & 63u, half = lane >> 5, in32 = lane & 31u;
  const u32 planes = a.planes, which = a.which;
  const int copy_type = a.copy_type;
  const float keep = a.keep;
  const bool turned = MODE >= kMuonFinish && a.t[of.i].turned;
  void *const params = MODE >= kMuonFinish ? a.t[of.i].param : nullptr, *const copy = MODE >= kMuonFinish ? a.t[of.i].copy : nullptr;
  const float step = MODE >= kMuonFinish ? -a.t[of.i].step * (1.0f / (kMuonScale * kMuonScale)) : 0.0f;
  if (MODE >= kMuonFinish && a.grad_scale && !(fabsf(*a.grad_scale) < __builtin_inff())) return;
  constexpr bool OF_X = MODE != kMuonGram && MODE != kMuonPoly;
  const u64 along = OF_X ? parts.row_x : parts.row_t, cols = OF_X ? c : r;
  // How many rows and columns there are from the wave's first on (what exceeds a tile does not matter), and values of a row with the zeros behind it.
  const i32 rows_left = i32(min(i64(r) - i64(row0), i64(1024))), cols_left = i32(min(i64(cols) - i64(col0), i64(1024))), along_left = i32(min(i64(along) - i64(col0), i64(1024)));
  // Rows of 32 x 32 one after the other: what is there already is asked for first, for the whole row.  WHOLE: the matrix has all of the wave's results.
  const auto row_of_blocks = [&](auto number, auto whole) __attribute__((always_inline)) {
    constexpr int i = decltype(number)::value;
    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
    for (int j = 0; j < TN; ++j) muon_hold<ALONE>(sum[i][j]);
    const bool row_there = WHOLE || 32 * i + i32(in32) < rows_left;
    if constexpr (MODE >= kMuonFinish) {
      using One = typename ValueOf<MODE - kMuonFinish>::One;
      constexpr bool WIDE = MODE == kMuonFinish + ZC_F32;
      One* const param = static_cast<One*>(params);
      // (Two blocks at a time: registers are short.)
      constexpr int TOGETHER = TN < 2 ? TN : 2;
#pragma unroll
      for (int j0 = 0; j0 < TN; j0 += TOGETHER) {
        if (turned) {
          const u64 first = (col0 + 16 * half) * r + row0 + 32 * i + in32;
          One old[TOGETHER][16];
#pragma unroll
          for (int d = 0; d < TOGETHER; ++d)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const int at_col = 32 * (j0 + d) + k;
              old[d][k] = j0 + d < TN && row_there && (WHOLE || at_col + 16 * i32(half) < cols_left) ? param[first + u64(at_col) * r] : One(0.0f);
            }
#pragma unroll
          for (int d = 0; d < TOGETHER; ++d)
            if (j0 + d < TN) {
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const int at_col = 32 * (j0 + d) + k;
                const float p = __builtin_fmaf(step, sum[i][j0 + d < TN ? j0 + d : 0][k], float(old[d][k]) * keep);
                if (row_there && (WHOLE || at_col + 16 * i32(half) < cols_left)) {
                  param[first + u64(at_col) * r] = One(p);
                  if (copy) store_value(copy, copy_type, first + u64(at_col) * r, p);
                }
              }
            }
        } else {
          const u64 first = (row0 + 32 * i + in32) * c + col0 + 16 * half;
          RawEight<WIDE> old[TOGETHER][2];
          const auto left_of_piece = [&](int j, int h) { return WHOLE ? 8 : row_there && j < TN ? cols_left - 32 * j - 16 * i32(half) - 8 * h : 0; };
#pragma unroll
          for (int d = 0; d < TOGETHER; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (j0 + d < TN) old[d][h] = load_eight<WIDE>(param, first + 32 * (j0 + d) + 8 * h, left_of_piece(j0 + d, h));
#pragma unroll
          for (int d = 0; d < TOGETHER; ++d)
            if (j0 + d < TN) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float p[8];
                numbers_of<WIDE>(old[d][h], MODE - kMuonFinish, p);
#pragma unroll
                for (int k = 0; k < 8; ++k) p[k] = __builtin_fmaf(step, sum[i][j0 + d < TN ? j0 + d : 0][8 * h + k], p[k] * keep);
                store_eight<WIDE>(param, MODE - kMuonFinish, first + 32 * (j0 + d) + 8 * h, left_of_piece(j0 + d, h), p);
                if (copy) store_numbers(copy, copy_type, first + 32 * (j0 + d) + 8 * h, left_of_piece(j0 + d, h), p);
              }
            }
        }
      }
    } else {
      // As it is, and turned: into the other half of a symmetric matrix (of a tile on the diagonal that is there already), or into the X turned that the next product reads.
      // (Values behind the matrix's rows and columns are zeros, there and in the workspace, whose rows go on to a multiple of 128.)
      const u64 to = uniform64((MODE == kMuonGram ? parts.a : MODE == kMuonPoly ? parts.b : parts.x) + 2 * ((row0 + 32 * i) * along + col0));
      const u64 turned_to = uniform64((MODE == kMuonGram ? parts.a : MODE == kMuonPoly ? parts.b : which ? parts.t0 : parts.t1) + 2 * (col0 * parts.row_t + row0 + 32 * i));
      const u32 mine = 2 * ((lane & 15u) * u32(along) + 8 * (lane >> 4)), mine_turned = 2 * ((16 * half + (lane & 3u)) * u32(parts.row_t) + (in32 & ~3u));
      const auto there = [&](int j, int q) { return WHOLE || (32 * i + 16 * q + i32(lane & 15u) < rows_left && 32 * j + 8 * i32(lane >> 4) < along_left); };
      const auto there_turned = [&](int j, int m) { return WHOLE || (32 * i + i32(in32 & ~3u) < rows_left && 32 * j + 16 * i32(half) + 4 * m + i32(lane & 3u) < cols_left); };
      const u64 plane_to = OF_X ? parts.plane_x : parts.plane_a, plane_turned = OF_X ? parts.plane_t : parts.plane_a;
      u32 old[MODE == kMuonPoly ? TN : 1][2][8];
      if constexpr (MODE == kMuonPoly) {
        const u8* const from = at + uniform64(parts.a + 2 * ((row0 + 32 * i) * along + col0));
#pragma unroll
        for (u32 plane = 0; plane < 2; ++plane)
          if (plane < planes) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const u32x4_t p = there(j, q) ? *reinterpret_cast<const u32x4_t*>(at_bytes(from + plane * parts.plane_a + 32 * q * along + 64 * j, mine)) : u32x4_t{};
#pragma unroll
                for (int d = 0; d < 4; ++d) old[j][plane][4 * q + d] = p[d];
              }
          }
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        float v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = sum[i][j][k] * (MODE == kMuonPoly ? kMuonC / kMuonScale : 1.0f / kMuonScale);
        if constexpr (MODE == kMuonPoly) {
#pragma unroll
          for (u32 plane = 0; plane < 2; ++plane)
            if (plane < planes) {
              sixteen_to_memory(old[j][plane]);      // (the same exchange takes them back)
#pragma unroll
              for (int k = 0; k < 16; ++k) v[k] = __builtin_fmaf(half_of(old[j][plane], k), kMuonB, v[k]);
            }
          if (row0 + 32 * i == col0 + 32 * j) {       // (on the diagonal)
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] += in32 == 16 * half + k ? kMuonA * kMuonScale : 0.0f;
          }
        }
        const auto write = [&](u32 (&w)[8], u64 plane, u64 plane_t) __attribute__((always_inline)) {
          if (MODE == kMuonUpdate || mirrored) {
            const MuonTurn turn(lane);
            u8* const base = at + turned_to + plane_t;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const u32x2_t four = turn(w[2 * m], w[2 * m + 1]);
              if (there_turned(j, m)) *reinterpret_cast<u32x2_t*>(at_bytes(base + 2 * (32 * j + 4 * m) * parts.row_t, mine_turned)) = four;
            }
          }
          sixteen_to_memory(w);
          u8* const base = at + to + plane;
#pragma unroll
          for (int q = 0; q < 2; ++q)
            if (there(j, q)) *reinterpret_cast<u32x4_t*>(at_bytes(base + 32 * q * along + 64 * j, mine)) = u32x4_t{w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]};
        };
        u32 w[8];
#pragma unroll
        for (int d = 0; d < 8; ++d) w[d] = word_of_two<_Float16>(v[2 * d], v[2 * d + 1]);
        if (planes > 1) {
          u32 low[8];
#pragma unroll
          for (int d = 0; d < 8; ++d) low[d] = word_of_two<_Float16>(v[2 * d] - half_of(w, 2 * d), v[2 * d + 1] - half_of(w, 2 * d + 1));
          write(low, plane_to, plane_turned);
        }
        write(w, 0, 0);
      }
    }
  };
  const auto all_rows = [&](auto whole) __attribute__((always_inline)) {
    [&]<int... N>(std::integer_sequence<int, N...>) { (row_of_blocks(std::integral_constant<int, N>(), whole), ...); }(std::make_integer_sequence<int, TM>());
  };
  if (rows_left >= 32 * TM && cols_left >= 32 * TN) all_rows(std::true_type());
  else all_rows(std::false_type());
}

// Waits for all but the last N requests (they come back in the order in which they were made), for LDS, and for the workgroup's other waves.
template <int N>
__device__ __forceinline__ void muon_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int TM, int TN, int S, int MODE>
__global__ __launch_bounds__(256, muon_groups(TM, TN, S)) void muon_product_kernel(MuonArgs) {
  const MuonArgs& a = kernel_args<MuonArgs, 0>();
  constexpr u32 KB = 64, RA = 64u * TM, RB = 64u * TN, BLOCKS = KB / 8, ROW = 2 * KB, AT_B = RA * ROW, STAGE = AT_B + RB * ROW;      // bytes of a row, of a stage
  constexpr u32 APART = 4096 / ROW, LOADS_A = AT_B / 4096, LOADS = STAGE / 4096, STEPS = KB / 16;    // rows between a thread's loads; its loads
  constexpr bool TRIANGLE = muon_symmetric(MODE), SMALL = TM * TN == 1;
  static_assert(!TRIANGLE || TM == TN);
  __shared__ u32x4_t memory[S * STAGE / 16];
  const u32 tid = threadIdx.x, lane = tid & 63u, wave = uniform(tid >> 6), half = lane >> 5, in32 = lane & 31u;
  const MuonTiles<MODE> tiles(a.count);
  if (tiles.first >= tiles.end) return;

  // What is asked for next: a tile's rows, and how far along them.
  MuonAsked asked{tiles.first, 0, 0};
  u32 ask_stages = 0;
  MuonRows rows_a, rows_b;
  const u32 my_row = tid / BLOCKS;
  // Which block of a row is where: the place's number exchanged by what tells the rows apart that are read together.
  const auto key_a = [](u32 row) { return row >> 1 & 7u; };
  const auto key_b = [](u32 row) { return (row >> 1 & 1u) | (row >> 3 & 2u) | (row & 4u); };
  u32 mine_a[LOADS_A], mine_b[LOADS - LOADS_A];          // a thread's places in the tile's rows
  const auto aim = [&] {
    const MuonOf of(a, asked.tile);
    const u32 r = of.r, c = of.c;
    const MuonParts parts(r, c, a.planes);
    u32 row, col;
    const u32 down = (r + RA - 1) / RA, across = TRIANGLE ? down : (c + RB - 1) / RB;
    MuonTiles<MODE>::place(asked.tile - of.first, down, across, row, col);
    const u64 at = reinterpret_cast<u64>(of.at);
    const u64 along = muon_along_of(parts, MODE);
    rows_a.aim(at + muon_operand_a(parts, MODE, asked.segment), u64(row) * RA, r, 2 * along, RA);
    rows_b.aim(at + muon_operand_b(parts, MODE, a.which, asked.segment), u64(col) * RB, TRIANGLE ? r : c, 2 * along, RB);
    const u32 apart = uniform(u32(2 * along));
#pragma unroll
    for (u32 k = 0; k < LOADS; ++k) {
      const u32 of = my_row + APART * (k < LOADS_A ? k : k - LOADS_A);
      if (k < LOADS_A) mine_a[k] = of * apart + 16u * ((tid ^ key_a(of)) & (BLOCKS - 1));
      else mine_b[k - LOADS_A] = of * apart + 16u * ((tid ^ key_b(of)) & (BLOCKS - 1));
    }
    ask_stages = uniform(u32(along / KB));
  };
  // (Behind the last tile there is nothing to ask for.)
  const auto next_stage = [&] {
    rows_a.move_on(ROW);
    rows_b.move_on(ROW);
    const MuonNext next = asked.next(ask_stages, a.planes, tiles.step, tiles.end);
    if (next == MuonNext::kAim) aim();
    else if (next == MuonNext::kNothing) rows_a.bytes = rows_b.bytes = 0;
  };
  const u32 lds0 = u32(reinterpret_cast<uintptr_t>((LdsWord*)&memory[0]));
  const auto ask = [&](u32 place, u32 i) {           // place: of the stage in LDS, in bytes
    const u32 to = lds0 + wave * 1024u + place + 4096u * i;
    if (i < LOADS_A) load_to_lds(rows_a.buffer(), to, mine_a[i]);
    else load_to_lds(rows_b.buffer(), to, mine_b[i - LOADS_A]);
  };

  const u32 wave_a = (wave >> 1) * 32u * TM, wave_b = (wave & 1u) * 32u * TN;
  const u32 lane_b = (in32 & 3u) + 16u * ((in32 >> 2) & 1u) + 4u * (in32 >> 3);
  // The blocks of this step and of the next two (one, where registers are short); in tiles of 64, where a step is one instruction, less than LDS takes to answer, those of this stage and of the next one.
  constexpr u32 AHEAD = SMALL ? STEPS : TM * TN > 9 || (TM * TN > 4 && MODE == kMuonPoly) ? 1 : 2, HELD = SMALL ? 2 * STEPS : STEPS;
  u32x4_t fa[HELD][TM], fb[HELD][TN];
  u32 at_a[STEPS], at_b[STEPS];                      // where a lane's block of step t is, in the first stage's place
#pragma unroll
  for (u32 t = 0; t < STEPS; ++t) {
    at_a[t] = lds0 + (wave_a + in32) * ROW + 16u * ((STEPS * half + t) ^ key_a(in32));
    at_b[t] = lds0 + AT_B + (wave_b + lane_b) * ROW + 16u * ((STEPS * half + t) ^ key_b(lane_b));
  }
  typedef const __attribute__((address_space(3))) u32x4_t LdsBlock;
  const auto read = [&](u32 to, u32 place, u32 t, u32 i) {
    if (i < TM) fa[to][i] = *reinterpret_cast<LdsBlock*>(at_a[t] + place + 32 * ROW * i);
    else fb[to][i - TM] = *reinterpret_cast<LdsBlock*>(at_b[t] + place + 32 * ROW * (i - TM));
  };

  // The instructions of a step and what goes between them: in the first half the reads for the steps to come; once everybody has read a stage, half of the requests for the one that takes
  // its place, and the other half in the step behind that.
  constexpr u32 SLOTS = TM * TN, READS = TM + TN, EARLY = LOADS / 2;
  aim();
  const auto behind = [](u32 place) { return place + STAGE == S * STAGE ? 0u : place + STAGE; };
  u32 now = 0, free = 0;                             // the stage that is multiplied; the one that is asked for
  constexpr int FIRST = SMALL || AHEAD == 1 ? S - 1 : S;    // stages that are asked for before the first one is multiplied
#pragma unroll
  for (int s = 0; s < FIRST; ++s) {
#pragma unroll
    for (u32 i = 0; i < LOADS; ++i) ask(free, i);
    next_stage();
    free = behind(free);
  }
  muon_wait<(FIRST - 1) * int(LOADS)>();
  if constexpr (SMALL || AHEAD == 1) {
#pragma unroll
    for (u32 i = 0; i < EARLY; ++i) ask(free, i);
  }
#pragma unroll
  for (u32 t = 0; t < AHEAD; ++t)
#pragma unroll
    for (u32 i = 0; i < READS; ++i) read(t, 0, t, i);
  for (u32 tile = tiles.first; tile < tiles.end; tile += tiles.step) {
    const MuonOf of(a, tile);
    const u32 r = of.r, c = of.c;
    const MuonParts parts(r, c, a.planes);
    const u32 stages = uniform(u32(muon_along_of(parts, MODE) / KB) * (a.planes > 1 ? 3u : 1u));
    f32x16_t sum[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[i][j][k] = 0.0f;
    if constexpr (SMALL) {
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
          if (t == STEPS - AHEAD) muon_wait<(S - 2) * int(LOADS)>();
#pragma unroll
          for (u32 slot = 0; slot < SLOTS; ++slot) {
#pragma unroll
            for (u32 i = 0; i < EARLY; ++i) {
              if (i * SLOTS / EARLY != slot) continue;
              if (t == STEPS - AHEAD) ask(now, i);
              if (AHEAD == 1 && t == 0) ask(free, EARLY + i);
              if (AHEAD > 1 && t == STEPS - AHEAD + 1) ask(now, EARLY + i);
            }
#pragma unroll
            for (u32 i = 0; i < READS; ++i)
              if (i * SLOTS / (2 * READS) == slot) read((t + AHEAD) % STEPS, t + AHEAD < STEPS ? now : next, (t + AHEAD) % STEPS, i);
            const u32 i = slot / TN, j = slot % TN;
            sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, fb[t][j]), __builtin_bit_cast(f16x8_t, fa[t][i]), sum[i][j], 0, 0, 0);
            muon_hold<muon_groups(TM, TN, S) == 1>(sum[i][j]);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (AHEAD == 1 && t == 0) next_stage();
        }
        if (AHEAD > 1) next_stage();
        free = now;
        now = next;
      }
    }
    // The results.
    u32 down, across;
    const u32 tiles_down = (r + RA - 1) / RA, tiles_across = TRIANGLE ? tiles_down : (c + RB - 1) / RB;
    MuonTiles<MODE>::place(tile - of.first, tiles_down, tiles_across, down, across);
    muon_results<TM, TN, MODE, muon_groups(TM, TN, S) == 1>(a, of, parts, u64(down) * RA + wave_a, u64(across) * RB + wave_b, down != across, sum);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the last requests, too, before the workgroup's LDS is given to another one)
}

// ---- Few and small results: workgroups make tiles of 32 x 32, and their four waves take every fourth stage of 64 values each, by themselves: a wave's requests go to a part of LDS of its own, and
// it waits for nobody.  At the end the first wave adds the four sums.  (Tiles of 64 of the sizes for which this is there are bound by what a workgroup waits for itself: three matrices of
// 333 x 1531 in two parts, 63 tiles on 256 CUs, 24 us for X X^T, 0.3 us a stage; here 10.4.)
template <int MODE>
__global__ __launch_bounds__(256, 2) void muon_small_kernel(MuonArgs) {
  const MuonArgs& a = kernel_args<MuonArgs, 0>();
  constexpr int S = 2;                               // stages of a wave in LDS
  constexpr u32 STAGE = 8192;                        // of a wave: 32 rows of each operand
  __shared__ u32x4_t memory[4 * S * STAGE / 16];
  const u32 lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), half = lane >> 5, in32 = lane & 31u;
  const MuonTiles<MODE> tiles(a.count);
  const MuonOf of(a, tiles.first);                   // (a workgroup has one tile)
  const u32 r = of.r, c = of.c;
  const MuonParts parts(r, c, a.planes);
  u32 down, across;
  constexpr bool TRIANGLE = muon_symmetric(MODE);
  const u32 tiles_down = (r + 31) / 32, tiles_across = TRIANGLE ? tiles_down : (c + 31) / 32;
  MuonTiles<MODE>::place(tiles.first - of.first, tiles_down, tiles_across, down, across);
  const u64 along = muon_along_of(parts, MODE), at = reinterpret_cast<u64>(of.at);
  const u32 per = u32(along / 64), stages = per * (a.planes > 1 ? 3u : 1u), apart = u32(2 * along);
  const auto key_a = [](u32 row) { return row >> 1 & 7u; };
  const auto key_b = [](u32 row) { return (row >> 1 & 1u) | (row >> 3 & 2u) | (row & 4u); };
  u32 mine_a[4], mine_b[4];
#pragma unroll
  for (u32 k = 0; k < 4; ++k) {
    const u32 row = (lane >> 3) + 8 * k;
    mine_a[k] = row * apart + 16u * ((lane ^ key_a(row)) & 7u);
    mine_b[k] = row * apart + 16u * ((lane ^ key_b(row)) & 7u);
  }
  const u32 lds0 = u32(reinterpret_cast<uintptr_t>((LdsWord*)&memory[0])) + wave * S * STAGE;
  MuonQuarter asked{0, wave, wave};
  const auto ask = [&](u32 place) {
    asked.settle(per);
    MuonRows rows_a, rows_b;
    rows_a.aim(at + muon_operand_a(parts, MODE, asked.segment), u64(down) * 32, r, apart, 32);
    rows_b.aim(at + muon_operand_b(parts, MODE, a.which, asked.segment), u64(across) * 32, TRIANGLE ? r : c, apart, 32);
    rows_a.move_on(128 * asked.at);
    rows_b.move_on(128 * asked.at);
    if (asked.all >= stages) rows_a.bytes = rows_b.bytes = 0;      // (behind the last stage there is nothing to ask for)
#pragma unroll
    for (u32 k = 0; k < 4; ++k) load_to_lds(rows_a.buffer(), lds0 + place + 1024u * k, mine_a[k]);
#pragma unroll
    for (u32 k = 0; k < 4; ++k) load_to_lds(rows_b.buffer(), lds0 + place + 4096u + 1024u * k, mine_b[k]);
    asked.next();
  };
  const u32 lane_b = (in32 & 3u) + 16u * ((in32 >> 2) & 1u) + 4u * (in32 >> 3);
  typedef const __attribute__((address_space(3))) u32x4_t LdsBlock;
  f32x16_t sum[1][1] = {}, other = {};
  u32 now = 0, free = 0;
  const auto behind = [](u32 place) { return place + STAGE == S * STAGE ? 0u : place + STAGE; };
#pragma unroll
  for (int s = 0; s + 1 < S; ++s) ask(free), free = behind(free);
  for (u32 stage = wave; stage < stages; stage += 4) {
    ask(free);
    free = behind(free);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * 8) : "memory");
    f16x8_t x[4], y[4];
#pragma unroll
    for (u32 t = 0; t < 4; ++t) {
      x[t] = __builtin_bit_cast(f16x8_t, *reinterpret_cast<LdsBlock*>(lds0 + now + in32 * 128u + 16u * ((4 * half + t) ^ key_a(in32))));
      y[t] = __builtin_bit_cast(f16x8_t, *reinterpret_cast<LdsBlock*>(lds0 + now + 4096u + lane_b * 128u + 16u * ((4 * half + t) ^ key_b(lane_b))));
    }
    now = behind(now);
#pragma unroll
    for (u32 t = 0; t < 4; t += 2) {
      sum[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(y[t], x[t], sum[0][0], 0, 0, 0);
      other = __builtin_amdgcn_mfma_f32_32x32x16_f16(y[t + 1], x[t + 1], other, 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (what has been read may be overwritten)
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(&memory[0]);   // [wave][value][lane]
  if (wave) {
#pragma unroll
    for (int k = 0; k < 16; ++k) sums[(wave * 16 + k) * 64 + lane] = sum[0][0][k] + other[k];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int k = 0; k < 16; ++k) sum[0][0][k] = ((sum[0][0][k] + other[k]) + sums[(16 + k) * 64 + lane]) + (sums[(32 + k) * 64 + lane] + sums[(48 + k) * 64 + lane]);
  muon_results<1, 1, MODE, false>(a, of, parts, u64(down) * 32, u64(across) * 32, down != across, sum);
}

}  // namespace zc
