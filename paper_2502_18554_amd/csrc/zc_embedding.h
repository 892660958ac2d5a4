// Rows of a table by tokens, times a factor, and the table's gradient: for every token the sum of the output gradient's rows where it stands.
//
// out[i] = factor table[token[i]], zeros where the token is not one of the table's.  grad[v] (+)= factor (sum over i with token[i] = v of dy[i]); rows that no token names are zeros.
//
// Both are bound by memory.  The gradient's sums are made without atomics, so that equal calls give equal results: a first launch puts the places of equal tokens
// next to each other, in an order that depends on the tokens only; a second one adds pieces of that order, `chunk` places each, and writes every row whose places lie in one piece;
// a third adds what the pieces have of the other rows.
#pragma once

#include "zc_rows.h"

namespace zc {

template <int BITS> struct TokenOf;
template <> struct TokenOf<32> { using One = i32; };
template <> struct TokenOf<64> { using One = i64; };

// A token as a row of the table, ~0 for one that the table has not.
template <int BITS>
__device__ inline u32 row_of_token(const void* tokens, u64 i, u64 rows) {
  const i64 t = i64(static_cast<const typename TokenOf<BITS>::One*>(tokens)[i]);
  return u64(t) < rows ? u32(t) : ~0u;
}

struct EmbeddingArgs {
  const void* table;
  const void* tokens;
  void* out;
  u64 n, rows, cols, table_stride, out_stride;
  float factor;
  int table_type, out_type;
  u32 pieces_log2;               // threads that share a row
};

// A workgroup has 256 >> pieces_log2 rows at a time; its threads go along a row by pieces of eight values.
template <int BITS, bool TABLE32, bool OUT32>
__global__ __launch_bounds__(256) void embedding_kernel(EmbeddingArgs a) {
  const u32 along = threadIdx.x & ((1u << a.pieces_log2) - 1u), in_group = threadIdx.x >> a.pieces_log2, at_once = 256u >> a.pieces_log2;
  const u64 first = u64(blockIdx.x) * at_once + in_group, step = u64(gridDim.x) * at_once;
  for (u64 i = first; i < a.n; i += step) {
    const u32 row = row_of_token<BITS>(a.tokens, i, a.rows);
    for (u64 col = 8 * (u64(blockIdx.y) << a.pieces_log2 | along); col < a.cols; col += u64(gridDim.y) << (a.pieces_log2 + 3)) {
      const i32 left = left_of(a.cols, col);
      float v[8];
      numbers_of<TABLE32>(load_eight<TABLE32>(a.table, u64(row) * a.table_stride + col, row == ~0u ? 0 : left), a.table_type, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = row == ~0u ? 0.0f : v[j] * a.factor;
      store_eight<OUT32>(a.out, a.out_type, i * a.out_stride + col, left, v);
    }
  }
}

// ---- The places of equal tokens next to each other.
//
// Rows of the table are dealt to the workgroups in turn: workgroup g of G (a power of two) has those with row % G = g, kTokenRows at most.  Every workgroup reads all tokens: it counts those
// of the workgroups before it, so that it knows where its own places begin, and its own ones, row by row for each of its waves, which have a stretch of the tokens each.  Then it goes
// through them again, and every wave writes down the places behind those of the waves before it.  Equal tokens of 64 are found by asking the lanes for each different one of them.
constexpr u32 kTokenWaves = 16;
constexpr u32 kTokenRows = 1024;
constexpr u32 kZeroRows = 64;                     // rows that a workgroup looks through for such as no token names: a lane each
struct TokenArgs {
  const void* tokens;
  u32* place;                    // [n]: the places, those of a row next to each other
  u32* row;                      // [n]: the rows that they belong to
  u32* first;                    // [G per + 1]: where those of row v begin, at [v % G per + v / G]; and the number of places that have a row
  u64 n, rows;
  u32 groups_log2, per;
};

template <int BITS>
__global__ __launch_bounds__(64 * kTokenWaves) void token_order_kernel(TokenArgs a) {
  __shared__ u32 count[kTokenWaves][kTokenRows];
  __shared__ u32 total[kTokenWaves];
  const u32 lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = blockIdx.x, mask = (1u << a.groups_log2) - 1u;
  for (u32 i = threadIdx.x; i < kTokenWaves * kTokenRows; i += 64 * kTokenWaves) (&count[0][0])[i] = 0;
  __syncthreads();
  const u64 stretch = (a.n + 64 * kTokenWaves - 1) / (64 * kTokenWaves) * 64, begin = u64(wave) * stretch, end = begin + stretch < a.n ? begin + stretch : a.n;
  u32 before = 0;
#pragma unroll 4
  for (u64 i = begin + lane; i < end; i += 64) {
    const u32 row = row_of_token<BITS>(a.tokens, i, a.rows);
    if (row == ~0u) continue;
    before += (row & mask) < g ? 1u : 0u;
    if ((row & mask) == g) atomicAdd(&count[wave][row >> a.groups_log2], 1u);
  }
  before = wave_sum_u32(before);
  if (lane == 0) total[wave] = before;
  __syncthreads();
  before = 0;
#pragma unroll
  for (u32 w = 0; w < kTokenWaves; ++w) before += total[w];
  // A thread has one of the workgroup's rows: how many places it has in all, and of the rows before it.
  static_assert(kTokenRows == 64 * kTokenWaves && kZeroRows == 64);
  u32 mine = 0;
#pragma unroll
  for (u32 w = 0; w < kTokenWaves; ++w) mine += count[w][threadIdx.x];
  const u32 through = wave_inclusive_sum(mine);
  __syncthreads();
  if (lane == 63) total[wave] = through;
  __syncthreads();
  u32 at = before + through - mine;
  for (u32 w = 0; w < wave; ++w) at += total[w];
  if (threadIdx.x < a.per) a.first[u64(g) * a.per + threadIdx.x] = at;
  if (g == mask && threadIdx.x == kTokenRows - 1) a.first[u64(g + 1) * a.per] = at + mine;
#pragma unroll
  for (u32 w = 0; w < kTokenWaves; ++w) {
    const u32 of_wave = count[w][threadIdx.x];
    count[w][threadIdx.x] = at;
    at += of_wave;
  }
  __syncthreads();
  for (u64 base = begin; base < end; base += 64) {
    const u64 i = base + lane;
    const u32 row = i < end ? row_of_token<BITS>(a.tokens, i, a.rows) : ~0u;
    u64 open = __ballot(row != ~0u && (row & mask) == g);
    while (open) {
      const u32 one = lane_value(row, __builtin_ctzll(open));
      const u64 same = __ballot(row == one);
      const u32 to = count[wave][one >> a.groups_log2];
      if (row == one) {
        const u32 mine_at = to + u32(__popcll(same & ((u64(1) << lane) - 1)));
        a.place[mine_at] = u32(i);
        a.row[mine_at] = one;
      }
      if (lane == 0) count[wave][one >> a.groups_log2] = to + u32(__popcll(same));     // (a wave's accesses to LDS are in order)
      __builtin_amdgcn_wave_barrier();
      open &= ~same;
    }
  }
}

// ---- The sums.
struct EmbeddingBackwardArgs {
  const void* dy;
  const u32* place;
  const u32* row;
  const u32* first;
  float* partial;                // [piece][2][cols]: sums of a row that began in a piece before, and of one that goes on in the next
  void* grad;
  u64 rows, cols, dy_stride, grad_stride;
  float factor;
  int dy_type, grad_type;
  u32 add, chunk_log2, slots, per, groups_log2, pieces;
};

template <bool DY32>
__device__ inline void finish_row(const EmbeddingBackwardArgs& a, u32 row, u64 col, i32 left, float (&sum)[8]) {
  const u64 at = u64(row) * a.grad_stride + col;
  float v[8] = {};
  if (a.add) load_numbers(a.grad, a.grad_type, at, left, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf(sum[j], a.factor, v[j]);
  store_numbers(a.grad, a.grad_type, at, left, v);
}

// Workgroups [0, pieces) of a column of the grid have a piece each; where the whole gradient is written, those behind have kZeroRows slots each, whose rows they fill with zeros
// if no token names them.
constexpr u32 kRowsAhead = 8;
template <bool DY32>
__global__ __launch_bounds__(256) void embedding_sums_kernel(EmbeddingBackwardArgs a) {
  const u64 col = u64(blockIdx.y) * 2048 + 8 * threadIdx.x;
  const i32 left = left_of(a.cols, col);
  const u32 there = a.first[a.slots];
  if (blockIdx.x >= a.pieces) {
    const u32 slot0 = (blockIdx.x - a.pieces) * kZeroRows, slot1 = min(slot0 + kZeroRows, a.slots);
    const u32 lane = threadIdx.x & 63u, slot = slot0 + lane;
    const bool empty = slot < slot1 && a.first[slot] == a.first[slot + 1];
    for (u64 open = __ballot(empty); open; open &= open - 1) {
      const u32 of = slot0 + u32(__builtin_ctzll(open));
      const u64 row = u64(of % a.per) << a.groups_log2 | of / a.per;
      const float zeros[8] = {};
      if (row < a.rows) store_numbers(a.grad, a.grad_type, row * a.grad_stride + col, left, zeros);
    }
    return;
  }
  const u32 begin = blockIdx.x << a.chunk_log2;
  if (begin >= there) return;
  const u32 end = min(begin + (1u << a.chunk_log2), there);
  const u32 ahead = begin ? a.row[begin - 1] : ~0u, behind = end < there ? a.row[end] : ~0u;
  float* const partial = a.partial + u64(blockIdx.x) * 2 * a.cols;
  u32 now = uniform(a.row[begin]);
  bool began_before = now == ahead;
  float sum[8] = {};
  for (u32 e = begin; e < end; e += kRowsAhead) {
    RawEight<DY32> raw[kRowsAhead];
    u32 row[kRowsAhead];
#pragma unroll
    for (u32 k = 0; k < kRowsAhead; ++k) {
      const u32 i = min(e + k, end - 1);
      row[k] = uniform(a.row[i]);
      raw[k] = load_eight<DY32>(a.dy, u64(uniform(a.place[i])) * a.dy_stride + col, left);
    }
#pragma unroll
    for (u32 k = 0; k < kRowsAhead; ++k) {
      if (e + k >= end) break;
      if (row[k] != now) {
        if (began_before) store_eight<true>(partial, ZC_F32, col, left, sum);
        else finish_row<DY32>(a, now, col, left, sum);
        now = row[k];
        began_before = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
      }
      float v[8];
      numbers_of<DY32>(raw[k], a.dy_type, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
  }
  if (began_before) store_eight<true>(partial, ZC_F32, col, left, sum);
  else if (now == behind) store_eight<true>(partial, ZC_F32, a.cols + col, left, sum);
  else finish_row<DY32>(a, now, col, left, sum);
}

// The row that begins in piece blockIdx.x and goes on, 256 columns (blockIdx.y) of it: the pieces' sums in four strands, then these.
__global__ __launch_bounds__(256) void embedding_joins_kernel(EmbeddingBackwardArgs a) {
  __shared__ float strand[4][256];
  const u32 there = a.first[a.slots], end = (blockIdx.x + 1) << a.chunk_log2;
  if (end >= there) return;
  const u32 row = a.row[end - 1];
  if (a.row[end] != row) return;
  const u32 slot = (row & ((1u << a.groups_log2) - 1u)) * a.per + (row >> a.groups_log2);
  if (a.first[slot] >> a.chunk_log2 != blockIdx.x) return;               // (it began in a piece before)
  const u32 last = (a.first[slot + 1] - 1) >> a.chunk_log2;
  const u32 lane = threadIdx.x & 63u, s = threadIdx.x >> 6;
  const u64 col = u64(blockIdx.y) * 256 + 4 * lane;
  const i32 left = col >= a.cols ? 0 : i32(a.cols - col < 4 ? a.cols - col : 4);
  float sum[4] = {};
#pragma unroll 4
  for (u32 p = blockIdx.x + s; p <= last; p += 4) {
    const float* from = a.partial + (u64(p) * 2 + (p == blockIdx.x ? 1 : 0)) * a.cols + col;
    if (left == 4) {
      const F32Four v = *reinterpret_cast<const F32Four*>(from);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += v.v[j];
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < left) sum[j] += from[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) strand[s][4 * lane + j] = sum[j];
  __syncthreads();
  const u64 to = u64(blockIdx.y) * 256 + threadIdx.x;
  if (to >= a.cols) return;
  float v = ((strand[0][threadIdx.x] + strand[1][threadIdx.x]) + (strand[2][threadIdx.x] + strand[3][threadIdx.x])) * a.factor;
  const u64 at = u64(row) * a.grad_stride + to;
  if (a.add) v += load_value(a.grad, a.grad_type, at);
  store_value(a.grad, a.grad_type, at, v);
}

}  // namespace zc
