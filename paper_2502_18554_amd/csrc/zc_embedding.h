// Rows of a table by tokens, times a factor, and the table's gradient: for every token the sum of the output gradient's rows where it stands.
//
// out[i] = factor table[token[i]], zeros where the token is not one of the table's.  grad[v] (+)= factor (sum over i with token[i] = v of dy[i]); rows that no token names are zeros.
//
// Both are bound by memory.  The gradient's sums are made without atomics, so that equal calls give equal results: a first launch puts the places of equal tokens
// next to each other, in an order that depends on the tokens only; a second one adds pieces of that order, `chunk` places each, and writes every row whose places lie in one piece;
// a third adds what the pieces have of the other rows.  (32768 rows of 2048 values of 16 bits, a tenth of them padding, into 50021 of 32 bits: 14, 121 and 10 us, 4.4 TB/s in the second, of
// which three quarters are writes; 5117 rows of 777 values of 32 bits, added to 1009: 5, 12.5 and 7.5 us, waiting for memory one answer after the other in each.)
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

// A workgroup has 256 >> pieces_log2 rows at a time; its threads go along a row by pieces of eight values, four rows' pieces on their way together (16384 rows of 2048 values,
// 32 bits to 16: 26.2 us, one row after the other 27.3).
constexpr u32 kEmbeddingRows = 4;
template <int BITS, bool TABLE32, bool OUT32>
__global__ __launch_bounds__(256) void embedding_kernel(EmbeddingArgs a) {
  const u32 along = threadIdx.x & ((1u << a.pieces_log2) - 1u), in_group = threadIdx.x >> a.pieces_log2, at_once = 256u >> a.pieces_log2;
  const u64 first = u64(blockIdx.x) * at_once + in_group, step = u64(gridDim.x) * at_once;
  for (u64 i = first; i < a.n; i += step * kEmbeddingRows) {
    u32 row[kEmbeddingRows];
#pragma unroll
    for (u32 k = 0; k < kEmbeddingRows; ++k) row[k] = i + k * step < a.n ? row_of_token<BITS>(a.tokens, i + k * step, a.rows) : ~0u;
    for (u64 col = 8 * (u64(blockIdx.y) << a.pieces_log2 | along); col < a.cols; col += u64(gridDim.y) << (a.pieces_log2 + 3)) {
      const i32 left = left_of(a.cols, col);
      RawEight<TABLE32> raw[kEmbeddingRows];
#pragma unroll
      for (u32 k = 0; k < kEmbeddingRows; ++k) raw[k] = load_eight<TABLE32>(a.table, u64(row[k]) * a.table_stride + col, row[k] == ~0u ? 0 : left);
#pragma unroll
      for (u32 k = 0; k < kEmbeddingRows; ++k) {
        float v[8];
        numbers_of<TABLE32>(raw[k], a.table_type, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = row[k] == ~0u ? 0.0f : v[j] * a.factor;
        store_eight<OUT32>(a.out, a.out_type, (i + k * step) * a.out_stride + col, i + k * step < a.n ? left : 0, v);
      }
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
  u32* row;                      // [n]: the rows that they belong to; ~0 behind them
  u32* first;                    // [G per + 1]: where those of row v begin, at [v % G per + v / G]; and the number of places that have one
  u64 n, rows;
  u32 groups_log2, per;
};

// Every workgroup looks at every token, so what bounds it is instructions: groups of 64 tokens are told apart by masks in scalar registers, and the workgroup's own tokens go to a list in LDS,
// so that they need not be looked for again (32768 tokens of 64 bits, a table of 50021 rows: 14 us; looked for again 29).  A wave with more of them than its list takes does that.
// Every workgroup begins at another group, so that they do not all ask the same part of the cache at once.
constexpr u32 kTokensAhead = 8;
constexpr u32 kTokenList = 256;                     // of a wave
template <int BITS>
__global__ __launch_bounds__(64 * kTokenWaves) void token_order_kernel(TokenArgs a) {
  __shared__ u32 count[kTokenWaves][kTokenRows];
  __shared__ u32x2_t list[kTokenWaves][kTokenList];  // rows and places
  __shared__ u32 total[kTokenWaves];
  const u32 lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), g = blockIdx.x, mask = (1u << a.groups_log2) - 1u;
  // A wave has `groups` groups of 64 tokens; its k-th one is number (k + g) % groups of them.
  const u32 n = u32(a.n), rows = u32(a.rows), groups = n / (64 * kTokenWaves) + 1, begin = wave * groups * 64, start = g % groups;
  const bool full = u64(begin) + u64(groups) * 64 <= n;
  const auto group_of = [&](u32 k) { return begin + 64 * (k + start < groups ? k + start : k + start - groups); };
  typedef u32 Words __attribute__((ext_vector_type(BITS / 32)));
  const auto read = [&](u32 k) {
    const u32 at = group_of(k) + lane;
    return k < groups && at < n ? static_cast<const Words*>(a.tokens)[at] : Words(~0u);
  };
  // Which of 64 tokens are rows of the table.
  const auto there_of = [&](Words w) {
    const u64 there = __ballot(w[0] < rows);
    if constexpr (BITS == 64) return there & __ballot(w[1] == 0);
    else return there;
  };
  if (threadIdx.x < a.per) {
#pragma unroll
    for (u32 w = 0; w < kTokenWaves; ++w) count[w][threadIdx.x] = 0;
  }
  __syncthreads();
  u32 before = 0, listed = 0;
  for (u32 k0 = 0; k0 < groups; k0 += kTokensAhead) {
    Words w[kTokensAhead];
    if (full && k0 + kTokensAhead <= groups) {
#pragma unroll
      for (u32 k = 0; k < kTokensAhead; ++k) w[k] = *at_bytes(static_cast<const Words*>(a.tokens) + group_of(k0 + k), u32(sizeof(Words)) * lane);
    } else {
#pragma unroll
      for (u32 k = 0; k < kTokensAhead; ++k) w[k] = read(k0 + k);
    }
#pragma unroll
    for (u32 k = 0; k < kTokensAhead; ++k) {
      const u32 of = w[k][0] & mask;
      const u64 there = there_of(w[k]), own = there & __ballot(of == g);
      before += u32(__popcll(there & __ballot(of < g)));
      if (own) {
        if (own >> lane & 1) {
          const u32 to = listed + u32(__popcll(own & ((u64(1) << lane) - 1)));
          if (to < kTokenList) list[wave][to] = u32x2_t{w[k][0], group_of(k0 + k) + lane};
          atomicAdd(&count[wave][w[k][0] >> a.groups_log2], 1u);
        }
        listed += u32(__popcll(own));
      }
    }
  }
  if (lane == 0) total[wave] = before;
  __syncthreads();
  before = 0;
#pragma unroll
  for (u32 w = 0; w < kTokenWaves; ++w) before += total[w];
  // A thread has one of the workgroup's rows: how many places it has in all, and of the rows before it.
  static_assert(kTokenRows == 64 * kTokenWaves && kZeroRows == 64);
  u32 mine = 0;
  if (threadIdx.x < a.per) {
#pragma unroll
    for (u32 w = 0; w < kTokenWaves; ++w) mine += count[w][threadIdx.x];
  }
  const u32 through = wave_inclusive_sum(mine);
  __syncthreads();
  if (lane == 63) total[wave] = through;
  __syncthreads();
  u32 at = before + through - mine;
  for (u32 w = 0; w < wave; ++w) at += total[w];
  if (threadIdx.x < a.per) {
    a.first[u64(g) * a.per + threadIdx.x] = at;
    u32 to = at;
#pragma unroll
    for (u32 w = 0; w < kTokenWaves; ++w) {
      const u32 of_wave = count[w][threadIdx.x];
      count[w][threadIdx.x] = to;
      to += of_wave;
    }
  }
  if (g == mask) {                                   // the last workgroup: the number of places that have a row, and no rows behind them
    u32 all = before;
#pragma unroll
    for (u32 w = 0; w < kTokenWaves; ++w) all += total[w];
    if (threadIdx.x == 0) a.first[u64(g + 1) * a.per] = all;
    for (u32 i = all + threadIdx.x; i < n; i += 64 * kTokenWaves) a.row[i] = ~0u;
  }
  __syncthreads();
  // The places of 64 tokens of which `own` are the workgroup's: equal ones one behind the other, behind those that came before.
  const auto put = [&](u32 row, u32 place, u64 own) {
    while (own) {
      const u32 one = lane_value(row, __builtin_ctzll(own));
      const u64 same = __ballot(row == one) & own;
      const u32 to = count[wave][one >> a.groups_log2];
      if (same >> lane & 1) {
        const u32 mine_at = to + u32(__popcll(same & ((u64(1) << lane) - 1)));
        a.place[mine_at] = place;
        a.row[mine_at] = one;
      }
      if (lane == 0) count[wave][one >> a.groups_log2] = to + u32(__popcll(same));       // (a wave's accesses to LDS are in order)
      __builtin_amdgcn_wave_barrier();
      own &= ~same;
    }
  };
  if (listed <= kTokenList) {
    for (u32 k = 0; k < listed; k += 64) {
      const u32x2_t w = list[wave][min(k + lane, kTokenList - 1)];
      put(w[0], w[1], __ballot(k + lane < listed));
    }
  } else {
    Words next = read(0);
    for (u32 k = 0; k < groups; ++k) {
      const Words w = next;
      next = read(k + 1);
      put(w[0], group_of(k) + lane, there_of(w) & __ballot((w[0] & mask) == g));
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
  u64 n, rows, cols, dy_stride, grad_stride;
  float factor;
  int dy_type, grad_type;
  u32 add, chunk_log2, slots, per, groups_log2;
  u64 zeros_share;               // of the workgroups, times 2^32
};

// A workgroup has a piece; or, where the whole gradient is written, kZeroRows slots, whose rows it fills with zeros if no token names them.  The two kinds come in turn, by their
// shares of the grid, so that reading and writing go on together.  A piece's places and rows are read at once, by the lanes, then eight rows of dy at a time, or
// four with what they are added to; a row of the gradient is written once.  (32768 rows of 2048 values of 16 bits into 50021 of 32 bits: written 138 us, 153 with four at a time; added 116 us, 129 with eight.)
// Zeros from one byte of a row to another (both of whole values), by all threads, 16 bytes each: neighbouring lanes write neighbouring bytes, past the caches.
__device__ inline void clear_bytes(u8* row, u64 from, u64 to) {
  struct __attribute__((packed, aligned(2))) Sixteen { u32x4_t v; };
  u64 at = from + 16 * threadIdx.x;
  for (; at + 16 <= to; at += 16 * blockDim.x) __builtin_nontemporal_store(u32x4_t{}, &reinterpret_cast<Sixteen*>(row + at)->v);
  for (; at < to; at += 2) *reinterpret_cast<u16*>(row + at) = 0;       // (one thread's, less than 16 bytes)
}

template <bool DY32, bool ADD>
__global__ __launch_bounds__(256) void embedding_sums_kernel(EmbeddingBackwardArgs a) {
  constexpr u32 AHEAD = ADD ? 4 : 8;
  const u64 col = u64(blockIdx.y) * 2048 + 8 * threadIdx.x;
  const i32 left = left_of(a.cols, col);
  const u32 lane = threadIdx.x & 63u;
  const u32 zeros_before = u32(u64(blockIdx.x) * a.zeros_share >> 32), piece = blockIdx.x - zeros_before;
  if (!ADD && u32((u64(blockIdx.x) + 1) * a.zeros_share >> 32) > zeros_before) {
    const u32 slot0 = zeros_before * kZeroRows, slot1 = min(slot0 + kZeroRows, a.slots), slot = slot0 + lane;
    const bool empty = slot < slot1 && a.first[slot] == a.first[slot + 1];
    for (u64 open = __ballot(empty); open; open &= open - 1) {
      const u32 of = slot0 + u32(__builtin_ctzll(open));
      const u64 row = u64(of % a.per) << a.groups_log2 | of / a.per;
      if (row >= a.rows) continue;
      u8* const to = static_cast<u8*>(a.grad) + row * a.grad_stride * value_bytes(a.grad_type);
      clear_bytes(to, u64(blockIdx.y) * 2048 * value_bytes(a.grad_type), min((u64(blockIdx.y) + 1) * 2048, a.cols) * value_bytes(a.grad_type));
    }
    return;
  }
  const u64 begin = u64(piece) << a.chunk_log2, end = min(begin + (u64(1) << a.chunk_log2), a.n);
  const u32 ahead = begin ? a.row[begin - 1] : ~0u, behind = end < a.n ? a.row[end] : ~0u;
  float* const partial = a.partial + u64(piece) * 2 * a.cols;
  float sum[8] = {};
  bool began_before = false;
  u32 last = ~0u;                                    // the row before
  for (u64 at = begin; at < end; at += 64) {
    const u64 mine = at + lane;
    const u32 my_row = mine < end ? a.row[mine] : ~0u, my_place = mine < end ? a.place[mine] : 0u;
    const u32 behind_these = at + 64 < end ? uniform(a.row[at + 64]) : uniform(behind);
    if (at == begin) {
      last = lane_value(my_row, 0);
      if (last == ~0u) return;
      began_before = last == uniform(ahead);
    }
    const u32 count = u32(min(end - at, u64(64)));
    for (u32 e = 0; e < count; e += AHEAD) {
      RawEight<DY32> raw[AHEAD];
      RawEight<true> old[ADD ? AHEAD : 1];      // what is added to, in its own type
      u32 row[AHEAD + 1];
#pragma unroll
      for (u32 k = 0; k < AHEAD; ++k) {
        row[k] = e + k < count ? lane_value(my_row, int(e + k)) : ~0u;
        raw[k] = load_eight<DY32>(a.dy, u64(lane_value(my_place, int((e + k) & 63u))) * a.dy_stride + col, row[k] == ~0u ? 0 : left);
      }
      row[AHEAD] = e + AHEAD < count ? lane_value(my_row, int((e + AHEAD) & 63u)) : e + AHEAD == count ? behind_these : ~0u;
      const auto ends = [&](u32 k) { return row[k] != ~0u && row[k] != (e + k + 1 == count ? behind_these : row[k + 1]); };
      if constexpr (ADD) {
        if (a.grad_type == ZC_F32) {
#pragma unroll
          for (u32 k = 0; k < AHEAD; ++k) old[k] = load_eight<true>(a.grad, u64(row[k]) * a.grad_stride + col, ends(k) ? left : 0);
        } else {
#pragma unroll
          for (u32 k = 0; k < AHEAD; ++k) {
            const RawEight<false> r = load_eight<false>(a.grad, u64(row[k]) * a.grad_stride + col, ends(k) ? left : 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) old[k].w[j] = r.w[j];
          }
        }
      }
#pragma unroll
      for (u32 k = 0; k < AHEAD; ++k) {
        if (row[k] == ~0u) break;
        float v[8];
        numbers_of<DY32>(raw[k], a.dy_type, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
        last = row[k];
        if (!ends(k)) continue;
        if (began_before) {
          store_eight<true>(partial, ZC_F32, col, left, sum);
        } else {
          float v[8] = {};
          if constexpr (ADD) {
            if (a.grad_type == ZC_F32) numbers_of<true>(old[k], ZC_F32, v);
            else numbers_of<false>(RawEight<false>{{old[k].w[0], old[k].w[1], old[k].w[2], old[k].w[3]}}, a.grad_type, v);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[j] = ADD ? __builtin_fmaf(sum[j], a.factor, v[j]) : sum[j] * a.factor;
          store_numbers(a.grad, a.grad_type, u64(row[k]) * a.grad_stride + col, left, sum);
        }
        began_before = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        last = ~0u;
      }
    }
  }
  if (last != ~0u) store_eight<true>(partial, ZC_F32, began_before ? col : a.cols + col, left, sum);         // (a row that goes on)
}

// The rows that begin in one of kJoinPieces pieces and go on, 256 columns (blockIdx.y) of them.  A row of few pieces is one wave's; of one with more, every wave adds every eighth
// piece, and then they are added.
constexpr u32 kJoinPieces = 8, kJoinWaves = 8, kFewPieces = 16;
struct JoinColumns {
  u64 col;
  i32 left;                                              // columns from there on, 4 at most
};
__device__ inline void add_partials(const EmbeddingBackwardArgs& a, JoinColumns c, u32 first, u32 last, u32 piece, u32 apart, float (&sum)[4]) {
#pragma unroll 4
  for (u32 p = first; p <= last; p += apart) {
    const float* from = a.partial + (u64(p) * 2 + (p == piece ? 1 : 0)) * a.cols + c.col;
    if (c.left == 4) {
      const F32Four v = *reinterpret_cast<const F32Four*>(from);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += v.v[j];
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < c.left) sum[j] += from[j];
    }
  }
}
__device__ inline void finish_join(const EmbeddingBackwardArgs& a, JoinColumns c, u32 row, const float (&sum)[4], const float (&old)[4]) {
  const u64 at = u64(row) * a.grad_stride + c.col;
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = a.add ? __builtin_fmaf(sum[j], a.factor, old[j]) : sum[j] * a.factor;
  if (c.left == 4) {
    store_four(a.grad, a.grad_type, at, v);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < c.left) store_value(a.grad, a.grad_type, at + j, v[j]);
  }
}
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_joins_kernel(EmbeddingBackwardArgs a) {
  __shared__ float strand[kJoinWaves][256];
  const u32 lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
  u32 row = ~0u, last = 0;                               // of piece blockIdx.x * kJoinPieces + lane
  const u32 my_piece = blockIdx.x * kJoinPieces + lane;
  if (lane < kJoinPieces) {
    const u64 end = (u64(my_piece) + 1) << a.chunk_log2;
    if (end < a.n) {
      const u32 before = a.row[end - 1], behind = a.row[end];
      if (before == behind && before != ~0u) {
        const u32 slot = (before & ((1u << a.groups_log2) - 1u)) * a.per + (before >> a.groups_log2), from = a.first[slot], to = a.first[slot + 1];
        if (from >> a.chunk_log2 == my_piece) row = before, last = (to - 1) >> a.chunk_log2;
      }
    }
  }
  const u64 col = u64(blockIdx.y) * 256 + 4 * lane;
  const JoinColumns c{col, col >= a.cols ? 0 : i32(a.cols - col < 4 ? a.cols - col : 4)};
  const auto load_old = [&](u32 of_row, float (&old)[4]) {
    if (!a.add) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < c.left) old[j] = load_value(a.grad, a.grad_type, u64(of_row) * a.grad_stride + c.col + j);
  };
  u64 open = __ballot(row != ~0u);
  const u64 few = __ballot(row != ~0u && last - my_piece < kFewPieces);
  static_assert(kJoinPieces <= kJoinWaves);
  if (few >> wave & 1) {
    const u32 piece = lane_value(my_piece, int(wave)), end = lane_value(last, int(wave)), of_row = lane_value(row, int(wave));
    float old[4] = {}, sum[4] = {};
    load_old(of_row, old);
    add_partials(a, c, piece, end, piece, 1, sum);
    finish_join(a, c, of_row, sum, old);
  }
  for (open &= ~few; open; open &= open - 1) {           // (the same for all waves)
    const int of = __builtin_ctzll(open);
    const u32 piece = lane_value(my_piece, of), end = lane_value(last, of), of_row = lane_value(row, of);
    float old[4] = {}, sum[4] = {};
    if (wave == 0) load_old(of_row, old);
    add_partials(a, c, piece + wave, end, piece, kJoinWaves, sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) strand[wave][4 * lane + j] = sum[j];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] = 0.0f;
#pragma unroll
      for (u32 k = 0; k < kJoinWaves; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += strand[k][4 * lane + j];
      finish_join(a, c, of_row, sum, old);
    }
    __syncthreads();
  }
}

}  // namespace zc
