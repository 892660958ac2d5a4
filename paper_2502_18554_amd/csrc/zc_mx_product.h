// Products of matrices held in 4 bits, both along their rows: out[i][j] (+)= sum over k of a[i][k] b[j][k], + bias[j].
//
// The matrix instructions take a block as it lies in memory: a lane's operand is the 16 bytes of one block with its scale byte, and they
// scale, multiply and add in binary32.  Sums are rounded once, to the output's type.
#pragma once

#include "zc_mx.h"
#include "zc_to_lds.h"

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

// Four neighbouring results of a row: the bias, what is there already, and the one rounding.
__device__ inline void mx_finish(const MxProductArgs& a, u64 row, u64 col, float (&v)[4]) {
  const u64 at = row * a.out_stride + col;
  if (col + 4 <= a.n) {
    if (a.bias) {
      const F32Four b = *reinterpret_cast<const F32Four*>(a.bias + col);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += b.v[j];
    }
    if (a.add) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += load_value(a.out, a.out_type, at + j);
    }
    store_four(a.out, a.out_type, at, v);
  } else {
    for (int j = 0; j < 4; ++j) {
      if (col + j >= a.n) break;
      if (a.bias) v[j] += a.bias[col + j];
      if (a.add) v[j] += load_value(a.out, a.out_type, at + j);
      store_value(a.out, a.out_type, at + j, v[j]);
    }
  }
}

// ---- Products of many rows: workgroups of 2 x 2 waves, a wave makes (32 TM) x (32 TN) results.
//
// A stage is 8 blocks (128 bytes) of every row of the tile, brought straight to LDS while the stage before is multiplied.  Rows follow each
// other in LDS, their eight 16-byte blocks exchanged by the row's number, so that 16 lanes that read LDS together find 64 different banks.
// Scale bytes come by four stages (32 bytes of a row, by two lanes) through registers.
//
// An instruction multiplies two blocks of 32 rows with 32 columns: lanes 0 .. 31 bring one block each, lanes 32 .. 63 the other.  Which two blocks of the
// stage these are is free: it is blocks t and 4 + t, so that a lane's scale bytes of the stage are the four bytes of one word, of which
// the instruction takes the one that it is told.  Which column of the tile a lane brings is free as well: it is chosen so that a lane ends
// with 16 neighbouring results, which it writes itself.
//
// A workgroup goes through several tiles without a pause: the requests run two stages ahead, into the next tile too, while the results of this one are written.
//
// Bound by the matrix instructions, and by what they wait for each other and LDS: 8192 x 8192 x 8192 by tiles of 256 249-256 us (4.3 PFLOP/s; a tile of 256 x 256 alone on the GPU
// would go at 5.2, the instruction by itself, on constant operands, at 8.2).  A turn of tiles of 256 costs some 8 us beyond its products: half of it the results' way out of the matrix
// instructions' registers, half the 33 MB that all CUs write at once.  Tiles of 64: 333 x 1531 x 1000 4.3 us, of 128: 2048 x 2048 x 2048 10 us.
constexpr u32 kStageBlocks = 8;
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) u32 MxLdsWord;

__host__ __device__ constexpr u32 mx_tile_rows(int t) { return 64u * u32(t); }

// Tiles in the order of the workgroups: every XCD has a run of neighbouring tiles (workgroups go round the eight XCDs), which goes down strips of eight rows of
// tiles; its workgroups take the tiles of the run in turn.
struct MxTiles {
  u32 down, across, first, count, step;          // of the grid; a workgroup's own: first one, one behind the run's last one, from one to the next
  __device__ MxTiles(u32 tiles_down, u32 tiles_across) : down(tiles_down), across(tiles_across) {
    const u32 tiles = down * across, xcd = blockIdx.x & 7u, share = tiles >> 3, more = tiles & 7u;
    const u32 begin = xcd * share + min(xcd, more);
    first = begin + (blockIdx.x >> 3);
    count = begin + share + (xcd < more ? 1u : 0u);
    step = (gridDim.x + 7u - xcd) >> 3;
  }
  __device__ void place(u32 t, u32& row, u32& col) const {
    const u32 strip = t / (8u * across), rest = t - strip * 8u * across, high = min(8u, down - 8u * strip);
    const u32 c = rest / high;
    col = u32(__builtin_amdgcn_readfirstlane(int(c)));
    row = u32(__builtin_amdgcn_readfirstlane(int(8u * strip + rest - c * high)));
  }
};

// Rows of a tile as a buffer, seen from some bytes along them: what lies behind the last row's `used` bytes reads as zeros.  (Everything that a lane adds
// to the address is in its own offset: of the instruction's offsets that is the one whose bounds are checked.)
struct MxRows {
  u64 at;
  u32 bytes;
  __device__ void aim(const u8* base, u64 first, u64 rows, u64 stride, u32 most, u32 used) {
    at = reinterpret_cast<u64>(base) + first * stride;
    bytes = u32((min(rows - first, u64(most)) - 1) * stride) + used;
  }
  __device__ void move_on(u32 by) {
    at += by;
    bytes = bytes > by ? bytes - by : 0u;
  }
  __device__ __amdgpu_buffer_rsrc_t buffer() const {
    const u32 low = u32(__builtin_amdgcn_readfirstlane(int(u32(at)))), high = u32(__builtin_amdgcn_readfirstlane(int(u32(at >> 32))));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u64(low) | u64(high) << 32), 0, __builtin_amdgcn_readfirstlane(int(bytes)), 0x00027000);
  }
};
constexpr u64 kMostTileStride = u64(1) << 23;       // (256 rows are less than 2^32 bytes)

template <typename T>
__device__ inline const __attribute__((address_space(3))) T* mx_lds(u32 at) {
  return reinterpret_cast<const __attribute__((address_space(3))) T*>(at);
}

// Between two registers: 16 lanes 1 and 3 (of 0 .. 3) of the first with 16 lanes 0 and 2 of the second; the upper half of the first with the lower half of the second.
__device__ inline void swap_sixteens(u32& a, u32& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0], b = r[1];
}
__device__ inline void swap_halves(u32& a, u32& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0], b = r[1];
}

// The compiler has to have these sums here, in the matrix instructions' own registers where a wave has more of them than the others would hold (of those
// every value has to be moved before it can be written: 2048 x 2048 x 2048 10.0 us, 10.3 so).
template <int OF>
__device__ __forceinline__ void mx_hold(f32x16_t& sum) {
  if constexpr (OF > 4) asm volatile("" : "+a"(sum));
  else asm volatile("" : "+v"(sum));
}

// Two neighbouring values of a type, rounded, as a word; a value of 32 bits is one.
template <int TYPE>
__device__ inline u32 packed_pair(float low, float high) {
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef typename ValueOf<TYPE>::One Pair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u32, __builtin_convertvector((Two{low, high}), Pair));
}

// The results of a wave: row0 and col0 are its tile's first.  Lane l has, of 32 x 32, 16 neighbouring ones of row l % 32, from column 16 (l / 32) on.  Its pieces of 16 bytes go to
// other lanes so that four lanes write 64 bytes of a row together (16 rows a store): single pieces would be that many more requests to L2.
// WHOLE: the matrix has all of these results.  MORE: there may be a bias, or something to add to; then the sums themselves change lanes, and what is added is
// read as the results are written, 16 bytes a lane (333 x 1531 x 1000 with both 6.4 us; a value at a time, where a lane's sums were, 9.3).
template <int TM, int TN, int TYPE, bool WHOLE, bool MORE>
__device__ __forceinline__ void mx_write_tile(const MxProductArgs& a, u64 row0, u64 col0, u32 lane, f32x16_t (&sum)[TM][TN]) {
  using One = typename ValueOf<TYPE>::One;
  constexpr u32 N = 16 / sizeof(One), PIECES = 16 / N;   // values of a piece; a lane's pieces
  struct __attribute__((packed, aligned(2))) Piece { u32 w[4]; };
  const u64 to_row0 = row0 + (lane & 15u), to_col0 = col0 + N * (lane >> 4);
  One* const to0 = static_cast<One*>(a.out) + to_row0 * a.out_stride + to_col0;
  // How many rows and columns there are from a lane's first on: what exceeds a tile does not matter.
  const int rows_left = int(min(i64(a.m) - i64(to_row0), i64(1024))), cols_left = int(max(min(i64(a.n) - i64(to_col0), i64(1024)), i64(-1024)));
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    float bias[8] = {};                                  // (added where there is none as well: loads that a branch may leave unused would be waited for in the next tile)
    if (MORE && a.bias) {
#pragma unroll
      for (u32 c = 0; c < 8; ++c) {
        const u64 col = to_col0 + 32 * j + (TYPE == ZC_F32 ? 16 * (c / 4) + c % 4 : c);
        bias[c] = a.bias[WHOLE ? col : min(col, a.n - 1)];                       // (of columns that there are none of: any)
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      mx_hold<TM * TN>(sum[i][j]);                       // (leaves the results in their registers until they are wanted)
      // The words that change lanes: rounded values in pairs, or, where something is added first, the sums.
      constexpr u32 WORDS = MORE || TYPE == ZC_F32 ? N : 4;
      u32 w[PIECES][WORDS];
#pragma unroll
      for (u32 d = 0; d < WORDS * PIECES; ++d) {
        if constexpr (WORDS == N) w[d / N][d % N] = __float_as_uint(sum[i][j][d]);
        else w[d / 4][d % 4] = packed_pair<TYPE>(sum[i][j][2 * d], sum[i][j][2 * d + 1]);
      }
#pragma unroll
      for (u32 d = 0; d < WORDS; ++d) {
        if constexpr (PIECES == 4) {
          swap_halves(w[0][d], w[2][d]);
          swap_halves(w[1][d], w[3][d]);
          swap_sixteens(w[2][d], w[3][d]);
        }
        swap_sixteens(w[0][d], w[1][d]);
      }
      // Piece q of a lane is now: row 16 (q % 2) + l % 16, 64 bytes number q / 2, of those the 16 bytes l / 16.
#pragma unroll
      for (u32 q = 0; q < PIECES; ++q) {
        One* const to = to0 + (32 * i + 16 * (q & 1u)) * a.out_stride + (32 * j + 4 * N * (q / 2));
        const int left = WHOLE || rows_left > int(32 * i + 16 * (q & 1u)) ? cols_left - int(32 * j + 4 * N * (q / 2)) : 0;
        Piece piece;
        if constexpr (MORE) {
          float v[N];
#pragma unroll
          for (u32 c = 0; c < N; ++c) v[c] = __uint_as_float(w[q][c]);
#pragma unroll
          for (u32 c = 0; c < N; ++c) v[c] += bias[TYPE == ZC_F32 ? 4 * (q / 2) + c : c];
          if (a.add) {
            One before[N] = {};
            if (WHOLE || left >= int(N)) {
              piece = *reinterpret_cast<const Piece*>(to);
              __builtin_memcpy(before, &piece, 16);
            } else if (left > 0) {
#pragma unroll
              for (u32 c = 0; c < N; ++c) before[c] = to[min(int(c), left - 1)];
            }
#pragma unroll
            for (u32 c = 0; c < N; ++c) v[c] += float(before[c]);
          }
#pragma unroll
          for (u32 d = 0; d < 4; ++d) {
            if constexpr (TYPE == ZC_F32) piece.w[d] = __float_as_uint(v[d]);
            else piece.w[d] = packed_pair<TYPE>(v[2 * d], v[2 * d + 1]);
          }
        } else {
          piece = Piece{{w[q][0], w[q][1], w[q][2], w[q][3]}};
        }
        if (WHOLE || left >= int(N)) {
          *reinterpret_cast<Piece*>(to) = piece;
        } else if (left > 0) {
          u32 d[4] = {piece.w[0], piece.w[1], piece.w[2], piece.w[3]};
#pragma unroll 1
          for (int c = 0; c < left; ++c) {               // one by one from the low end, as the rest moves down
            asm volatile("" ::: "memory");               // (keeps the stores above in one piece)
            if constexpr (TYPE == ZC_F32) {
              to[c] = __uint_as_float(d[0]);
              d[0] = d[1], d[1] = d[2], d[2] = d[3];
            } else {
              to[c] = __builtin_bit_cast(One, u16(d[0]));
#pragma unroll
              for (u32 e = 0; e < 4; ++e) d[e] = d[e] >> 16 | (e < 3 ? d[e + 1] << 16 : 0u);
            }
          }
        }
      }
    }
  }
}

template <int TM, int TN, int TYPE>
__global__ __launch_bounds__(256, TM * TN > 4 ? 1 : TM * TN > 1 ? 2 : 4) void mx_tile_kernel(MxProductArgs a, u32 tiles_down, u32 tiles_across) {
  constexpr u32 RA = mx_tile_rows(TM), RB = mx_tile_rows(TN), ROWS = RA + RB, LOADS = ROWS / 32;
  constexpr u32 SCALE_LOADS = ROWS / 128;
  // In LDS: two stages of a's rows, two of b's, the scale bytes of four pairs of stages of a's rows, of b's.
  constexpr u32 AT_B = 2 * RA * 128, AT_SCALES_A = 2 * ROWS * 128, AT_SCALES_B = AT_SCALES_A + 4 * RA * 16, LDS_BYTES = AT_SCALES_B + 4 * RB * 16;
  __shared__ u32x4_t memory[LDS_BYTES / 16];
  const u32 tid = threadIdx.x, lane = tid & 63u, wave = u32(__builtin_amdgcn_readfirstlane(int(tid >> 6)));
  const u32 half = lane >> 5, in32 = lane & 31u;
  const MxTiles tiles(tiles_down, tiles_across);
  if (tiles.first >= tiles.count) return;
  const u32 row_bytes = kMxBytes * a.blocks, scale_bytes = (a.blocks + 3u) & ~3u;
  const u32 pairs = (a.blocks + 2 * kStageBlocks - 1) / (2 * kStageBlocks);

  // What is asked for next: a tile's rows, and how far along them.
  u32 ask_tile = tiles.first, ask_pair = 0;
  MxRows rows_a, rows_b, scales_a, scales_b;
  const auto aim = [&] {
    u32 r, c;
    tiles.place(ask_tile, r, c);
    const u64 row = u64(r) * RA, col = u64(c) * RB;
    rows_a.aim(a.a, row, a.m, a.a_stride, RA, row_bytes);
    rows_b.aim(a.b, col, a.n, a.b_stride, RB, row_bytes);
    scales_a.aim(a.a_scales, row, a.m, a.a_scales_stride, RA, scale_bytes);
    scales_b.aim(a.b_scales, col, a.n, a.b_scales_stride, RB, scale_bytes);
  };
  // (Behind the last tile there is nothing to ask for.)
  const auto next_pair = [&] {
    if (++ask_pair < pairs) {
      scales_a.move_on(16);
      scales_b.move_on(16);
      return;
    }
    ask_pair = 0;
    ask_tile += tiles.step;
    if (ask_tile < tiles.count) aim();
    else rows_a.bytes = rows_b.bytes = scales_a.bytes = scales_b.bytes = 0;
  };

  // A thread's loads: 32 rows apart, so that the exchange of blocks is the same for all of them.
  const u32 my_row = tid >> 3;
  const u32 key_b = ((my_row >> 1) & 1u) | ((my_row >> 3) & 2u) | (my_row & 4u);
  u32 from_a[RA / 32], from_b[RB / 32];
#pragma unroll
  for (u32 i = 0; i < RA / 32; ++i) from_a[i] = (my_row + 32 * i) * u32(a.a_stride) + 16u * ((tid ^ (my_row >> 1)) & 7u);
#pragma unroll
  for (u32 i = 0; i < RB / 32; ++i) from_b[i] = (my_row + 32 * i) * u32(a.b_stride) + 16u * ((tid ^ key_b) & 7u);
  const u32 lds0 = u32(reinterpret_cast<uintptr_t>((MxLdsWord*)&memory[0]));
  const auto ask = [&](u32 u, u32 i) {
    const u32 to = lds0 + wave * 1024u;
    if (i < RA / 32) load_to_lds(rows_a.buffer(), to + u * (RA * 128u) + 4096u * i, from_a[i]);
    else load_to_lds(rows_b.buffer(), to + AT_B + u * (RB * 128u) + 4096u * (i - RA / 32), from_b[i - RA / 32]);
  };
  const auto next_stage = [&] {
    rows_a.move_on(128);
    rows_b.move_on(128);
  };
  u32x4_t held[SCALE_LOADS];
  const auto of_a = [&](u32 i) { return RA % 128 == 0 ? 128 * i < RA : 32 * wave + 128 * i < RA; };     // whose rows the loads are of
  u32 scales_at[SCALE_LOADS];
#pragma unroll
  for (u32 i = 0; i < SCALE_LOADS; ++i) {
    const u32 row = (tid >> 1) + 128 * i;
    scales_at[i] = (of_a(i) ? row * u32(a.a_scales_stride) : (row - RA) * u32(a.b_scales_stride)) + 16 * (tid & 1u);
  }
  const auto ask_scales = [&] {                         // 16 scale bytes of a row for the pair that is asked for, 16 for the next one; those behind the last block as zeros
    if (16 * ask_pair + 32 <= a.blocks) {
#pragma unroll
      for (u32 i = 0; i < SCALE_LOADS; ++i) held[i] = __builtin_amdgcn_raw_buffer_load_b128(of_a(i) ? scales_a.buffer() : scales_b.buffer(), scales_at[i], 0, 0);
    } else {
#pragma unroll
      for (u32 i = 0; i < SCALE_LOADS; ++i)
#pragma unroll
        for (u32 j = 0; j < 4; ++j) {
          const u32 first = 16 * (ask_pair + (tid & 1u)) + 4 * j;
          const u32 w = __builtin_amdgcn_raw_buffer_load_b32(of_a(i) ? scales_a.buffer() : scales_b.buffer(), first < a.blocks ? scales_at[i] + 4 * j : ~0u, 0, 0);
          held[i][j] = first + 4 <= a.blocks || first >= a.blocks ? w : w & ((1u << (8 * (a.blocks - first))) - 1u);
        }
    }
  };
  const auto put_scales = [&](u32 plane) {              // into this plane and the next one
#pragma unroll
    for (u32 i = 0; i < SCALE_LOADS; ++i) {
      const u32 row = (tid >> 1) + 128 * i;
      memory[(of_a(i) ? AT_SCALES_A : AT_SCALES_B - RA * 16) / 16 + (plane + (tid & 1u)) * (of_a(i) ? RA : RB) + row] = held[i];
    }
  };

  const u32 wave_a = (wave >> 1) * 32u * TM, wave_b = (wave & 1u) * 32u * TN;
  const u32 lane_b = (in32 & 3u) + 16u * ((in32 >> 2) & 1u) + 4u * (in32 >> 3);
  u32x4_t fa[2][TM], fb[2][TN];                         // of this step and of the next one
  u32 sa[2][TM], sb[2][TN];                             // of this stage and of the next one
  u32 at_a[4], at_b[4];                                 // where a lane's block of step t is, in the first stage's place
#pragma unroll
  for (u32 t = 0; t < 4; ++t) {
    at_a[t] = lds0 + (wave_a + in32) * 128u + 16u * ((4 * half + t) ^ (in32 >> 1 & 7u));
    at_b[t] = lds0 + AT_B + (wave_b + lane_b) * 128u + 16u * ((4 * half + t) ^ (((lane_b >> 1) & 1u) | ((lane_b >> 3) & 2u) | (lane_b & 4u)));
  }
  const u32 at_sa = lds0 + AT_SCALES_A + 16u * (wave_a + in32) + 4 * half, at_sb = lds0 + AT_SCALES_B + 16u * (wave_b + lane_b) + 4 * half;
  const auto read = [&](u32 buffer, u32 t, u32 i) {
    if (i < TM) fa[t & 1][i] = *mx_lds<u32x4_t>(at_a[t] + (buffer * RA * 128u + 4096u * i));
    else fb[t & 1][i - TM] = *mx_lds<u32x4_t>(at_b[t] + (buffer * RB * 128u + 4096u * (i - TM)));
  };
  const auto read_scales = [&](u32 plane, u32 u, u32 i) {
    if (i < TM) sa[u][i] = *mx_lds<u32>(at_sa + plane * (RA * 16u) + (8 * u + 512u * i));
    else sb[u][i - TM] = *mx_lds<u32>(at_sb + plane * (RB * 16u) + (8 * u + 512u * (i - TM)));
  };

  // The instructions of a step and what goes between them: in the first half the reads for the next step, and from the last step of a stage on, when its
  // place has been read for the last time, the requests for the stage after the next one: half of them in that step, half in the one behind it.  (A CU takes 64 bytes a
  // cycle: all of the four waves' requests in one step would hold the waves up for another one.)
  constexpr u32 SLOTS = TM * TN, READS = TM + TN, EARLY = LOADS / 2;
  aim();
#pragma unroll
  for (u32 i = 0; i < LOADS; ++i) ask(0, i);
  next_stage();
  ask_scales();
  put_scales(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (u32 i = 0; i < EARLY; ++i) ask(1, i);
#pragma unroll
  for (u32 i = 0; i < READS; ++i) read(0, 0, i), read_scales(0, 0, i);
  u32 plane = 0;                                        // of the four with scale bytes: the pair's
  for (u32 tile = tiles.first; tile < tiles.count; tile += tiles.step) {
    f32x16_t sum[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[i][j][r] = 0.0f;
    for (u32 pair = 0; pair < pairs; ++pair) {
      const u32 next_plane = (pair & 1u) == 0 && pair + 1 < pairs ? plane + 1u : (plane & 2u) ^ 2u;
      const bool fresh = (next_plane & 1u) == 0;        // the scale bytes of the next two pairs are asked for during this one
#pragma unroll
      for (u32 u = 0; u < 2; ++u) {
#pragma unroll
        for (u32 t = 0; t < 4; ++t) {
          if (t == 3) {
            if (u == 1 && fresh) put_scales(next_plane);
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
            for (u32 i = 0; i < READS; ++i) {
              if (i * SLOTS / (2 * READS) == slot) read(t < 3 ? u : u ^ 1, (t + 1) & 3u, i);
              if (t == 3 && SLOTS / 2 + i * SLOTS / (2 * READS) == slot) read_scales(u ? next_plane : plane, u ^ 1, i);
            }
            const u32 i = slot / TN, j = slot % TN;
            const i32x8_t b = mx_operand(fb[t & 1][j]), x = mx_operand(fa[t & 1][i]);
            const int scale_b = int(sb[u][j]), scale_a = int(sa[u][i]);
            if (t == 0) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 0, scale_b, 0, scale_a);
            if (t == 1) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 1, scale_b, 1, scale_a);
            if (t == 2) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 2, scale_b, 2, scale_a);
            if (t == 3) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 3, scale_b, 3, scale_a);
            mx_hold<TM * TN>(sum[i][j]);                 // (holds the instruction at its place)
            __builtin_amdgcn_sched_barrier(0);
          }
          if (t == 0) next_stage();
          if (u == 0 && t == 0) {
            next_pair();
            if (fresh) ask_scales();
          }
        }
      }
      plane = next_plane;
    }
    u32 down, across;
    tiles.place(tile, down, across);
    const u64 row0 = u64(down) * RA + wave_a, col0 = u64(across) * RB + wave_b;
    const bool whole = row0 + 32 * TM <= a.m && col0 + 32 * TN <= a.n, more = a.bias || a.add;
    if (whole && !more) mx_write_tile<TM, TN, TYPE, true, false>(a, row0, col0, lane, sum);
    else if (whole) mx_write_tile<TM, TN, TYPE, true, true>(a, row0, col0, lane, sum);
    else if (!more) mx_write_tile<TM, TN, TYPE, false, false>(a, row0, col0, lane, sum);
    else mx_write_tile<TM, TN, TYPE, false, true>(a, row0, col0, lane, sum);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the last requests, too, before the workgroup's LDS is given to another one)
}

// ---- Products of any size: a wave makes 16 x 16 results.  The rows of b go in as the instruction's first operand, so that a lane ends with four
// neighbouring results of one row.  For rows further apart than a buffer of a tile's rows reaches, and for no products at all (k = 0, where there may still be a bias
// to write): every wave reads its operands from memory, 28 times what the tiles take at 8192 x 8192 x 8192.
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
  float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  if (row < a.m && col0 + 4 * part < a.n) mx_finish(a, row, col0 + 4 * part, v);
}

}  // namespace zc
