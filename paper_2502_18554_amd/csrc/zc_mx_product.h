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
// other in LDS, their eight 16-byte blocks exchanged by the row's number, so that the eight lanes that read LDS at a time find eight different
// places of the banks.  Scale bytes come by two stages (16 bytes of a row) through registers.
//
// An instruction multiplies two blocks of 32 rows with 32 columns: lanes 0 .. 31 bring one block each, lanes 32 .. 63 the other.  Which two blocks of the
// stage these are is free: it is blocks t and 4 + t, so that a lane's scale bytes of the stage are the four bytes of one word, of which
// the instruction takes the one that it is told.
//
// Results go through LDS once more, 32 rows at a time, so that whole lines are written.
constexpr u32 kStageBlocks = 8;
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) u32 MxLdsWord;

__host__ __device__ constexpr u32 mx_tile_rows(int t) { return 64u * u32(t); }

// Tiles in the order of the workgroups: every XCD has a run of neighbouring tiles (workgroups go round the eight XCDs), which goes down strips of eight rows of tiles.
__device__ inline void mx_tile_of(u32 group, u32 tiles_down, u32 tiles_across, u32& down, u32& across) {
  const u32 tiles = tiles_down * tiles_across, xcd = group & 7u, share = tiles >> 3, more = tiles & 7u;
  const u32 t = xcd * share + min(xcd, more) + (group >> 3);
  const u32 strip = t / (8u * tiles_across), rest = t - strip * 8u * tiles_across, high = min(8u, tiles_down - 8u * strip);
  across = rest / high;
  down = 8u * strip + rest - across * high;
}

// Rows of a tile, `used` bytes each, as a buffer: what lies behind the last one reads as zeros.
__device__ inline __amdgpu_buffer_rsrc_t mx_rows(const u8* base, u64 first, u64 rows, u64 stride, u32 most, u32 used) {
  const u64 bytes = (min(rows - first, u64(most)) - 1) * stride + used;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<u8*>(base) + first * stride, 0, u32(bytes), 0x00027000);
}
constexpr u64 kMostTileStride = u64(1) << 23;       // (256 rows are less than 2^32 bytes)

// 16 bytes a lane to LDS, at `to` and on.  (Written out: of its own loads to LDS the compiler thinks that any read of LDS may have to wait for them.)
__device__ inline void mx_load_to_lds(__amdgpu_buffer_rsrc_t from, u32 to, u32 lane_offset, u32 offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(lane_offset), "s"(from), "s"(offset) : "memory");
}

template <typename T>
__device__ inline const __attribute__((address_space(3))) T* mx_lds(u32 at) {
  return reinterpret_cast<const __attribute__((address_space(3))) T*>(at);
}

template <int TM, int TN>
__global__ __launch_bounds__(256, TM * TN > 4 ? 1 : 2) void mx_tile_kernel(MxProductArgs a, u32 tiles_down, u32 tiles_across) {
  constexpr u32 RA = mx_tile_rows(TM), RB = mx_tile_rows(TN), ROWS = RA + RB, LOADS = ROWS / 32;
  constexpr u32 SCALE_ROWS = (ROWS + 255) / 256;
  // In LDS: two stages of a's rows, two of b's, the scale bytes of two pairs of stages of a's rows, of b's.
  constexpr u32 AT_B = 2 * RA * 128, AT_SCALES_A = 2 * ROWS * 128, AT_SCALES_B = AT_SCALES_A + 2 * RA * 16, LDS_BYTES = AT_SCALES_B + 2 * RB * 16;
  __shared__ u32x4_t memory[LDS_BYTES / 16];
  const u32 tid = threadIdx.x, lane = tid & 63u, wave = u32(__builtin_amdgcn_readfirstlane(int(tid >> 6)));
  const u32 half = lane >> 5, in32 = lane & 31u;
  u32 down, across;
  mx_tile_of(blockIdx.x, tiles_down, tiles_across, down, across);
  down = u32(__builtin_amdgcn_readfirstlane(int(down)));
  across = u32(__builtin_amdgcn_readfirstlane(int(across)));
  const u64 row0 = u64(down) * RA, col0 = u64(across) * RB;
  const u32 row_bytes = kMxBytes * a.blocks, scale_bytes = (a.blocks + 3u) & ~3u;
  const auto rows_a = mx_rows(a.a, row0, a.m, a.a_stride, RA, row_bytes), rows_b = mx_rows(a.b, col0, a.n, a.b_stride, RB, row_bytes);
  const auto scales_a = mx_rows(a.a_scales, row0, a.m, a.a_scales_stride, RA, scale_bytes), scales_b = mx_rows(a.b_scales, col0, a.n, a.b_scales_stride, RB, scale_bytes);

  // A thread's loads: 32 rows apart, so that the exchange of blocks is the same for all of them.
  const u32 my_row = tid >> 3, my_block = (tid ^ my_row) & 7u;
  u32 from_a[RA / 32], from_b[RB / 32];
#pragma unroll
  for (u32 i = 0; i < RA / 32; ++i) from_a[i] = (my_row + 32 * i) * u32(a.a_stride) + 16u * my_block;
#pragma unroll
  for (u32 i = 0; i < RB / 32; ++i) from_b[i] = (my_row + 32 * i) * u32(a.b_stride) + 16u * my_block;
  const u32 lds0 = u32(reinterpret_cast<uintptr_t>((MxLdsWord*)&memory[0]));
  // (Beyond the last stage there is nothing or the next row's; nobody looks at it.)
  const auto ask = [&](u32 stage, u32 buffer, u32 i) {
    const u32 to = lds0 + wave * 1024u;
    if (i < RA / 32) mx_load_to_lds(rows_a, to + buffer * (RA * 128u) + 4096u * i, from_a[i], 128u * stage);
    else mx_load_to_lds(rows_b, to + AT_B + buffer * (RB * 128u) + 4096u * (i - RA / 32), from_b[i - RA / 32], 128u * stage);
  };
  u32x4_t held[SCALE_ROWS];
  const auto ask_scales = [&](u32 pair) {               // 16 scale bytes of a row, those behind the last block as zeros
#pragma unroll
    for (u32 i = 0; i < SCALE_ROWS; ++i) {
      const u32 r = tid + 256 * i;
      const bool of_a = 64 * wave + 256 * i < RA;
      const u32 at = of_a ? r * u32(a.a_scales_stride) : (r - RA) * u32(a.b_scales_stride);
      u32x4_t w = {0, 0, 0, 0};
      if (64 * wave + 256 * i < ROWS) {
        if (16 * pair + 16 <= a.blocks) {
          w = of_a ? __builtin_amdgcn_raw_buffer_load_b128(scales_a, at, 16 * pair, 0) : __builtin_amdgcn_raw_buffer_load_b128(scales_b, at, 16 * pair, 0);
        } else {
#pragma unroll
          for (u32 j = 0; j < 4; ++j) {
            const u32 first = 16 * pair + 4 * j;
            if (first >= a.blocks) continue;
            w[j] = of_a ? __builtin_amdgcn_raw_buffer_load_b32(scales_a, at, first, 0) : __builtin_amdgcn_raw_buffer_load_b32(scales_b, at, first, 0);
            if (first + 4 > a.blocks) w[j] &= (1u << (8 * (a.blocks - first))) - 1u;
          }
        }
      }
      held[i] = w;
    }
  };
  const auto put_scales = [&](u32 pair) {
#pragma unroll
    for (u32 i = 0; i < SCALE_ROWS; ++i)
      if (64 * wave + 256 * i < ROWS) {
        const bool of_a = 64 * wave + 256 * i < RA;
        memory[(of_a ? AT_SCALES_A : AT_SCALES_B - RA * 16) / 16 + (pair & 1u) * (of_a ? RA : RB) + tid + 256 * i] = held[i];
      }
  };

  const u32 wave_a = (wave >> 1) * 32u * TM, wave_b = (wave & 1u) * 32u * TN;
  u32x4_t fa[2][TM], fb[2][TN];                         // of this step and of the next one
  u32 sa[2][TM], sb[2][TN];                             // of this stage and of the next one
  u32 at_a[4], at_b[4];                                 // where a lane's block of step t is, in the first stage's place
#pragma unroll
  for (u32 t = 0; t < 4; ++t) {
    const u32 place = in32 * 128u + 16u * ((4 * half + t) ^ (in32 & 7u));
    at_a[t] = lds0 + wave_a * 128u + place;
    at_b[t] = lds0 + AT_B + wave_b * 128u + place;
  }
  const u32 at_sa = lds0 + AT_SCALES_A + 16u * (wave_a + in32) + 4 * half, at_sb = lds0 + AT_SCALES_B + 16u * (wave_b + in32) + 4 * half;
  const auto read = [&](u32 buffer, u32 t, u32 i) {
    if (i < TM) fa[t & 1][i] = *mx_lds<u32x4_t>(at_a[t] + (buffer * RA * 128u + 4096u * i));
    else fb[t & 1][i - TM] = *mx_lds<u32x4_t>(at_b[t] + (buffer * RB * 128u + 4096u * (i - TM)));
  };
  const auto read_scales = [&](u32 pair, u32 u, u32 i) {
    if (i < TM) sa[u][i] = *mx_lds<u32>(at_sa + (pair & 1u) * (RA * 16u) + (8 * u + 512u * i));
    else sb[u][i - TM] = *mx_lds<u32>(at_sb + (pair & 1u) * (RB * 16u) + (8 * u + 512u * (i - TM)));
  };

  f32x16_t sum[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[i][j][r] = 0.0f;

  // The instructions of a step and what goes between them: in the first half the reads for the next step, in the last step of a stage also
  // the requests for the stage after the next one, whose place has just been read for the last time.
  constexpr u32 SLOTS = TM * TN, READS = TM + TN;
  const u32 pairs = (a.blocks + 2 * kStageBlocks - 1) / (2 * kStageBlocks);
#pragma unroll
  for (u32 i = 0; i < LOADS; ++i) ask(0, 0, i);
  ask_scales(0);
  put_scales(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (u32 i = 0; i < LOADS; ++i) ask(1, 1, i);
#pragma unroll
  for (u32 i = 0; i < READS; ++i) read(0, 0, i), read_scales(0, 0, i);
  for (u32 pair = 0; pair < pairs; ++pair) {
    if (16 * (pair + 1) < a.blocks) ask_scales(pair + 1);
#pragma unroll
    for (u32 u = 0; u < 2; ++u) {
#pragma unroll
      for (u32 t = 0; t < 4; ++t) {
        if (t == 3) {
          if (u == 1) put_scales(pair + 1);
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          __syncthreads();
        }
#pragma unroll
        for (u32 slot = 0; slot < SLOTS; ++slot) {
          if (t == 3) {
#pragma unroll
            for (u32 i = 0; i < LOADS; ++i)
              if (i * SLOTS / LOADS == slot) ask(2 * pair + u + 2, u, i);
          }
#pragma unroll
          for (u32 i = 0; i < READS; ++i) {
            if (i * SLOTS / (2 * READS) == slot) read(t < 3 ? u : u ^ 1, (t + 1) & 3u, i);
            if (t == 3 && SLOTS / 2 + i * SLOTS / (2 * READS) == slot) read_scales(u ? pair + 1 : pair, u ^ 1, i);
          }
          const u32 i = slot / TN, j = slot % TN;
          const i32x8_t b = mx_operand(fb[t & 1][j]), x = mx_operand(fa[t & 1][i]);
          const int scale_b = int(sb[u][j]), scale_a = int(sa[u][i]);
          if (t == 0) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 0, scale_b, 0, scale_a);
          if (t == 1) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 1, scale_b, 1, scale_a);
          if (t == 2) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 2, scale_b, 2, scale_a);
          if (t == 3) sum[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, x, sum[i][j], kMxFp4, kMxFp4, 3, scale_b, 3, scale_a);
          asm volatile("" : "+a"(sum[i][j]));            // (holds the instruction at its place)
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the last requests, too, before their place is used for something else)
  // Lane l has of 32 x 32 results those of row l % 32 and columns 8 q + 4 (l / 32) + 0 .. 3.  (A row's 16 bytes more spread the rows over the banks.)
  constexpr u32 COLS = 32 * TN, PITCH = COLS / 4 + 1, LANES = COLS / 4;
  static_assert(AT_SCALES_A >= 4 * 32 * PITCH * 16);
  __syncthreads();
  f32x4_t* const out = reinterpret_cast<f32x4_t*>(&memory[0]) + wave * 32u * PITCH;
  const u64 col = col0 + wave_b + 4 * (lane % LANES);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        out[in32 * PITCH + 8 * j + 2 * q + half] = f32x4_t{sum[i][j][4 * q], sum[i][j][4 * q + 1], sum[i][j][4 * q + 2], sum[i][j][4 * q + 3]};
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (u32 r = lane / LANES; r < 32; r += 64 / LANES) {
      const f32x4_t w = out[r * PITCH + lane % LANES];
      float v[4] = {w[0], w[1], w[2], w[3]};
      const u64 row = row0 + wave_a + 32 * i + r;
      if (row < a.m && col < a.n) mx_finish(a, row, col, v);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- Products of any size: a wave makes 16 x 16 results.  The rows of b go in as the instruction's first operand, so that a lane ends with four
// neighbouring results of one row.
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
