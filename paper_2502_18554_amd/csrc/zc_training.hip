// C ABI of the other calls of a training step: layer norm, embedding, and the optimiser's step for matrices.  Argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "zc_embedding.h"
#include "zc_muon.h"
#include "zc_norm.h"

using namespace zc;

namespace {

bool aligned(const void* p, u64 to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool type_valid(int type) { return type == ZC_F32 || type == ZC_BF16 || type == ZC_F16; }
int launched() { return hipGetLastError() == hipSuccess ? ZC_OK : ZC_ERR_HIP; }
bool matrix_valid(const void* p, int type, u64 rows, u64 cols, u64 stride) {
  return type_valid(type) && stride >= cols && stride <= (u64(1) << 32) && (rows == 0 || cols == 0 || (p && aligned(p, value_bytes(type))));
}
// A result that begins where an operand does has to be that matrix: anything else would overwrite what is still to be read.
bool same_or_apart(const void* out, int out_type, u64 out_stride, const void* in, int in_type, u64 in_stride) { return out != in || (out_type == in_type && out_stride == in_stride); }

// ---- Layer norm

constexpr u64 kMostNormCols = u64(1) << 27;
constexpr u64 kMostHeldCols = 16384;                     // of a row that stays in registers
constexpr u32 kLongGroups = 128;
bool norm_sizes_valid(u64 rows, u64 cols) { return rows <= 0x7fffffffu && cols <= kMostNormCols; }

u32 at_most(u64 wanted, u32 most) { return u32(wanted < most ? wanted : most); }

// Calls `launch` with the lanes of a row and their pieces of eight values, as few as hold it.
template <typename F>
void by_cols(u64 cols, const F& launch) {
  if (cols <= 128) launch(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  else if (cols <= 512) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  else if (cols <= 1024) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  else if (cols <= 2048) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
  else if (cols <= 4096) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  else if (cols <= 8192) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
  else launch(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
}
u32 norm_backward_groups(u64 rows, u64 cols) {
  if (cols > kMostHeldCols) return at_most(rows, kLongGroups);
  const u64 at_once = cols <= 128 ? 16 : cols <= 2048 ? 4 : 1;
  return at_most((rows + at_once - 1) / at_once, cols > 8192 ? 256 : 512);
}
u64 norm_workspace(u64 rows, u64 cols) { return u64(norm_backward_groups(rows, cols)) * 2 * cols * 4 + (cols > kMostHeldCols ? 8 * rows : 0); }

// ---- Embedding

constexpr u64 kMostTableRows = u64(1) << 29, kMostTableCols = u64(1) << 23;
bool table_valid(u64 rows, u64 cols, u64 n, int token_bits) { return rows <= kMostTableRows && cols <= kMostTableCols && n <= 0x7fffffffu && (token_bits == 32 || token_bits == 64); }

struct TokenPlan {
  u32 groups_log2, per, chunk_log2, pieces;
  u64 at_row, at_first, at_partial, bytes;               // in the workspace, whose beginning has the places
  TokenPlan(u64 n, u64 rows, u64 cols) {
    groups_log2 = 8;
    while ((kTokenRows << u64(groups_log2)) < rows) ++groups_log2;
    per = u32((rows + (u64(1) << groups_log2) - 1) >> groups_log2);
    chunk_log2 = 3;                                      // pieces enough for four workgroups on every CU, of 64 places at most where that is no more than 2^20 pieces
    while ((n >> chunk_log2) >= (chunk_log2 < 6 ? 2048u : 1u << 20)) ++chunk_log2;
    pieces = u32((n + (u64(1) << chunk_log2) - 1) >> chunk_log2);
    at_row = pad16(4 * n);
    at_first = at_row + pad16(4 * n);
    at_partial = at_first + pad16(4 * ((u64(per) << groups_log2) + 1));
    bytes = at_partial + u64(pieces) * 2 * cols * 4;
  }
};

template <int BITS>
void launch_embedding(const EmbeddingArgs& a, dim3 grid, hipStream_t stream) {
  const bool in = a.table_type == ZC_F32, out = a.out_type == ZC_F32;
  if (in && out) hipLaunchKernelGGL((embedding_kernel<BITS, true, true>), grid, dim3(256), 0, stream, a);
  else if (in) hipLaunchKernelGGL((embedding_kernel<BITS, true, false>), grid, dim3(256), 0, stream, a);
  else if (out) hipLaunchKernelGGL((embedding_kernel<BITS, false, true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((embedding_kernel<BITS, false, false>), grid, dim3(256), 0, stream, a);
}

// ---- The optimiser's step for matrices

constexpr u64 kMostMuonSide = u64(1) << 20;
constexpr int kMostIterations = 100;

bool muon_sizes_valid(int k, const size_t* rows, const size_t* cols) {
  if (k < 0 || (k > 0 && (!rows || !cols))) return false;
  for (int i = 0; i < k; ++i)
    if (rows[i] > kMostMuonSide || cols[i] > kMostMuonSide) return false;
  return true;
}
u64 muon_padded(u64 values) { return (values + 31) / 32 * 32; }
u64 pad256(u64 n) { return (n + 255) / 256 * 256; }
u32 smaller(u64 a, u64 b) { return u32(a < b ? a : b); }
u32 larger(u64 a, u64 b) { return u32(a < b ? b : a); }

// Matrices go through the launches together, up to kMuonTensors of them and up to kMuonTogether bytes of workspace (more only where one alone needs them).
constexpr u64 kMuonTogether = u64(8) << 30;
struct MuonGroup {
  int begin, end;
  u64 bytes;
};
MuonGroup muon_group(int begin, int k, const size_t* rows, const size_t* cols, u32 planes) {
  MuonGroup g{begin, begin, 0};
  int count = 0;
  for (; g.end < k; ++g.end) {
    const u64 r = rows[g.end], c = cols[g.end];
    if (r == 0 || c == 0) continue;
    const u64 more = pad256(MuonParts(smaller(r, c), larger(r, c), planes).bytes);
    if (count == kMuonTensors || (count && g.bytes + more > kMuonTogether)) break;
    g.bytes += more;
    ++count;
  }
  g.bytes += u64(count) * kMuonPartials * 8;
  return g;
}
u64 muon_workspace(int k, const size_t* rows, const size_t* cols, u32 planes) {
  u64 most = 0;
  for (int i = 0; i < k;) {
    const MuonGroup g = muon_group(i, k, rows, cols, planes);
    if (g.bytes > most) most = g.bytes;
    i = g.end;
  }
  return most;
}

// What lr is multiplied by for a matrix.
double muon_factor(u64 r, u64 c, unsigned flags) {
  return flags & ZC_MUON_MATCH_RMS ? 0.2 * std::sqrt(double(larger(r, c))) : r > c ? std::sqrt(double(r) / double(c)) : 1.0;
}

// Whether no two of a call's results, the momentum among them, have a byte in common: launches take many matrices together, so that one would be lost.  Not known (no memory to sort them in): -1.
struct MuonResult {
  uintptr_t begin, end;
};
int results_apart(int k, const size_t* rows, const size_t* cols, void* const* params, int param_type, void* const* copies, int copy_type, const void* state, u64 state_bytes) {
  const std::unique_ptr<MuonResult[]> all(new (std::nothrow) MuonResult[2 * size_t(k) + 1]);
  if (!all) return -1;
  size_t n = 0;
  const auto add = [&](const void* p, u64 bytes) {
    if (p && bytes) all[n++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes};
  };
  add(state, state_bytes);
  for (int i = 0; i < k; ++i) {
    add(params[i], u64(rows[i]) * cols[i] * value_bytes(param_type));
    if (copies) add(copies[i], u64(rows[i]) * cols[i] * value_bytes(copy_type));
  }
  std::sort(all.get(), all.get() + n, [](const MuonResult& a, const MuonResult& b) { return a.begin < b.begin; });
  for (size_t i = 1; i < n; ++i)
    if (all[i].begin < all[i - 1].end) return 0;
  return 1;
}

u64 muon_tiles(const MuonTensor& t, int mode, u64 high, u64 wide) {
  const u64 down = (t.r + high - 1) / high, across = (t.c + wide - 1) / wide;
  return muon_symmetric(mode) ? down * (down + 1) / 2 : down * across;
}
template <int MODE>
void count_muon_tiles(MuonArgs& a, u64 high, u64 wide) {
  a.count = 0;
  for (u32 i = 0; i < a.tensors; ++i) {
    a.first[i] = a.count;
    a.count += u32(muon_tiles(a.t[i], MODE, high, wide));
  }
  if (a.each) a.each = a.count / a.tensors;
}
template <int TM, int TN, int S, int MODE>
void launch_muon_tiles(MuonArgs& a, hipStream_t stream) {
  count_muon_tiles<MODE>(a, 64 * TM, 64 * TN);
  const u32 at_once = 256 * muon_groups(TM, TN, S);
  hipLaunchKernelGGL((muon_product_kernel<TM, TN, S, MODE>), dim3(a.count < at_once ? a.count : at_once), dim3(256), 0, stream, a);
}
// The kind of tile that takes the least time, in us, by what a turn of all CUs takes: a tile's begin and end, and its stages of 64 values.  The constants were measured on single products, over and over on
// the same operands; in steps they are low by some tenth, all alike.  What the kinds take in steps, us, the one that the rule picks with a *:
//   3 of 333 x 1531, two parts    X X^T by 32*, 64, 128, 192  10.4, 24.4, 38.8, 63.8    A A by the same  6.1*, 12.1, 19.7, 33.4    B X by 32, 64, 64 x 128*, 128, 192  21.7, 16.6, 17.2, 20.8, 32.6
//   24 of 256 x 512               X X^T by 32, 64*, 128  8.2, 6.9, 10.2    A A  7.6, 6.0*, 9.0    B X by 32, 64, 64 x 128*, 128, 128 x 256  18.8, 10.4, 10.5, 10.3, 14.1
//   6 of 1024 x 4096, two parts   X X^T by 64, 128*, 192, 256  163, 114, 161, 252    A A  53, 40*, 62    B X by 64 x 128, 128, 128 x 256*, 192, 256  261, 220, 193, 236, 210
//   4096 x 8192                   X X^T by 128, 192*, 256  201, 147, 184    A A by 64, 128, 192*  149, 111, 86    B X by 128, 128 x 256, 192, 256*  298, 284, 291, 255
// A stage takes longer the more CUs work: X X^T of matrices of 384 x 8192 (128 stages) by 192 takes 96, 111, 125, 131 and 132 us with 18, 60, 120, 159 and 192 tiles, of 512 x 8192 by 256 152, 181, 195,
// 202 and 214; the rule has one step of it, at 160.  By 32 it is whether a CU has one workgroup or two (320 x 4096, 64 stages: 9.3, 9.4, 15.0, 20.0 and 26.8 us with 110, 220, 495, 550 and 990 tiles).
struct MuonKind {
  u64 high, wide;
};
constexpr MuonKind kMuonKinds[] = {{32, 32}, {64, 64}, {128, 128}, {192, 192}, {256, 256}, {64, 128}, {128, 256}};
constexpr int kMuonKindsOf = 7;
template <int MODE>
void launch_muon_product(MuonArgs& a, hipStream_t stream) {
  double tiles[kMuonKindsOf] = {}, along[kMuonKindsOf] = {};
  for (u32 i = 0; i < a.tensors; ++i) {
    const double stages = double(muon_along(MODE == kMuonGram ? a.t[i].c : a.t[i].r)) / 64 * (a.planes > 1 ? 3 : 1);
    for (int t = 0; t < kMuonKindsOf; ++t) {
      const double of_this = double(muon_tiles(a.t[i], MODE, kMuonKinds[t].high, kMuonKinds[t].wide));
      tiles[t] += of_this;
      along[t] += of_this * stages;
    }
  }
  const auto stages = [&](int t) { return along[t] / tiles[t]; };
  const auto turns = [&](int t, double at_once) { return std::ceil(tiles[t] / at_once); };
  const double cost[kMuonKindsOf] = {2 + turns(0, 512) * (2.3 + (tiles[0] <= 256 ? 0.075 : 0.16) * stages(0)),
                                     3 + (tiles[1] <= 256 ? 2 + 0.25 * stages(1) : turns(1, 512) * (3 + 0.5 * stages(1))),
                                     tiles[2] <= 256 ? 8 + 0.46 * stages(2) : 4 + turns(2, 512) * (12 + 1.1 * stages(2)),
                                     turns(3, 256) * (12 + (tiles[3] <= 160 ? 0.68 : 0.83) * stages(3)),
                                     turns(4, 256) * (22 + (tiles[4] <= 160 ? 1.1 : 1.4) * stages(4)),
                                     tiles[5] <= 256 ? 5 + 0.47 * stages(5) : 4 + turns(5, 512) * (2.5 + 0.7 * stages(5)),
                                     turns(6, 256) * (12 + 0.87 * stages(6))};
  // (Tiles of symmetric results are squares; those of 256 have no registers left for what the second product reads as well.)
  constexpr int KINDS = MODE == kMuonPoly ? 4 : MODE == kMuonGram ? 5 : kMuonKindsOf;
  int best = 0;
  for (int t = 1; t < KINDS; ++t)
    if (cost[t] < cost[best]) best = t;
  if (best == 0) {
    count_muon_tiles<MODE>(a, 32, 32);
    hipLaunchKernelGGL((muon_small_kernel<MODE>), dim3(a.count), dim3(256), 0, stream, a);
  } else if (best == 1) {
    launch_muon_tiles<1, 1, 4, MODE>(a, stream);
  } else if (best == 2) {
    // Where every CU has one tile at most, a third stage lies in LDS instead of a second workgroup's (X X^T of six matrices of 1024 x 4096 in two parts, 216 tiles, 114 us, 139 by two;
    // of 4096 x 8192, 528 tiles, 202 and 192).
    if (tiles[2] <= 256) launch_muon_tiles<2, 2, 3, MODE>(a, stream);
    else launch_muon_tiles<2, 2, 2, MODE>(a, stream);
  } else if (best == 3) {
    launch_muon_tiles<3, 3, 3, MODE>(a, stream);
  } else if constexpr (KINDS > 4) {
    if (best == 4) launch_muon_tiles<4, 4, 2, MODE>(a, stream);
    else if constexpr (KINDS > 5) {
      if (best == 5) launch_muon_tiles<1, 2, 3, MODE>(a, stream);
      else launch_muon_tiles<2, 4, 3, MODE>(a, stream);
    }
  }
}

// A launch of `groups(i)` workgroups for matrix i.
template <typename K, typename F>
void launch_muon(K kernel, MuonArgs& a, const F& groups, hipStream_t stream) {
  a.count = 0;
  for (u32 i = 0; i < a.tensors; ++i) {
    a.first[i] = a.count;
    a.count += u32(groups(a.t[i]));
  }
  if (a.each) a.each = a.count / a.tensors;
  if (a.count) hipLaunchKernelGGL(kernel, dim3(a.count), dim3(256), 0, stream, a);
}

}  // namespace

extern "C" {

int zc_layer_norm(const void* d_x, int x_type, size_t rows, size_t cols, size_t x_stride, const void* d_w, const void* d_b, int w_type, double eps,
                  void* d_out, int out_type, size_t out_stride, float* d_stats, void* hip_stream) {
  if (!norm_sizes_valid(rows, cols) || !matrix_valid(d_x, x_type, rows, cols, x_stride) || !matrix_valid(d_out, out_type, rows, cols, out_stride)) return ZC_ERR_ARG;
  if (!type_valid(w_type) || !aligned(d_w, value_bytes(w_type)) || !aligned(d_b, value_bytes(w_type)) || !aligned(d_stats, 4)) return ZC_ERR_ARG;
  if (!(std::isfinite(float(eps)) && eps >= 0) || !same_or_apart(d_out, out_type, out_stride, d_x, x_type, x_stride)) return ZC_ERR_ARG;
  if (rows == 0 || cols == 0) return ZC_OK;
  const NormArgs a{d_x, d_w, d_b, d_out, d_stats, rows, cols, x_stride, out_stride, float(eps), x_type, w_type, out_type};
  const auto stream = static_cast<hipStream_t>(hip_stream);
  if (cols > kMostHeldCols) {
    hipLaunchKernelGGL(norm_long_kernel, dim3(at_most(rows, 1 << 20)), dim3(1024), 0, stream, a);
    return launched();
  }
  by_cols(cols, [&](auto lanes, auto pieces) {
    constexpr int T = decltype(lanes)::value, P = decltype(pieces)::value, W = norm_threads<T>();
    const dim3 grid(at_most((rows + W / T - 1) / (W / T), W == 256 ? 2048 : 256));
    if (x_type == ZC_F32) hipLaunchKernelGGL((norm_kernel<T, P, true>), grid, dim3(W), 0, stream, a);
    else hipLaunchKernelGGL((norm_kernel<T, P, false>), grid, dim3(W), 0, stream, a);
  });
  return launched();
}

size_t zc_layer_norm_workspace_bytes(size_t rows, size_t cols) { return norm_sizes_valid(rows, cols) ? size_t(pad16(norm_workspace(rows, cols))) : 0; }

int zc_layer_norm_backward(const void* d_dy, int dy_type, size_t dy_stride, const void* d_x, int x_type, size_t x_stride, const float* d_stats, const void* d_w,
                           int w_type, size_t rows, size_t cols, void* d_dx, int dx_type, size_t dx_stride, void* d_dw, void* d_db, int dw_type, unsigned flags,
                           void* d_ws, size_t ws_bytes, void* hip_stream) {
  if (!norm_sizes_valid(rows, cols) || !matrix_valid(d_dy, dy_type, rows, cols, dy_stride) || !matrix_valid(d_x, x_type, rows, cols, x_stride)) return ZC_ERR_ARG;
  if (!type_valid(w_type) || !type_valid(dw_type) || !type_valid(dx_type) || (flags & ~(ZC_ADD | ZC_ADD_WEIGHTS))) return ZC_ERR_ARG;
  if (!aligned(d_w, value_bytes(w_type)) || !aligned(d_dw, value_bytes(dw_type)) || !aligned(d_db, value_bytes(dw_type)) || !aligned(d_stats, 4) || !aligned(d_ws, 16)) return ZC_ERR_ARG;
  if (d_dx && (!matrix_valid(d_dx, dx_type, rows, cols, dx_stride) || !same_or_apart(d_dx, dx_type, dx_stride, d_dy, dy_type, dy_stride) ||
               !same_or_apart(d_dx, dx_type, dx_stride, d_x, x_type, x_stride)))
    return ZC_ERR_ARG;
  if (d_dw && d_dw == d_db) return ZC_ERR_ARG;
  if ((rows && cols && !d_stats) || ws_bytes < norm_workspace(rows, cols) || (rows && cols && !d_ws)) return ZC_ERR_ARG;
  const bool sums = d_dw || d_db;
  if (cols == 0 || (!sums && (rows == 0 || !d_dx))) return ZC_OK;
  const auto stream = static_cast<hipStream_t>(hip_stream);
  const u32 groups = norm_backward_groups(rows, cols);
  float* const partial = static_cast<float*>(d_ws);
  NormBackwardArgs a{d_dy, d_x, d_stats, d_w, d_dx, sums ? partial : nullptr, partial + u64(groups) * 2 * cols, rows, cols, dy_stride, x_stride, dx_stride,
                     dy_type, x_type, w_type, dx_type, flags & ZC_ADD ? 1u : 0u};
  if (rows) {
    if (cols > kMostHeldCols) {
      hipLaunchKernelGGL(norm_long_sums_kernel, dim3(at_most(rows, 1 << 20)), dim3(1024), 0, stream, a);
      hipLaunchKernelGGL(norm_long_backward_kernel, dim3(u32((cols + 2047) / 2048), groups), dim3(256), 0, stream, a);
    } else {
      by_cols(cols, [&](auto lanes, auto pieces) {
        constexpr int T = decltype(lanes)::value, P = decltype(pieces)::value, W = norm_threads<T>();
        const bool x = x_type == ZC_F32, dy = dy_type == ZC_F32;
        if (x && dy) hipLaunchKernelGGL((norm_backward_kernel<T, P, true, true>), dim3(groups), dim3(W), 0, stream, a);
        else if (x) hipLaunchKernelGGL((norm_backward_kernel<T, P, true, false>), dim3(groups), dim3(W), 0, stream, a);
        else if (dy) hipLaunchKernelGGL((norm_backward_kernel<T, P, false, true>), dim3(groups), dim3(W), 0, stream, a);
        else hipLaunchKernelGGL((norm_backward_kernel<T, P, false, false>), dim3(groups), dim3(W), 0, stream, a);
      });
    }
  }
  if (sums) {
    const NormColumnsArgs c{partial, {d_dw, d_db}, cols, rows ? groups : 0, dw_type, flags & ZC_ADD_WEIGHTS ? 1u : 0u};
    hipLaunchKernelGGL(norm_columns_kernel, dim3(u32((cols + 63) / 64), 2), dim3(1024), 0, stream, c);
  }
  return launched();
}

int zc_embedding(const void* d_table, int table_type, size_t table_rows, size_t cols, size_t table_stride, const void* d_tokens, int token_bits, size_t n, double scale,
                 void* d_out, int out_type, size_t out_stride, void* hip_stream) {
  if (!table_valid(table_rows, cols, n, token_bits) || !matrix_valid(d_table, table_type, table_rows, cols, table_stride) || !matrix_valid(d_out, out_type, n, cols, out_stride)) return ZC_ERR_ARG;
  if (!std::isfinite(float(scale)) || (n && !d_tokens) || !aligned(d_tokens, u64(token_bits / 8))) return ZC_ERR_ARG;
  if (n == 0 || cols == 0) return ZC_OK;
  EmbeddingArgs a{d_table, d_tokens, d_out, n, table_rows, cols, table_stride, out_stride, float(scale), table_type, out_type, 4};
  while (a.pieces_log2 < 8 && (u64(8) << a.pieces_log2) < cols) ++a.pieces_log2;
  const u64 at_once = u64(256) >> a.pieces_log2, across = (cols + (u64(8) << a.pieces_log2) - 1) / (u64(8) << a.pieces_log2);
  // As many workgroups as rows where they are few, of up to four rows each where the GPU is full.
  const u64 groups = (n + at_once - 1) / at_once, full = groups * across > 4096 ? (groups + kEmbeddingRows - 1) / kEmbeddingRows : groups;
  const dim3 grid(at_most(full, 1 << 20), at_most(across, 1 << 12));
  if (token_bits == 32) launch_embedding<32>(a, grid, static_cast<hipStream_t>(hip_stream));
  else launch_embedding<64>(a, grid, static_cast<hipStream_t>(hip_stream));
  return launched();
}

size_t zc_embedding_workspace_bytes(size_t n, size_t table_rows, size_t cols) { return table_valid(table_rows, cols, n, 32) ? size_t(TokenPlan(n, table_rows, cols).bytes) : 0; }

int zc_embedding_backward(const void* d_dy, int dy_type, size_t dy_stride, const void* d_tokens, int token_bits, size_t n, double scale, void* d_grad, int grad_type,
                          size_t table_rows, size_t cols, size_t grad_stride, unsigned flags, void* d_ws, size_t ws_bytes, void* hip_stream) {
  if (!table_valid(table_rows, cols, n, token_bits) || !matrix_valid(d_dy, dy_type, n, cols, dy_stride) || !matrix_valid(d_grad, grad_type, table_rows, cols, grad_stride)) return ZC_ERR_ARG;
  if (!std::isfinite(float(scale)) || (n && !d_tokens) || !aligned(d_tokens, u64(token_bits / 8)) || (flags & ~ZC_ADD) || !aligned(d_ws, 16)) return ZC_ERR_ARG;
  const TokenPlan plan(n, table_rows, cols);
  if (ws_bytes < plan.bytes || !d_ws) return ZC_ERR_ARG;
  const bool add = flags & ZC_ADD;
  if (table_rows == 0 || cols == 0 || (n == 0 && add)) return ZC_OK;
  const auto stream = static_cast<hipStream_t>(hip_stream);
  u8* const ws = static_cast<u8*>(d_ws);
  u32 *const place = reinterpret_cast<u32*>(ws), *const row = reinterpret_cast<u32*>(ws + plan.at_row), *const first = reinterpret_cast<u32*>(ws + plan.at_first);
  const TokenArgs t{d_tokens, place, row, first, n, table_rows, plan.groups_log2, plan.per};
  const dim3 groups(1u << plan.groups_log2);
  if (token_bits == 32) hipLaunchKernelGGL(token_order_kernel<32>, groups, dim3(64 * kTokenWaves), 0, stream, t);
  else hipLaunchKernelGGL(token_order_kernel<64>, groups, dim3(64 * kTokenWaves), 0, stream, t);
  const u32 slots = plan.per << plan.groups_log2, zeros = add ? 0 : (slots + kZeroRows - 1) / kZeroRows, groups_of_sums = plan.pieces + zeros;
  const EmbeddingBackwardArgs a{d_dy, place, row, first, reinterpret_cast<float*>(ws + plan.at_partial), d_grad, n, table_rows, cols, dy_stride, grad_stride, float(scale), dy_type, grad_type,
                                add ? 1u : 0u, plan.chunk_log2, slots, plan.per, plan.groups_log2, ((u64(zeros) << 32) + groups_of_sums - 1) / groups_of_sums};
  const dim3 grid(groups_of_sums, u32((cols + 2047) / 2048)), threads(cols > 1536 ? 256 : u32((cols + 511) / 512) * 64);
  if (dy_type == ZC_F32 && add) hipLaunchKernelGGL((embedding_sums_kernel<true, true>), grid, threads, 0, stream, a);
  else if (dy_type == ZC_F32) hipLaunchKernelGGL((embedding_sums_kernel<true, false>), grid, threads, 0, stream, a);
  else if (add) hipLaunchKernelGGL((embedding_sums_kernel<false, true>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((embedding_sums_kernel<false, false>), grid, threads, 0, stream, a);
  if (plan.pieces > 1) hipLaunchKernelGGL(embedding_joins_kernel, dim3((plan.pieces + kJoinPieces - 1) / kJoinPieces, u32((cols + 255) / 256)), dim3(64 * kJoinWaves), 0, stream, a);
  return launched();
}

size_t zc_muon_state_bytes(int k, const size_t* rows, const size_t* cols) {
  if (!muon_sizes_valid(k, rows, cols)) return 0;
  u64 values = 0;
  for (int i = 0; i < k; ++i) values += muon_padded(u64(rows[i]) * cols[i]);
  return size_t(4 * values);
}

size_t zc_muon_workspace_bytes(int k, const size_t* rows, const size_t* cols, unsigned flags) {
  return muon_sizes_valid(k, rows, cols) ? size_t(muon_workspace(k, rows, cols, flags & ZC_MUON_WIDE ? 2 : 1)) : 0;
}

int zc_muon(int k, const size_t* rows, const size_t* cols, void* const* d_params, int param_type, const void* const* d_grads, int grad_type, void* const* d_copies, int copy_type,
            void* d_state, size_t state_bytes, double lr, double momentum, double weight_decay, int iterations, unsigned flags, const float* d_grad_scale, void* d_ws,
            size_t ws_bytes, void* hip_stream) {
  if (!muon_sizes_valid(k, rows, cols) || (k > 0 && (!d_params || !d_grads)) || !type_valid(param_type) || !type_valid(grad_type) || (d_copies && !type_valid(copy_type))) return ZC_ERR_ARG;
  if (!(std::isfinite(lr) && lr >= 0 && momentum >= 0 && momentum < 1 && std::isfinite(weight_decay) && weight_decay >= 0) || iterations < 1 || iterations > kMostIterations) return ZC_ERR_ARG;
  if (!(float(momentum) < 1) || !std::isfinite(float(1 - lr * weight_decay))) return ZC_ERR_ARG;
  if ((flags & ~(ZC_MUON_NESTEROV | ZC_MUON_MATCH_RMS | ZC_MUON_WIDE)) || !aligned(d_grad_scale, 4) || !aligned(d_state, 16) || !aligned(d_ws, 256)) return ZC_ERR_ARG;
  const u32 planes = flags & ZC_MUON_WIDE ? 2 : 1;
  const u64 state = zc_muon_state_bytes(k, rows, cols), ws = muon_workspace(k, rows, cols, planes);
  if (state_bytes < state || ws_bytes < ws || (state && (!d_state || !d_ws))) return ZC_ERR_ARG;
  for (int i = 0; i < k; ++i) {
    if (rows[i] == 0 || cols[i] == 0) continue;
    if (!d_params[i] || !d_grads[i] || !aligned(d_params[i], value_bytes(param_type)) || !aligned(d_grads[i], value_bytes(grad_type))) return ZC_ERR_ARG;
    if (d_copies && !aligned(d_copies[i], value_bytes(copy_type))) return ZC_ERR_ARG;
    if (!std::isfinite(float(lr * muon_factor(rows[i], cols[i], flags)))) return ZC_ERR_ARG;
  }
  const int apart = results_apart(k, rows, cols, d_params, param_type, d_copies, copy_type, d_state, state);
  if (apart != 1) return apart ? ZC_ERR_HIP : ZC_ERR_ARG;
  const auto stream = static_cast<hipStream_t>(hip_stream);
  float* m = static_cast<float*>(d_state);
  for (int i = 0; i < k;) {
    const MuonGroup group = muon_group(i, k, rows, cols, planes);
    MuonArgs a = {};
    a.planes = planes;
    a.grad_scale = d_grad_scale;
    a.partial = static_cast<double*>(d_ws);
    a.keep = float(1 - lr * weight_decay);
    a.mu = float(momentum);
    a.rest = float(1 - momentum);
    a.nesterov = flags & ZC_MUON_NESTEROV ? 1 : 0;
    a.param_type = param_type, a.grad_type = grad_type, a.copy_type = copy_type;
    for (; i < group.end; ++i) {
      const u64 r = rows[i], c = cols[i];
      if (r && c) {
        MuonTensor& t = a.t[a.tensors];
        t.param = d_params[i];
        t.copy = d_copies ? d_copies[i] : nullptr;
        t.grad = d_grads[i];
        t.m = m;
        t.r = smaller(r, c), t.c = larger(r, c);
        t.step = float(lr * muon_factor(r, c, flags));
        t.turned = r > c;
        ++a.tensors;
      }
      m += muon_padded(r * c);
    }
    if (!a.tensors) continue;
    u8* at = static_cast<u8*>(d_ws) + u64(a.tensors) * kMuonPartials * 8;
    bool padded = false, alike = true;
    for (u32 j = 0; j < a.tensors; ++j) {
      a.t[j].at = at;
      at += pad256(MuonParts(a.t[j].r, a.t[j].c, planes).bytes);
      padded |= a.t[j].r % kMuonAlong != 0;
      alike &= a.t[j].r == a.t[0].r && a.t[j].c == a.t[0].c;
    }
    a.r = a.t[0].r, a.c = a.t[0].c;
    a.at = a.t[0].at;
    a.bytes = pad256(MuonParts(a.r, a.c, planes).bytes);
    a.each = alike ? 1 : 0;                              // (each launch puts its number here)
    launch_muon(muon_momentum_kernel, a, [](const MuonTensor& t) { return muon_partials(u64(t.r) * t.c); }, stream);
    launch_muon(muon_begin_kernel, a, [](const MuonTensor& t) { return muon_along(t.r) / 64 * (muon_along(t.c) / 64); }, stream);
    if (padded) launch_muon(muon_zeros_kernel, a, [](const MuonTensor& t) { return (t.c + 15) / 16; }, stream);
    for (int n = 0; n < iterations; ++n) {
      launch_muon_product<kMuonGram>(a, stream);
      launch_muon_product<kMuonPoly>(a, stream);
      if (n + 1 < iterations) launch_muon_product<kMuonUpdate>(a, stream);
      else if (param_type == ZC_F32) launch_muon_product<kMuonFinish + ZC_F32>(a, stream);
      else if (param_type == ZC_BF16) launch_muon_product<kMuonFinish + ZC_BF16>(a, stream);
      else launch_muon_product<kMuonFinish + ZC_F16>(a, stream);
      a.which ^= 1u;
    }
    const int st = launched();
    if (st != ZC_OK) return st;
  }
  return ZC_OK;
}

}  // extern "C"
