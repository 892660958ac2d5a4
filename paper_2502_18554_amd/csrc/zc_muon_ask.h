// What the products of the step for matrices ask memory for: where a matrix's parts lie, which tiles a workgroup has, which rows of which operand a tile takes, and the order of the requests (host
// code too, so that a test goes through all of it on the CPU).
#pragma once

#include <cstdint>

namespace zc {

using u8 = uint8_t;
using u32 = uint32_t;
using u64 = uint64_t;

constexpr u32 kMuonAlong = 128;                      // rows of X, A, B and of X turned are filled up with zeros to a multiple of so many values
constexpr u64 muon_along(u64 n) { return (n + kMuonAlong - 1) / kMuonAlong * kMuonAlong; }

// Places of a matrix's parts in its share of the workspace: X, X turned twice (one is read while the other is written), A, B; the low parts of two behind the high ones of each.
struct MuonParts {
  u64 row_x, row_t;                                  // values of a row of X; of X turned, A and B
  u64 plane_x, plane_t, plane_a;                     // bytes
  u64 x, t0, t1, a, b, bytes;
  constexpr MuonParts(u32 r, u32 c, u32 planes)
      : row_x(muon_along(c)), row_t(muon_along(r)), plane_x(2 * r * row_x), plane_t(2 * c * row_t), plane_a(2 * r * row_t), x(0), t0(x + planes * plane_x), t1(t0 + planes * plane_t),
        a(t1 + planes * plane_t), b(a + planes * plane_a), bytes(b + planes * plane_a) {}
};

enum { kMuonGram, kMuonPoly, kMuonUpdate, kMuonFinish };       // kMuonFinish + the weights' type
constexpr bool muon_symmetric(int mode) { return mode == kMuonGram || mode == kMuonPoly; }

// The operands of a product, of which both are summed along their rows: where they begin, for the segments high high, high low, low high.
constexpr u64 muon_along_of(const MuonParts& p, int mode) { return mode == kMuonGram ? p.row_x : p.row_t; }
constexpr u64 muon_operand_a(const MuonParts& p, int mode, u32 segment) {
  return (mode == kMuonGram ? p.x : mode == kMuonPoly ? p.a : p.b) + (segment == 2 ? (mode == kMuonGram ? p.plane_x : p.plane_a) : 0);
}
constexpr u64 muon_operand_b(const MuonParts& p, int mode, u32 which, u32 segment) {
  return (mode == kMuonGram ? p.x : mode == kMuonPoly ? p.a : which ? p.t1 : p.t0) + (segment == 1 ? (mode == kMuonGram ? p.plane_x : mode == kMuonPoly ? p.plane_a : p.plane_t) : 0);
}

// The tiles of workgroup `block` of `blocks`: every XCD has a run of neighbouring tiles (workgroups go round the eight XCDs).
struct MuonShare {
  u32 first, end, step;
  constexpr MuonShare(u32 tiles, u32 block, u32 blocks) : first(0), end(0), step(0) {
    const u32 xcd = block & 7u, share = tiles >> 3, more = tiles & 7u, begin = xcd * share + (xcd < more ? xcd : more);
    first = begin + (block >> 3);
    end = begin + share + (xcd < more ? 1u : 0u);
    step = (blocks + 7u - xcd) >> 3;
  }
};

// Row and column of tile t of a matrix whose results are `down` x `across` tiles; of symmetric results, those on and under the diagonal.  guess: a root of t / 32, about.
struct MuonPlace {
  u32 row, col;
};
template <bool SYMMETRIC>
constexpr MuonPlace muon_place(u32 t, u32 down, u32 across, u32 guess) {
  if constexpr (SYMMETRIC) {
    // Strips of eight rows of tiles, down their columns: 32 s^2 + 4 s tiles are before strip s, which has 8 s whole columns and a triangle.
    u32 s = guess;
    while (s && 32 * s * s + 4 * s > t) --s;
    while (32 * (s + 1) * (s + 1) + 4 * (s + 1) <= t) ++s;
    u32 rest = t - (32 * s * s + 4 * s), c = 0;
    const u32 left = down - 8u * s, high = left < 8u ? left : 8u;
    if (rest < 8u * s * high) {
      c = rest / high;
      return {8u * s + rest - c * high, c};
    }
    rest -= 8u * s * high;
    while (rest >= high - c) rest -= high - c++;
    return {8u * s + c + rest, 8u * s + c};
  } else {
    const u32 strip = t / (8u * across), rest = t - strip * 8u * across, left = down - 8u * strip, high = left < 8u ? left : 8u, c = rest / high;
    return {8u * strip + rest - c * high, c};
  }
}

// Rows of a tile, seen from some bytes along them: `bytes` from `at` on may be read, whatever is behind reads as zeros.
struct MuonSpan {
  u64 at;
  u32 bytes;
  constexpr void aim(u64 base, u64 first, u64 rows, u64 stride, u32 most) {
    at = base + first * stride;
    bytes = u32((rows - first < most ? rows - first : most) * stride);
  }
  constexpr void move_on(u32 by) {
    at += by;
    bytes = bytes > by ? bytes - by : 0u;
  }
};

// The order of a workgroup's requests.  A tile has `stages` stages of 64 values, for operands in two parts three times so many: the segments.  Requests run ahead of the products, into the next tile
// and at last behind the last one, where there is nothing left to ask for and no tile to look at, however many more are made.
enum class MuonNext { kMoveOn, kAim, kNothing };     // along the same rows; at others; no longer
struct MuonAsked {
  u32 tile, stage, segment;
  // Behind the request for a stage: what the next one is.
  constexpr MuonNext next(u32 stages, u32 planes, u32 step, u32 end) {
    if (++stage < stages) return MuonNext::kMoveOn;
    stage = 0;
    if (tile >= end) return MuonNext::kNothing;
    if (planes > 1 && ++segment < 3) return MuonNext::kAim;
    segment = 0;
    tile += step;
    return tile < end ? MuonNext::kAim : MuonNext::kNothing;
  }
};

// The same for a wave that takes every fourth stage of one tile, from its own number on: the next one's segment, its number there, and in all.
struct MuonQuarter {
  u32 segment, at, all;
  constexpr void settle(u32 per) {
    while (at >= per) at -= per, ++segment;
  }
  constexpr void next() { at += 4, all += 4; }
};

}  // namespace zc
