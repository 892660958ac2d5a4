// Every request that the products of the step for matrices make of memory (csrc/zc_muon_ask.h), for every kind of tile, one and two parts, from one row on: it asks for the tile's rows of the right
// operand at the right place, no byte of it lies outside that operand, and behind a workgroup's last stage nothing is asked for, however far the requests run ahead.
// With an argument: the same with an order of requests that goes on behind the last tile (in which the next segments' rows are looked for there), which this has to find.
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "../../paper_2502_18554_amd/csrc/zc_muon_ask.h"

using namespace zc;

static bool g_on_and_on = false;
static long g_wrong = 0, g_requests = 0;

struct Shape {
  u32 r, c, planes, count;
};
struct Kind {
  u32 high, wide, per_cu, stages;        // of a tile; workgroups that a CU holds; stages in LDS
};

static MuonNext next_of(MuonAsked& asked, u32 stages, u32 planes, u32 step, u32 end) {
  if (!g_on_and_on) return asked.next(stages, planes, step, end);
  if (++asked.stage < stages) return MuonNext::kMoveOn;
  asked.stage = 0;
  if (planes > 1 && ++asked.segment < 3) return MuonNext::kAim;
  asked.segment = 0;
  asked.tile += step;
  return asked.tile < end ? MuonNext::kAim : MuonNext::kNothing;
}

static void say(const char* what, const Shape& s, int mode, const Kind& k, u32 block, u32 request) {
  if (++g_wrong <= 10) std::printf("%s: %u x %u, parts %u, matrices %u, product %d, tiles %u x %u, workgroup %u, request %u\n", what, s.r, s.c, s.planes, s.count, mode, k.high, k.wide, block, request);
}

template <bool SYMMETRIC>
static MuonPlace place_of(u32 t, u32 down, u32 across) {
  return muon_place<SYMMETRIC>(t, down, across, SYMMETRIC ? u32(std::sqrt(float(t) * (1.0f / 32.0f))) : 0u);
}
static MuonPlace place_of(int mode, u32 t, u32 down, u32 across) { return muon_symmetric(mode) ? place_of<true>(t, down, across) : place_of<false>(t, down, across); }

// One operand's rows for a request: `first` and `most` of the tile, `rows` of the operand, which begins at `from`.
static bool right(const MuonSpan& span, u64 from, u32 first, u32 most, u32 rows, u64 stride, u32 stage) {
  const u64 there = rows - first < most ? rows - first : most;
  return first < rows && span.at == from + first * stride + 128 * stage && span.bytes == there * stride - 128 * stage && span.at + span.bytes <= from + rows * stride &&
         128 * (stage + 1) <= stride && there * stride < (u64(1) << 32);
}

static void go(const Shape& s, int mode, const Kind& k, u32 which) {
  const MuonParts parts(s.r, s.c, s.planes);
  const bool symmetric = muon_symmetric(mode);
  const u64 bytes = (parts.bytes + 255) / 256 * 256, stride = 2 * muon_along_of(parts, mode);
  const u32 down = (s.r + k.high - 1) / k.high, across = symmetric ? down : (s.c + k.wide - 1) / k.wide, each = symmetric ? down * (down + 1) / 2 : down * across, tiles = each * s.count;
  const u32 per = u32(stride / 128), segments = s.planes > 1 ? 3 : 1, of_b = symmetric ? s.r : s.c;
  const bool quarters = k.high == 32;
  const u32 blocks = quarters || tiles < 256 * k.per_cu ? tiles : 256 * k.per_cu;
  u32 visited = 0;
  for (u32 block = 0; block < blocks; ++block) {
    const MuonShare share(tiles, block, blocks);
    if (share.first >= share.end) continue;
    u32 of_block = 0;
    for (u32 tile = share.first; tile < share.end; tile += share.step) ++of_block;
    visited += of_block;
    // What a request for (tile, segment, stage) has to be.
    const auto check = [&](const MuonSpan& a, const MuonSpan& b, u32 tile, u32 segment, u32 stage, u32 request) {
      const u64 base = tile / each * bytes;
      const MuonPlace p = place_of(mode, tile % each, down, across);
      const u64 plane_a = mode == kMuonGram ? parts.plane_x : parts.plane_a, plane_b = mode == kMuonGram ? parts.plane_x : mode == kMuonPoly ? parts.plane_a : parts.plane_t;
      const u64 begin_a = base + (mode == kMuonGram ? parts.x : mode == kMuonPoly ? parts.a : parts.b) + (segment == 2 ? plane_a : 0);
      const u64 begin_b = base + (mode == kMuonGram ? parts.x : mode == kMuonPoly ? parts.a : which ? parts.t1 : parts.t0) + (segment == 1 ? plane_b : 0);
      if (p.row >= down || p.col >= across || (symmetric && p.col > p.row)) say("a tile that is not there", s, mode, k, block, request);
      else if (!right(a, begin_a, p.row * k.high, k.high, s.r, stride, stage) || !right(b, begin_b, p.col * k.wide, k.wide, of_b, stride, stage)) say("another place", s, mode, k, block, request);
      if (a.at + a.bytes > base + bytes || b.at + b.bytes > base + bytes) say("behind the matrix", s, mode, k, block, request);
      ++g_requests;
    };
    const auto aim = [&](MuonSpan& a, MuonSpan& b, u32 tile, u32 segment) {
      const u64 base = tile / each * bytes;
      const MuonPlace p = place_of(mode, tile % each, down, across);
      a.aim(base + muon_operand_a(parts, mode, segment), u64(p.row) * k.high, s.r, stride, k.high);
      b.aim(base + muon_operand_b(parts, mode, which, segment), u64(p.col) * k.wide, of_b, stride, k.wide);
    };
    if (quarters) {                      // a workgroup has one tile, and each of its four waves every fourth stage
      for (u32 wave = 0; wave < 4; ++wave) {
        MuonQuarter asked{0, wave, wave};
        for (u32 n = 0; n < (per * segments + 3) / 4 + k.stages + 8; ++n) {
          MuonSpan a, b;
          asked.settle(per);
          aim(a, b, share.first, asked.segment);
          a.move_on(128 * asked.at);
          b.move_on(128 * asked.at);
          if (asked.all < per * segments) check(a, b, share.first, (wave + 4 * n) / per, (wave + 4 * n) % per, n);
          asked.next();                  // (behind the last stage the length is set to nothing)
        }
      }
      continue;
    }
    MuonAsked asked{share.first, 0, 0};
    MuonSpan a, b;
    aim(a, b, asked.tile, asked.segment);
    const u32 stages = of_block * segments * per;
    for (u32 n = 0; n < stages + k.stages + 8; ++n) {
      if (n < stages) check(a, b, share.first + n / (segments * per) * share.step, n / per % segments, n % per, n);
      else if (a.bytes || b.bytes) say("something behind the last stage", s, mode, k, block, n);
      a.move_on(128);
      b.move_on(128);
      const MuonNext next = next_of(asked, per, s.planes, share.step, share.end);
      if (next == MuonNext::kAim) {
        if (asked.tile >= share.end) {   // (there is no such tile to aim at here)
          say("a tile behind the last one", s, mode, k, block, n);
          break;
        }
        aim(a, b, asked.tile, asked.segment);
      } else if (next == MuonNext::kNothing) {
        a.bytes = b.bytes = 0;
      }
    }
  }
  if (visited != tiles) say("tiles left out", s, mode, k, 0, visited);
}

static void all(const Shape& s) {
  for (int mode : {int(kMuonGram), int(kMuonPoly), int(kMuonUpdate)})
    for (const Kind& k : {Kind{32, 32, 2, 2}, Kind{64, 64, 2, 4}, Kind{128, 128, 2, 2}, Kind{128, 128, 1, 3}, Kind{192, 192, 1, 3}, Kind{256, 256, 1, 2}, Kind{64, 128, 2, 3}, Kind{128, 256, 1, 3}})
      if (!muon_symmetric(mode) || k.high == k.wide)
        for (u32 which : {0u, 1u}) go(s, mode, k, which);
}

int main(int argc, char**) {
  g_on_and_on = argc > 1;
  for (u32 planes : {1u, 2u}) {
    for (u32 r = 1; r <= 130; ++r)
      for (u32 c : {r, r + 1, 300u, 4001u}) all({r, c, planes, 1});
    for (u32 r : {1u, 2u, 3u, 64u, 128u, 129u}) all({r, 70001, planes, 1});
    all({3, 50001, planes, 1});
    for (u32 r : {192u, 193u, 256u, 257u, 511u, 1000u, 2050u}) all({r, 2 * r + 1, planes, 1});
    for (u32 count : {2u, 5u, 24u}) {
      all({2, 7001, planes, count});
      all({100, 300, planes, count});
      all({256, 512, planes, count});
    }
  }
  // The largest sides: a tile's rows stay below 2^32 bytes, and its place is one of the matrix's.
  for (u32 high : {32u, 64u, 128u, 192u, 256u}) {
    const u32 down = ((1u << 20) + high - 1) / high;
    const u32 half = down * (down + 1) / 2;
    for (u32 t : {0u, 1u, half / 3, half / 2, half - 2, half - 1}) {
      const MuonPlace p = place_of<true>(t, down, down);
      if (p.row >= down || p.col > p.row) ++g_wrong, std::printf("tile %u of %u rows of them: %u, %u\n", t, down, p.row, p.col);
    }
    MuonSpan a;
    a.aim(0, u64(down - 1) * high, u64(1) << 20, u64(2) << 20, high);
    if (a.bytes == 0 || a.at + a.bytes != u64(2) << 40) ++g_wrong, std::printf("the last rows of 2^20 by %u\n", high);
  }
  std::printf("%ld requests, %ld of them wrong\n", g_requests, g_wrong);
  return g_wrong != 0;
}
