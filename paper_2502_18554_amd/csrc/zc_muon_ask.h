// In which order a workgroup asks for the stages of its tiles (host code too).
#pragma once

#include <cstdint>

namespace zc {

// A tile has `stages` stages, for operands in two parts three times so many: the segments high high, high low, low high.  Requests run ahead of the products, into the next tile and at last behind the
// last one, where there is nothing left to ask for and no tile to look at, however many more are made.
enum class MuonNext { kMoveOn, kAim, kNothing };     // along the same rows; at others; no longer
struct MuonAsked {
  uint32_t tile, stage, segment;
  // Behind the request for a stage: what the next one is.
  constexpr MuonNext next(uint32_t stages, uint32_t planes, uint32_t step, uint32_t end) {
    if (++stage < stages) return MuonNext::kMoveOn;
    stage = 0;
    if (tile >= end) return MuonNext::kNothing;
    if (planes > 1 && ++segment < 3) return MuonNext::kAim;
    segment = 0;
    tile += step;
    return tile < end ? MuonNext::kAim : MuonNext::kNothing;
  }
};

}  // namespace zc
