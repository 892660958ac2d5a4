// The order in which a workgroup asks for stages (csrc/zc_muon_ask.h): every stage of every segment of its tiles once, and no look at a tile behind the last one however far the requests run ahead.
#include <cstdio>
#include <initializer_list>

#include "../../paper_2502_18554_amd/csrc/zc_muon_ask.h"

int main() {
  int wrong = 0;
  for (uint32_t stages : {2u, 4u, 6u, 26u})
    for (uint32_t planes : {1u, 2u})
      for (uint32_t step : {1u, 64u})
        for (uint32_t tiles : {1u, 2u, 5u}) {
          const uint32_t first = 3, end = first + (tiles - 1) * step + 1, segments = planes > 1 ? 3 : 1;
          zc::MuonAsked asked{first, 0, 0};
          bool there = true;                               // whether the rows are those of a tile
          uint32_t made = 0;
          for (uint32_t k = 0; k < tiles * segments * stages + 40; ++k) {
            if (there) {
              const uint32_t tile = first + k / (segments * stages) * step, segment = k / stages % segments, stage = k % stages;
              if (asked.tile != tile || asked.segment != segment || asked.stage != stage) ++wrong;
              ++made;
            }
            const zc::MuonNext next = asked.next(stages, planes, step, end);
            if (next == zc::MuonNext::kAim) {
              if (asked.tile >= end) ++wrong, std::printf("stages %u planes %u tiles %u: looks at tile %u of %u after %u requests\n", stages, planes, tiles, asked.tile, end, k + 1);
              there = true;
            } else if (next == zc::MuonNext::kNothing) {
              there = false;
            }
          }
          if (made != tiles * segments * stages) ++wrong, std::printf("stages %u planes %u tiles %u: %u requests\n", stages, planes, tiles, made);
        }
  return wrong != 0;
}
