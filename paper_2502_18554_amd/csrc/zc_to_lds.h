// A load from memory straight to LDS, written out.  gfx950 only.
#pragma once

#include "zc_common.h"

namespace zc {

// 16 bytes a lane to LDS, at `to` and on.  (Written out: of its own loads to LDS the compiler thinks that any read of LDS may have to wait for them.  m0 is reserved, so
// that it cannot be named among what is overwritten: nothing else in kernels that use this may use it, as another load to LDS, a message or an indexed register would.)
// The buffer's words may come from a vector instruction (uniform values that the compiler has in lanes) right before: a load reads them five wait states later at the earliest, which the compiler
// keeps for its own loads, but not for what is written out.  With fewer the load would see the words of before, another place or length.
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t from, u32 to, u32 lane_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(lane_offset), "s"(from) : "memory");
}

}  // namespace zc
