// Direct loads, global -> LDS, of the kernels on microscaled operands, in wavefronts whose lanes are all active: by all lanes (more = ~0) or by none (0), so
// that a wavefront's loads count the same whether there is something to load or not.  The execution mask is changed and put back inside the
// statement.
#pragma once
#include "lds_pipe.h"

namespace ss {

__device__ inline void mx4_load16(const uint8_t* base, uint32_t lane_off, uint32_t lds, uint32_t more)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(more) : "memory", "m0");
}
// four bytes a lane, by the lanes of lo (0 .. 31) and hi (32 .. 63)
__device__ inline void mx4_load4(const uint8_t* base, uint32_t lane_off, uint32_t lds, uint32_t lo, uint32_t hi)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %4\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(lo), "s"(hi) : "memory", "m0");
}

}  // namespace ss
