// Direct loads, global -> LDS, of the kernels on microscaled operands, in wavefronts whose lanes are all active: by all lanes (more < 0) or by none (more >= 0),
// so that a wavefront's loads count the same whether there is something to load or not.  The execution mask is set and put back inside the
// statement, from a sign, which stays a scalar where a truth value would go through a vector register.
#pragma once
#include "lds_pipe.h"

namespace ss {

__device__ inline void mx4_load16(const uint8_t* base, uint32_t lane_off, uint32_t lds, int more)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_ashr_i32 exec_lo, %3, 31\n\ts_mov_b32 exec_hi, exec_lo\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(more) : "memory", "m0", "scc");
}
__device__ inline void mx4_load4(const uint8_t* base, uint32_t lane_off, uint32_t lds, int more)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_ashr_i32 exec_lo, %3, 31\n\ts_mov_b32 exec_hi, exec_lo\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
                 ::"s"(lds), "v"(lane_off), "s"(base), "s"(more) : "memory", "m0", "scc");
}

}  // namespace ss
