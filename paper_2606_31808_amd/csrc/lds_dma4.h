// Masked 4-byte loads from global memory straight to LDS, beside the 16-byte
// ones of lds_dma.h (the same rules: the loads are unknown to the compiler's
// counters, and M0 holds the LDS address).
#pragma once
#include "common.h"

namespace lmop {

// 4 bytes per lane to LDS at lds_addr + 4*lane, for the lanes of a wave-uniform
// mask (none: no load); every lane must be active
LMOP_DEVICE void g2l4_m0_mask(const void* sbase, uint32_t voff, uint32_t lds_addr, uint64_t mask) {
  // (the compiler may compute a uniform mask in vector registers)
  mask = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(mask >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)mask);
  asm volatile(
      "s_mov_b32 m0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dword %0, %1\n\t"
      "s_mov_b64 exec, -1"
      :
      : "v"(voff), "s"(sbase), "s"(lds_addr), "s"(mask)
      : "memory");
}

}  // namespace lmop
