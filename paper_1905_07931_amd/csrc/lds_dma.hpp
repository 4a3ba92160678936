// Copies from global memory straight into LDS, and the wait that counts them.
#pragma once

#include "common.hpp"

namespace l1csr {

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(lds_void *)p; }

// One 1 KB block global -> LDS (16 bytes per lane), base and lds wave-uniform.
// As an instruction of its own rather than the builtin: the compiler orders the
// builtin's loads against the reads of the other buffers and waited for the
// loads just issued (vmcnt(0)) in one step of three.  It writes no register;
// wait_vm() below counts it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is reserved: the clobber orders it, nothing keeps it
__device__ __forceinline__ void dma16(const char *base, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N>
__device__ __forceinline__ void wait_vm() {  // at most N vector memory operations and no LDS access outstanding
    static_assert(N < 16, "low field only");
    __builtin_amdgcn_s_waitcnt(0x0070 | N);
}

}  // namespace l1csr
