// Memory straight into LDS, and the waits for it (why in assembler: gemm_f32_async.hpp).
#pragma once

#include <cstdint>

namespace tma {

typedef __attribute__((address_space(3))) const void lds_void;
__device__ __forceinline__ uint32_t lds_address(const void *p) { return uint32_t(reinterpret_cast<uintptr_t>((lds_void *)(p))); }

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // (m0 is named as reserved: it is set, all the same, and the compiler sets it again for its own use)
// E elements per lane from base + the lane's offset in bytes, to consecutive LDS addresses from `lds` on
template <int E>
__device__ __forceinline__ void lds_fetch(uint32_t lds, const float *base, uint32_t offset)
{
    if constexpr (E == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
template <int E>
__device__ __forceinline__ void lds_fetch(uint32_t lds, const float *p)
{
    if constexpr (E == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop
// All but this wavefront's kVm youngest memory operations are done, and its LDS reads; then the whole block meets.
template <int kVm>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kVm) : "memory");
}

}  // namespace tma
