// A pair of fp32 values taken apart into three bf16 pairs whose sum it is (why, and for what range: gemm_split.hpp).
#pragma once
#include "common.hpp"

namespace tma {

constexpr float kSplitScale = 0x1p24f, kSplitUnscale = 0x1p-48f;   // of both operands; of their product (see Range)

// two values -> their three parts as bf16 pairs (first value in the low half).  What a rounding left over is exact, and
// comes from one instruction: v - h as the dot product of the pair (h0, h1) with (-1, 0) or (0, -1), plus v.
struct SplitPair {
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    uint32_t first, second;
    __device__ __forceinline__ SplitPair() : first(0x0000BF80u), second(0xBF800000u)
    {
        // held in registers: as an inline constant of this instruction -1.0 would stand in the other half
        asm("" : "+s"(first));
        asm("" : "+s"(second));
    }
    __device__ __forceinline__ float left(float v, uint32_t parts, uint32_t which) const
    {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, parts), __builtin_bit_cast(Pair, which), v, false);
    }
    __device__ __forceinline__ void operator()(float x, float y, uint32_t &h, uint32_t &m, uint32_t &l) const
    {
        x *= kSplitScale;
        y *= kSplitScale;
        h = pack_bf16(x, y);
        x = left(x, h, first);
        y = left(y, h, second);
        m = pack_bf16(x, y);
        l = pack_bf16(left(x, m, first), left(y, m, second));
    }
};

}  // namespace tma
