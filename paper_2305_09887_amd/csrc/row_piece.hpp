// Rows of any width and pitch in pieces of 16 bytes.
#pragma once
#include "common.hpp"

namespace tma {

typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ uint32_t bits1(const float *p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits1(const uint16_t *p) { return *p; }

// A piece of 16 bytes from element `at` on of an array, of which the first `valid` elements are wanted and the others read as zero.
// kWords (4-byte aligned, the load needs no more): one load without a branch; a piece that would run past `last`, the last place where
// 16 bytes of whole words are left, comes from there and is moved back in registers.  Else element by element.
// Two-byte elements in rows of an odd width: whole words then end an element before the array does (the place at its end would be an odd element,
// two bytes off a word).  That one element is fetched by itself, where a piece is moved that wants it.
template <typename T, bool kWords>
struct RowPiece {
    static constexpr int E = 16 / sizeof(T);
    static __host__ __device__ __forceinline__ int64_t last_place(int64_t n, int64_t ld, int F)
    {
        return (n - 1) * ld + F - E - (sizeof(T) == 2 ? F & 1 : 0);
    }
    // the bits of the element that no such piece ends with (zero: there is none, or h, where given, closes it)
    static __device__ __forceinline__ uint32_t left_out(const T *x, const T *h, int64_t n, int64_t ld, int F)
    {
        if constexpr (!kWords || sizeof(T) == 4) return 0u;
        else {
            const int64_t at = (n - 1) * ld + F - 1;
            return F & 1 && (!h || bf16_to_f32(h[at]) > 0.0f) ? x[at] : 0u;
        }
    }
    static __device__ __forceinline__ uint4 load(const T *__restrict__ x, int64_t at, int valid, int64_t last)
    {
        if constexpr (kWords) {
            const Words4 w = *reinterpret_cast<const Words4 *>(x + (at < last ? at : last));
            return make_uint4(w.x, w.y, w.z, w.w);
        } else {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < valid) w[j * int(sizeof(T)) / 4] |= bits1(x + at + j) << (sizeof(T) == 2 ? 16 * (j & 1) : 0);
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // back: elements by which the piece was fetched too early; what follows its elements then is `rest`, the element of left_out (in the last row
    // the one that is missing, in others behind what is wanted)
    static __device__ __forceinline__ uint4 moved(const uint4 &p, int back, uint32_t rest)
    {
        uint64_t lo = uint64_t(p.y) << 32 | p.x, hi = uint64_t(p.w) << 32 | p.z, top = rest;
        int bits = back * int(sizeof(T)) * 8;
        if (bits >= 64) {
            lo = hi;
            hi = top;
            top = 0;
            bits -= 64;
        }
        if (sizeof(T) == 2 && bits >= 64) {       // (an array of one column)
            lo = hi;
            hi = 0;
        } else if (bits > 0) {
            lo = lo >> bits | hi << (64 - bits);
            hi = hi >> bits | top << (64 - bits);
        }
        return make_uint4(uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32));
    }
    static __device__ __forceinline__ uint4 cut(const uint4 &p, int valid)
    {
        uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = valid > i ? w[i] : 0u;
            else w[i] &= valid > 2 * i + 1 ? ~0u : valid > 2 * i ? 0xFFFFu : 0u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

}  // namespace tma
