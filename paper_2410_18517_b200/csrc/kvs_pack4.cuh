// The row of a 4-bit cache, shared by the kernels that write, read and attend over it.
//
// A row of D elements is cut into four groups of D/4.  With lo and hi the group's smallest and largest element (fp32):
//   s = (hi - lo) * (1/15) rounded up to bf16,  b = lo - 16 s rounded to bf16
//   code c = clamp(rint((x - b) / s) - 16, 0, 15),  value = s * (16 + c) + b rounded once to the storage type
// Why 16 + c and not c: four bits laid at bits 3..6 of a bf16 whose upper bits are those of 16.0 ARE the number 16 + c, so
// one OR makes a factor of the code and one fused multiply-add the value.  Why s is rounded up: the largest element then has
// a code of its own, and every element is off by at most s/2 plus the rounding of b (half a bf16 step).
// A group that holds an infinity or a NaN, or whose s or b overflows, gets NaN for both: all its values are NaN.
//
// Layout, 16 + D/2 bytes: four words s | b << 16 (bf16 each), one per group, then D/2 bytes of codes, element 8 w + i in
// bits 4 i .. 4 i + 3 of word w.  80 and 48 bytes are odd multiples of 16: rows that lie side by side in shared memory start
// in different banks.
#pragma once
#include "kvs_device.cuh"

namespace kvs {

template <int D>
struct Pack4Row {
    static constexpr int RB = 16 + D / 2;
    static constexpr int WORDS = D / 8;        // words of codes
    static constexpr int GROUP = D / 4;        // elements per group
};

// bf16 pairs: {16 + nibble, 16 + nibble} of bits 4 I .. 4 I + 3 of either half of w
template <int I>
__device__ __forceinline__ uint32_t pack4_pair(uint32_t w) {
    const uint32_t at = I == 0 ? w << 3 : w >> (4 * I - 3);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(at), "r"(0x00780078u), "r"(0x41804180u));      // (at & mask) | magic
    return r;
}

// fused multiply-add of two bf16 pairs, rounded once
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// value of code c in fp32 (exact product, one rounding)
__device__ __forceinline__ float pack4_value(uint32_t c, float s, float b) { return fmaf(s, 16.f + (float)c, b); }

}  // namespace kvs
