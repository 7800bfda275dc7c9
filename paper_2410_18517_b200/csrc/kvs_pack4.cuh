// The row of a 4-bit cache, shared by the kernels that write, read and attend over it.
//
// A row of D elements is cut into four groups of D/4.  With lo and hi the group's smallest and largest element (fp32):
//   s = (hi - lo) * (1/15) rounded up to bf16,  b = lo - 16 s rounded to bf16
//   code c = clamp(rint((x - b) / s) - 16, 0, 15),  value = s * (16 + c) + b rounded once to the storage type
// Why 16 + c and not c: four bits laid at bits 3..6 of a bf16 whose upper bits are those of 16.0 ARE the number 16 + c, so
// one OR makes a factor of the code and one fused multiply-add the value.  Why s is rounded up: the largest element then has
// a code of its own, and every element is off by at most s/2 plus the rounding of b (half a bf16 step).  The nearest fp32 of 1/15
// is above 1/15, so a range of exactly 15 bf16 steps mostly gets the next larger step: rows' values are not stored as they are.
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

// ---- making a row

__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.4028234e38f; }

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// smallest and largest of the elements in N 16-byte pieces (NaN if one is)
template <int N>
__device__ __forceinline__ void range_of(const uint4 (&in)[N], float* lo, float* hi, __nv_bfloat16) {      // two at a time
    uint32_t l = in[0].x, h = in[0].x;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        l = min_bf16x2(min_bf16x2(l, in[i].x), min_bf16x2(min_bf16x2(in[i].y, in[i].z), in[i].w));
        h = max_bf16x2(max_bf16x2(h, in[i].x), max_bf16x2(max_bf16x2(in[i].y, in[i].z), in[i].w));
    }
    *lo = min_nan(bf16_lo(l), bf16_hi(l));
    *hi = max_nan(bf16_lo(h), bf16_hi(h));
}
template <int N>
__device__ __forceinline__ void range_of(const uint4 (&in)[N], float* lo, float* hi, float) {
    *lo = *hi = __uint_as_float(in[0].x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = __uint_as_float(in[i].x), y = __uint_as_float(in[i].y), z = __uint_as_float(in[i].z), w = __uint_as_float(in[i].w);
        *lo = min_nan(min_nan(*lo, x), min_nan(min_nan(y, z), w));
        *hi = max_nan(max_nan(*hi, x), max_nan(max_nan(y, z), w));
    }
}

// eight elements: one piece of bf16, two of fp32
__device__ __forceinline__ void eight_of(const uint4* in, float (&x)[8], __nv_bfloat16) { Unpack<__nv_bfloat16>::run(in[0], x); }
__device__ __forceinline__ void eight_of(const uint4* in, float (&x)[8], float) {
    Unpack<float>::run(in[0], *reinterpret_cast<float(*)[4]>(x));
    Unpack<float>::run(in[1], *reinterpret_cast<float(*)[4]>(x + 4));
}

constexpr float kRint = 12582912.f;       // 1.5 * 2^23
__host__ __device__ constexpr uint32_t rint_offset() {        // sum over i of (bits of kRint + 16) * 16^i
    uint32_t sum = 0;
    for (int i = 0; i < 8; ++i) sum = sum * 16u + (0x4b400000u + 16u);
    return sum;
}

// the code of x, exactly
__device__ __forceinline__ uint32_t code_of(float x, float s, float b, float inv) {
    const float d = __fsub_rn(x, b), back = __fsub_rn(x, d);
    const float lost = __fadd_rn(__fsub_rn(x, __fadd_rn(d, back)), __fsub_rn(back, b));      // x - b = d + lost
    const float below = floorf(__fmul_rn(d, inv) - 0.5f);             // f lies in [below + 1/2 - 1e-5, below + 3/2 + 1e-5]
    // which of the borders below + 1/2 and below + 3/2 it is at or past (a tie goes to the even one)
    const float first = __fadd_rn(__fmaf_rn(-(below + 0.5f), s, d), lost), second = __fadd_rn(__fmaf_rn(-(below + 1.5f), s, d), lost);
    const bool odd = (int)below & 1;
    float r = below;
    if (first > 0.f || (first == 0.f && odd)) r += 1.f;
    if (second > 0.f || (second == 0.f && !odd)) r += 1.f;
    return (uint32_t)(fminf(fmaxf(r, 16.f), 31.f) - 16.f);
}

// Codes by adding 1.5 * 2^23 to the quotient: its lowest bits are then rint's, and a multiply-add by 16 strings them together.
// In fp32 the quotient, at most 32, is off by less than 1e-5, so it is taken twice, 1e-6 of itself too large and too
// small: where the two words agree, they are right.  An element next to the border between two codes is settled by the sign
// of x - b - (k + 1/2) s, which two fp32 operations and their remainders give exactly.  (Ties are real: bf16 elements lie on
// few values; of normal draws 1 in 300, so that of a warp's words of eight codes every other has one.)
// The group in `in` (its 16-byte pieces) becomes the pair s | b << 16 and its words of codes.
template <typename T, int D>
__device__ __forceinline__ void pack_group(const uint4 (&in)[Pack4Row<D>::GROUP * sizeof(T) / 16], uint32_t* pair,
                                           uint32_t (&words)[Pack4Row<D>::GROUP / 8]) {
    constexpr int WORDS = Pack4Row<D>::GROUP / 8, V = sizeof(T) / 2;      // words; 16-byte pieces of eight elements
    float lo, hi;
    range_of(in, &lo, &hi, T());
    const float step = __fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f);
    const float s = __uint_as_float((__float_as_uint(step) + 0xffffu) & 0xffff0000u);
    const float b = __bfloat162float(__float2bfloat16_rn(__fsub_rn(lo, 16.f * s)));
    const bool broken = !(finite(step) && finite(s) && finite(b));
    // Where s is tiny its reciprocal may overflow and products may lose bits, where it is huge x - b, up to 31 s, may overflow:
    // code_of takes all of it times a power of two there (exact but for an element below 2^-147 beside a step above 1e36).
    const float scale = s > 1e36f ? 0.25f : s < 1e-30f ? 18446744073709551616.f : 1.f;
    const float inv = 1.f / (s * scale);
    // What the two words say is not taken then, nor where the rounding of b (up to 2^-8 |b|) can bring a quotient past 15.5 or 31.5.
    const bool plain = fabsf(b) <= 100.f * s && scale == 1.f;
    const uint64_t minus = pair_of(-b, -b), above = pair_of(inv * 1.000001f, inv * 1.000001f), under = pair_of(inv * 0.999999f, inv * 0.999999f);
    const uint64_t magic = pair_of(kRint, kRint);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        float x[8];
        eight_of(in + w * V, x, T());
        uint32_t one = 0, two = 0;
#pragma unroll
        for (int i = 6; i >= 0; i -= 2) {
            const uint64_t d = add2(pair_of(x[i], x[i + 1]), minus), y = fma2(d, above, magic), z = fma2(d, under, magic);
            one = (one * 16 + (uint32_t)(y >> 32)) * 16 + (uint32_t)y;
            two = (two * 16 + (uint32_t)(z >> 32)) * 16 + (uint32_t)z;
        }
        one -= rint_offset();
        two -= rint_offset();
        uint32_t unsure = plain ? one ^ two : 0xffffffffu;
        if (unsure && !broken) {
            if (s == 0.f) {
                one = 0;
            } else {
                while (unsure) {
                    const int i = (__ffs(unsure) - 1) / 4;
                    const float y0 = i & 1 ? x[1] : x[0], y1 = i & 1 ? x[3] : x[2], y2 = i & 1 ? x[5] : x[4], y3 = i & 1 ? x[7] : x[6];
                    const float y = i & 4 ? (i & 2 ? y3 : y2) : (i & 2 ? y1 : y0);
                    one = (one & ~(15u << (4 * i))) | code_of(y * scale, s * scale, b * scale, inv) << (4 * i);
                    unsure &= ~(15u << (4 * i));
                }
            }
        }
        words[w] = broken ? 0u : one;
    }
    *pair = broken ? 0x7fc07fc0u : (__float_as_uint(s) >> 16) | (__float_as_uint(b) & 0xffff0000u);
}

template <int D>
__device__ __forceinline__ void store_group(uint32_t* row, uint32_t group, uint32_t pair, const uint32_t (&words)[Pack4Row<D>::GROUP / 8]) {
    row[group] = pair;
    if constexpr (D == 128) reinterpret_cast<uint4*>(row)[1 + group] = make_uint4(words[0], words[1], words[2], words[3]);
    else reinterpret_cast<uint2*>(row)[2 + group] = make_uint2(words[0], words[1]);
}

}  // namespace kvs
