// Rows of 128 elements in 4 bits: eight groups of 16 with a scale each, an element is a whole number -7 .. 7 times its group's scale.
//
// Scale byte u = 8 E + M, E = 0 .. 30: s = 2^(E - 17) (1 + M / 8), from 2^-17 to 15360, so that rows of any size that a model has need no second
// scale.  E = 31: not a number.  A code is stored as c + 8; of the eight elements in a 32-bit word, element 2 i has bits
// 4 i .. 4 i + 3 and element 2 i + 1 the same of the upper half, so that a mask leaves a pair of neighbours in the two halves.
//
// Every number of this format is a bf16 number: c has three bits, M and its leading one four.  It is rebuilt, times 2^-19, from bf16 arithmetic on pairs.
// A bf16 pattern below 256 is that whole number times 2^-133 (subnormal numbers and the first normal ones are spaced alike), so a code v = c + 8 in bits 0 .. 3 of
// a half is v 2^-133, one in bits 4 .. 7 is 16 v 2^-133, and a mask is all that either needs:
//     t * S - 8 2^-133 S = c s 2^-19,     S = 2^114 s (over 16 for the upper codes)
// with one rounding of a number that needs none: nine instructions for eight elements (eleven with a shift for each pair).  S has E + 224 as its exponent bits, so
// that the byte times 16 plus a constant is S, and E = 31 is infinite or NaN by itself: the element comes out as NaN.  The 2^19 goes into the softmax
// scale for keys and is taken back with the result for values.
#pragma once
#include <stdint.h>

#include <cuda_runtime.h>

#include "sm100_ptx.cuh"

namespace mage {
namespace kv4 {

struct View {
    uint8_t *k4, *v4;                         // half a byte an element, addressed like the 16-bit cache
    uint8_t *k_scale, *v_scale;               // eight bytes a row
};

constexpr int kRowBytes = 64;
constexpr float kUnit = 524288.f;             // 2^19: what Scale::pair leaves out

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// The scale of a pair of elements as the products need it: of one group, or of two (one for each half).
struct Scale {
    uint32_t s, s16, z;
    __device__ __forceinline__ explicit Scale(uint32_t u) : Scale(u * 0x00100010u + 0x70007000u, true) {}
    __device__ __forceinline__ Scale(uint32_t u_lo, uint32_t u_hi) : Scale(u_hi * 0x00100000u + (u_lo * 16u + 0x70007000u), true) {}
    // elements 2 i and 2 i + 1 of word w, times 2^-19
    __device__ __forceinline__ uint32_t pair(uint32_t w, int i) const {
        const uint32_t v = i < 2 ? w : w >> 8;
        return i & 1 ? fma_bf16x2(v & 0x00f000f0u, s16, z) : fma_bf16x2(v & 0x000f000fu, s, z);
    }

private:
    __device__ __forceinline__ Scale(uint32_t s_, bool) : s(s_), s16(mul_bf16x2(s_, 0x3d803d80u)), z(mul_bf16x2(s_, 0x80088008u)) {}
};
// the elements themselves
__device__ __forceinline__ uint32_t exact_pair(const Scale &sc, uint32_t w, int i) { return mul_bf16x2(sc.pair(w, i), 0x49004900u); }
// Whether one of four scale bytes is no number.
__device__ __forceinline__ bool odd_scales(uint32_t u4) { return __vcmpeq4(u4 & 0xf8f8f8f8u, 0xf8f8f8f8u) != 0u; }

// Scale byte of a group from its largest magnitude (bf16 bits): the scale nearest to amax / 7, halves up.  A bf16 number over 7 is a midpoint of
// two scales or at least 2^-9 of itself away from it, so a factor 1 + 2^-13 decides the halves and nothing else.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    constexpr float kSeventh = 0.14285714285714285f * 1.0001220703125f;
    const int r = (int)((__float_as_uint(__uint_as_float(amax << 16) * kSeventh) + 0x80000u) >> 20) - (110 << 3);
    return (uint32_t)min(max(r, 0), 247);
}
__device__ __forceinline__ float rcp(float x) {        // off by 2^-23 at most, which is nothing beside 2^-13
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Codes of this lane's eight elements (as a word) and its group's scale byte.  Sixteen lanes hold a row, two a group; m2: the lane's largest magnitudes
// by halves.  x / s is a half of an odd number or at least 2^-9 of itself away from one, so with the reciprocal taken 2^-13 too small halves go
// toward zero and the rest to the nearest.  An fma with 1.5 2^23 + 8 rounds and leaves c + 8 in the lowest bits; the words' constant parts add up to a
// constant modulo 2^32.  A row that holds a NaN or an infinity: scales 255, codes of zero.  Called by whole warps.
__device__ __forceinline__ uint32_t code8(const uint4 &raw, uint32_t m2, int lane, uint32_t &u) {
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const bool odd = (__ballot_sync(0xffffffffu, m >= 0x7f80u) & (0xffffu << (lane & 16))) != 0;
    u = scale_byte(m);
    const float s = __uint_as_float((u + (110u << 3)) << 20), inv = rcp(s) * 0.9998779296875f;
    const uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[2 * i] = __uint_as_float(x[i] << 16);
        y[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
    if (__builtin_expect(u == 247u, 0)) {                  // (it may be beyond the largest scale: the largest code)
        const float most = 7.25f * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -most), most);
    }
    uint32_t t[4];
    const uint64_t inv2 = ptx::pack2(inv, inv), round2 = ptx::pack2(12582920.f, 12582920.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        ptx::unpack2(ptx::fma2(ptx::pack2(y[2 * i], y[2 * i + 1]), inv2, round2), lo, hi);
        t[i] = __float_as_uint(hi) * 65536u + __float_as_uint(lo);
    }
    const uint32_t w = t[3] * 4096u + (t[2] * 256u + (t[1] * 16u + t[0])) - (uint32_t)(0x4b400000ull * 0x11111111ull);
    if (odd) u = 255u;
    return odd ? 0x88888888u : w;
}

}  // namespace kv4
}  // namespace mage
