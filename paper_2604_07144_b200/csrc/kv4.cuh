// The 4-bit page format and its arithmetic.
//
// A tile, the 16 token rows of one (page, kv head) of one plane, is
//     16 x d / 2 bytes of codes, row after row, then 16 x d / 32 steps (bf16), row after row:
// 1152 bytes at d = 128, 576 at d = 64.  A group of 32 consecutive elements of a row shares one step s;
// code c (0 .. 15, 8 is zero) stands for (c - 8) s.  A row is d / 8 words of eight codes, lowest nibble
// first; the word of elements 32 g + 8 t .. + 7 (t = 0 .. 3) is stored at index t * (d / 32) + g, so that
// the codes of all groups that one lane of an MMA fragment needs lie next to one another.
//
// Quantisation: s = max |x| / 7, rounded UP to five significant bits; c = rint(x / s) + 8.
// Rounding up keeps |x / s| <= 7.  c - 8 has at most three significant bits, so (c - 8) s has at most
// eight and IS a bf16 number: the cache stands for bf16 values, and every reader (decode, prefill,
// read-back) gets exactly the same ones whatever it does with codes and steps.  x has eight significant
// bits and 7 s has eight, so the quotients of fp32 division fall on the same side of every rounding border
// as the real ones: codes are those of exact arithmetic.
// A group with an element that is not finite, or not below 2^120, gets the step NaN: it stands for NaN.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace ap {
namespace kv4 {

constexpr int kGroup = 32;
constexpr float kSmallStep = 7.8886090522101181e-31f;      // 2^-100

template <int D>
struct Tile {
    static constexpr int kGroups = D / kGroup;
    static constexpr int kRowBytes = D / 2;
    static constexpr int kCodeBytes = 16 * kRowBytes;
    static constexpr int kBytes = kCodeBytes + 16 * kGroups * 2;
};

// stored index of the word that holds elements 8 * chunk .. + 7 of a row
template <int D>
__device__ __forceinline__ int stored_word(int chunk) {
    return (chunk & 3) * Tile<D>::kGroups + (chunk >> 2);
}

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Step of a group from the largest absolute value's bit pattern (as an unsigned integer: NaN is largest).
__device__ __forceinline__ float group_step(uint32_t amax_bits) {
    if (amax_bits >= 0x7B800000u) return __uint_as_float(0x7FC00000u);          // 2^120 and beyond, inf, NaN
    const uint32_t s = __float_as_uint(__fdiv_rn(__uint_as_float(amax_bits), 7.f));
    return __uint_as_float((s + 0x7FFFFu) & ~0x7FFFFu);
}

// Quantises eight bf16 values; the four lanes of an aligned quad hold the four chunks of a group.
// Every lane of the warp has to call it.
__device__ __forceinline__ uint32_t quantise8(const uint4 x, float &step) {
    float f[8];
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    step = group_step(amax);
    uint32_t w = 0;
    if (step >= kSmallStep) {
        // rint(x / s) by a product with 1 / s.  x / s = 2^n X / S with X below 2^8 and S from 16 to 31, so a quotient
        // between 1/4 and 7 either is a half-integer or lies at least 2^-11 away from one, while the product is
        // off by less than 2^-20: moved to the nearest multiple of 2^-13 (by adding and subtracting 1.5 2^10, whose last
        // bit is worth that) it is on the same side of every half-integer as the quotient, and on it if the
        // quotient is.  Adding 1.5 2^23 + 8 then rounds to an integer, ties to even, and leaves c in the low bits.
        const float inv = __frcp_rn(step);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = __fsub_rn(__fadd_rn(__fmul_rn(f[i], inv), 1536.f), 1536.f);
            w |= (__float_as_uint(__fadd_rn(y, 12582920.f)) & 15u) << (4 * i);
        }
    } else {
        // (1 / s would overflow; a step of zero or NaN: every code is 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int c = 8;
            if (step > 0.f) c = min(max(__float2int_rn(__fdiv_rn(f[i], step)) + 8, 1), 15);
            w |= (uint32_t)c << (4 * i);
        }
    }
    return w;
}

// Eight codes -> the bf16 pairs (e0, e4), (e1, e5), (e2, e6), (e3, e7) of 16 + c: the nibble goes to
// mantissa bits 3 .. 6 of 16.0, whose last bit is worth 1/8.
__device__ __forceinline__ void codes_to_bf16(uint32_t w, uint32_t (&r)[4]) {
    r[0] = ((w << 3) & 0x00780078u) | 0x41804180u;
    r[1] = ((w >> 1) & 0x00780078u) | 0x41804180u;
    r[2] = ((w >> 5) & 0x00780078u) | 0x41804180u;
    r[3] = ((w >> 9) & 0x00780078u) | 0x41804180u;
}

// (16 + c) s - 24 s = (c - 8) s in one fused operation: 24 s has seven significant bits and is exact in
// bf16, the fused product is exact and so is the result.
__device__ __forceinline__ uint32_t scale_pair(uint32_t v, uint32_t s2, uint32_t minus24s2) {
    __nv_bfloat162 a, b, c;
    *reinterpret_cast<uint32_t *>(&a) = v;
    *reinterpret_cast<uint32_t *>(&b) = s2;
    *reinterpret_cast<uint32_t *>(&c) = minus24s2;
    const __nv_bfloat162 d = __hfma2(a, b, c);
    return *reinterpret_cast<const uint32_t *>(&d);
}
__device__ __forceinline__ uint32_t minus24(uint32_t s2) {
    __nv_bfloat162 a;
    *reinterpret_cast<uint32_t *>(&a) = s2;
    const __nv_bfloat162 d = __hmul2(a, __floats2bfloat162_rn(-24.f, -24.f));
    return *reinterpret_cast<const uint32_t *>(&d);
}

// The eight bf16 values of a word, in order.
__device__ __forceinline__ uint4 dequantise8(uint32_t w, uint16_t step) {
    const uint32_t s2 = (uint32_t)step * 0x10001u, n2 = minus24(s2);
    uint32_t r[4];
    codes_to_bf16(w, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = scale_pair(r[i], s2, n2);
    return make_uint4(prmt(r[0], r[1], 0x5410), prmt(r[2], r[3], 0x5410), prmt(r[0], r[1], 0x7632), prmt(r[2], r[3], 0x7632));
}

}  // namespace kv4
}  // namespace ap
