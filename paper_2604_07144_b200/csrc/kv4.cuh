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
constexpr uint32_t kHugeTop = 0x7B800000u, kSmallTop = 0x0E800000u;      // bits of 2^120, 2^-98

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

// Quantises eight bf16 values; the four lanes of an aligned quad hold the four chunks of a group.
// Every lane of the warp has to call it.  No division in the common case:
//   s    max |x| is m 2^e with m an integer from 128 to 255.  m (1 - 2^-16) / 7 lies below m / 7, and above every
//        number of five significant bits that m / 7 is above (m and 7 times such a number differ by a 255th or not at
//        all); where m / 7 is one itself, rounding up brings it back.  So rounding it up gives s.
//   c    x / s = 2^n X / S with X below 2^8 and S from 16 to 31, so a quotient between 1/4 and 7 either is a half-integer
//        or lies at least 2^-11 away from one.  x times the approximate 1 / s is off by less than 2^-19; added to
//        1.5 2^10, whose last bit is worth 2^-13, it becomes the multiple of 2^-13 that is on the same side of every
//        half-integer as the quotient, and on it if the quotient is.  A second addition moves it on to 1.5 2^23 + 8,
//        rounding to an integer with ties to even, and leaves c in the low bits.
__device__ __forceinline__ uint32_t quantise8(const uint4 x, float &step) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
    uint32_t top = __vmaxu2(__vmaxu2(u[0] & 0x7FFF7FFFu, u[1] & 0x7FFF7FFFu), __vmaxu2(u[2] & 0x7FFF7FFFu, u[3] & 0x7FFF7FFFu));
    top = max(top << 16, top & 0xFFFF0000u);                     // bits of max |x| (NaN is largest)
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
    auto round_up = [](float v) { return __uint_as_float((__float_as_uint(v) + 0x7FFFFu) & ~0x7FFFFu); };
    if (top - kSmallTop < kHugeTop - kSmallTop) {
        step = round_up(__fmul_rn(__uint_as_float(top), 0.14285496f));       // (1 - 2^-16) / 7
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
        uint32_t c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__fadd_rn(__fmaf_rn(f[i], inv, 1536.f), 12581384.f));
        // two codes a byte, four bytes a word
        const uint32_t b0 = c[1] * 16 + c[0], b1 = c[3] * 16 + c[2], b2 = c[5] * 16 + c[4], b3 = c[7] * 16 + c[6];
        return prmt(prmt(b0, b1, 0x0040), prmt(b2, b3, 0x0040), 0x5410);
    }
    // no step (zero or NaN), or one whose reciprocal might overflow
    uint32_t w = 0x88888888u;
    step = top >= kHugeTop ? __uint_as_float(0x7FC00000u) : round_up(__fdiv_rn(__uint_as_float(top), 7.f));
    if (step > 0.f) {
        w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint32_t)min(max(__float2int_rn(__fdiv_rn(f[i], step)) + 8, 1), 15) << (4 * i);
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
