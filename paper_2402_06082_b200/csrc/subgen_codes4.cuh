// Heads in 4 bits: 16 coordinates share a scale, a cell of 16 tokens holds codes and scales.
#pragma once
#include <cuda_fp16.h>
#include <stdint.h>

namespace sgk {

// A group is 16 consecutive coordinates of a head. S = the largest magnitude, rounded up to 4 significant bits (below 2^-14 to
// a multiple of 2^-17); code n = min(15, floor(8 x / S) + 8) stands for (n - 7.5) S / 8, so a coordinate is off by S / 16 at most.
// Why these: S has 4 significant bits and 2 n - 15 has 4, so every value is exact in bf16 and in fp16 (at most 8 bits, from 2^-21
// to 57600) and no product that the attention makes of it rounds the cache a second time. S is kept as the upper byte of the
// 15 bits that an fp16 has below its sign: 4.5 bits a value in all. A group whose largest magnitude is above 61440 or not
// finite has the byte 255, an fp16 NaN.
//
// A cell is what 16 tokens of a page have in one head: K codes [16][D / 2], K scales [16][D / 16], V codes, V scales: 2304 bytes at
// D = 128, one bulk copy. Eight coordinates are a 32-bit word, the even ones in the low half and the odd ones in the high
// half, each half rotated left by 2: three of the four pairs (c0 c1, c2 c3, ...) come into the top mantissa bits of two fp16 by
// one shift and one mask or a mask alone, the fourth by a byte permutation, and one fma takes the offset off and scales.
template <int D>
struct Cell4 {
    static constexpr int kCodes = D / 2, kScales = D / 16;           // bytes a token
    static constexpr int kHalf = 16 * (kCodes + kScales), kBytes = 2 * kHalf, kScaleAt = 16 * kCodes;
};

constexpr unsigned kMaxMagnitude4 = 0x47700000u;                     // 61440.f

// ---- rounding ----

// The scale byte of a group whose largest magnitude has the bits `top` (without sign; NaN counts as the largest).
__device__ __forceinline__ unsigned scale4(unsigned top) {
    if (top > kMaxMagnitude4) return 255u;
    if (top >= 0x38800000u) return ((top + 0xfffffu) >> 20) - (112u << 3);                  // 2^-14 and more
    return (unsigned)__float2int_ru(__uint_as_float(top) * 131072.f);                       // 2^17
}
// How a group is rounded: S / 8 = s4 2^-k with a whole s4 below 16, and floor(8 x / S) = floor(floor(2^k x) / s4), where 2^k x is exact, its
// floor comes with an fma that rounds down (to whole numbers, at 1.5 * 2^23) and a whole u = floor + 8 s4 <= 16 s4 is divided by s4
// by a product with m, up to 2 more than 2^16 / s4, and a shift: exact, since u * 2 / 2^16 < 1 / s4. The fma's result is taken as a
// whole number as it lies; `add` takes off what its exponent adds to the product.
struct Rounder4 {
    float factor, bias;
    uint32_t m, add;
    __device__ __forceinline__ explicit Rounder4(unsigned byte) {
        const unsigned e = byte >> 3, s4 = e ? 8 + (byte & 7) : byte ? byte : 1;             // a group of zeros: any s4
        factor = __uint_as_float((148u - (e ? e : 1)) << 23);
        bias = 12582912.f + 8.f * (float)s4;
        m = __float2uint_rz(__fdividef(65536.f, (float)s4)) + 1;
        add = 0u - 0x4b400000u * m;
    }
    __device__ __forceinline__ uint32_t operator()(float x) const {   // the code, 16 bits up
        return min(__float_as_uint(__fmaf_rd(x, factor, bias)) * m + add, 0xfffffu);
    }
};
// eight coordinates
__device__ __forceinline__ uint32_t word4(const float* x, const Rounder4& r) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int to = (i & 1) * 16 + (i >> 1) * 4;                  // its nibble before the rotation
        const uint32_t c = r(x[i]);
        w |= (to >= 16 ? c << (to - 16) : c >> (16 - to)) & (15u << to);
    }
    return ((w << 2) & 0xfffcfffcu) | ((w >> 14) & 0x00030003u);
}

// ---- reading ----
//
// Values come as fp16 pairs of value / 8: with S / 64 instead of S / 8 the offset 23.5 S / 64 of the fma below stays finite for all
// scales, and the smallest value (2^-24) is still an fp16.

//
// Logic, shifts and permutations share one pipe, 2 cycles each for a warp; fp16 pairs take the other, 2 cycles as well, where an integer
// multiply-add takes 1. So shifts to the left are products with a factor that the compiler does not see through (`opaque`).
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
    asm volatile("" : "+r"(x));
    return x;
}
// The constants of an expansion, in registers: as immediates mask and exponent would take two logic operations instead of one.
struct Consts4 {
    uint32_t f16, f128, f64k, mask, top;
    __device__ __forceinline__ Consts4() : f16(opaque(16u)), f128(opaque(128u)), f64k(opaque(65536u)), mask(opaque(0x03c003c0u)), top(opaque(0x4c004c00u)) {}
};

// S / 64 twice and -23.5 S / 64 twice, from S's byte in the low byte of both halves
__device__ __forceinline__ void scale_pair4(uint32_t bytes, const Consts4& c, __half2* s, __half2* o) {
    const uint32_t u = bytes * c.f128;
    const __half2 h = *reinterpret_cast<const __half2*>(&u);
    *s = __hmul2(h, __half2half2(__ushort_as_half(0x2400)));         // 2^-6
    *o = __hmul2(h, __half2half2(__ushort_as_half(0xb5e0)));         // -47 / 128
}
// Values / 8 of 8 codes x (or of 4 codes of each of two tokens): pair i = nibble i of both halves. 16 + n by the mantissa's top
// bits of an fp16 in [16, 32), then (16 + n) s - 23.5 s, which is exact. Nibbles 0 and 2 lie 4 bits below their place, 2 and 3
// after the bytes of each half have changed places.
__device__ __forceinline__ void pairs4(uint32_t x, __half2 s, __half2 o, const Consts4& c, uint32_t* v) {
    const uint32_t y = __byte_perm(x, 0, 0x2301);
    const uint32_t n[4] = {x * c.f16, x, y * c.f16, y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t e;
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(e) : "r"(n[i]), "r"(c.mask), "r"(c.top));       // (n & mask) | top
        const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&e), s, o);
        v[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
}

// The same as bf16 pairs of the value itself: 16 + n in [16, 32), - 23.5, times S / 8; each exact.
struct Consts4Bf16 {
    uint32_t f2, mask, top;
    __device__ __forceinline__ Consts4Bf16() : f2(opaque(2u)), mask(opaque(0x00780078u)), top(opaque(0x41804180u)) {}
};
// S / 8 twice, of bytes k and k + 1 of `bytes`
__device__ __forceinline__ void scale_bf16_4(uint32_t bytes, unsigned k, uint32_t* s) {
    const uint32_t u = __byte_perm(bytes, 0, 0x0404u + (k << 4) + ((k + 1) << 12)) >> 1;
    const float2 f = __half22float2(__hmul2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x3000))));      // 2^-3
    s[0] = __byte_perm(__float_as_uint(f.x), 0, 0x3232);
    s[1] = __byte_perm(__float_as_uint(f.y), 0, 0x3232);
}
__device__ __forceinline__ void pairs4_bf16(uint32_t x, uint32_t s, const Consts4Bf16& c, uint32_t* v) {
    const uint32_t y = __byte_perm(x, 0, 0x2301);
    const uint32_t n[4] = {x * c.f2, x >> 3, y * c.f2, y >> 3};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t e;
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(e) : "r"(n[i]), "r"(c.mask), "r"(c.top));
        asm("{\n\t.reg .b32 z;\n\tadd.rn.bf16x2 z, %1, %2;\n\tmul.rn.bf16x2 %0, z, %3;\n\t}\n" : "=r"(v[i]) : "r"(e), "r"(0xc1bcc1bcu), "r"(s));
    }
}

}  // namespace sgk
