// paged_q4.cuh -- rows in 4 bits, as the calls over 4-bit pages share them.
//
// 32 consecutive elements of a head's row share a scale s (one byte: bits 7 to 14
// of the fp16 number s) and an element is (c - 8) s with a 4-bit code c.  c - 8 has
// 3 bits and s has 4, so that the product has at most 7: exact in bf16 and, since
// s is 9216 at most and a multiple of 2^-17, in fp16.  Nothing is rounded between
// the pages and the tensor cores.
#pragma once

#include "paged.cuh"

namespace tv {

constexpr int kGroup = 32;          // elements of a scale
constexpr int kMaxScaleByte = 225;  // 9216; 7 * 9216 is finite in fp16
constexpr int kNanScaleByte = 255;

__host__ __device__ constexpr int code_bytes(int d)
{
    return d / 2;
}
__host__ __device__ constexpr int scale_bytes(int d)
{
    return d / kGroup;
}
// of a slot: its codes and its scales
__host__ __device__ constexpr int row_bytes(int d)
{
    return code_bytes(d) + scale_bytes(d);
}

__device__ __forceinline__ float scale_of(uint32_t byte)
{
    return __half2float(__ushort_as_half((unsigned short)(byte << 7)));
}

// fl(x / n) for a number n of at most 4 significant bits and its reciprocal to one unit in the last place: a
// product and one correction.  y = fl(x inv) is x / n (1 + e) with |e| <= 2^-22, its remainder x - y n is a
// float (a few units of y's last place times n's), and y plus remainder times inv is x / n but for e^2 and
// e 2^-23, 2^-43 of it, before the one rounding.  That cannot round otherwise than x / n does: a midpoint
// between two floats has 25 bits, times n 29, so that x (24 bits) is never n times a midpoint, and never nearer
// to one than 2^-29.
__device__ __forceinline__ uint64_t quotient_two(uint64_t x, uint64_t minus_n, uint64_t inv)
{
    const uint64_t y = mul_two(x, inv);
    return fma_two(fma_two(y, minus_n, x), inv, y);
}

// The scale byte of a group whose largest magnitude is `top` (NaN if one of it is none).
__device__ __forceinline__ uint32_t scale_byte(float top)
{
    constexpr float kInv = 1.f / 7.f;
    const float y = __fmul_rn(top, kInv), t = __fmaf_rn(__fmaf_rn(y, -7.f, top), kInv, y);  // as above
    // up to 4 significant bits; below 2^-14 (byte 8) up to a multiple of 2^-17, which are the 4 bits of the
    // sum with 2^-14 (rounded up, which changes nothing about that)
    const bool small = !(t > 0x1p-14f);
    const float u = small ? __fadd_ru(t, 0x1p-14f) : t;
    const uint32_t b = ((__float_as_uint(u) + 0xfffffu) >> 20) - (((small ? 128 : 127) - 15) << 3);
    return top < INFINITY ? min(b, (uint32_t)kMaxScaleByte) : (uint32_t)kNanScaleByte;
}

// Codes of 8 elements (pairs), the first in the lowest 4 bits; inv = 1 / s as quotient_two wants it (0 where s
// is 0); clamp: s may be the largest scale or NaN.
__device__ __forceinline__ uint32_t quantize8(const uint64_t (&x)[4], float s, float inv, bool clamp)
{
    // adding 1.5 * 2^23 + 8 leaves rint(y) + 8, at most 15, in the lowest byte, ties to even
    constexpr float kRound = 12582912.f + 8.f;
    uint32_t b[4];  // two codes each
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint64_t y = quotient_two(x[i], two(-s, -s), two(inv, inv));
        if (clamp) {  // some scale is the largest one, or NaN (which gives 7)
            const float2 f = halves(y);
            y = two(fmaxf(fminf(f.x, 7.f), -7.f), fmaxf(fminf(f.y, 7.f), -7.f));
        }
        const float2 f = halves(add_two(y, two(kRound, kRound)));
        b[i] = (__float_as_uint(f.y) << 4) + __float_as_uint(f.x);  // (of which the lowest byte)
    }
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

// 16-bit pairs.  In bf16 128 + c is 0x4300 | c, and (128 + c) s - 136 s is (c - 8) s,
// whose one rounding changes nothing (136 s = 17 * 8 s has 8 bits).  In fp16 1024 + c
// is 0x6400 | c; c - 8 first, since 1032 s may pass the largest number.
template <bool kF16>
struct Scale {
    uint32_t s, bias;  // bf16: s and -136 s, each twice; fp16: s twice
};

template <bool kF16>
__device__ __forceinline__ Scale<kF16> scale_pair(float lo, float hi)
{
    Scale<kF16> r;
    r.s = pack_pair<kF16>(lo, hi);
    if constexpr (kF16)
        r.bias = 0xe408e408u;  // -1032
    else
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r.bias) : "r"(r.s), "r"(0xc308c308u));  // * -136
    return r;
}

// The elements whose codes are bits 0 to 3 and 16 to 19 of w.
template <bool kF16>
__device__ __forceinline__ uint32_t dequant_pair(uint32_t w, const Scale<kF16> &s)
{
    uint32_t x, y;
    if constexpr (kF16) {
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w), "r"(0x000f000fu), "r"(0x64006400u));  // (w & m) | base
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(s.bias));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(x) : "r"(y), "r"(s.s));
        return x;
    } else {
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w), "r"(0x000f000fu), "r"(0x43004300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(y) : "r"(x), "r"(s.s), "r"(s.bias));
        return y;
    }
}

// ---- for the products of the attention: all the elements times one power of two
//
// In bf16 the numbers with bits 0 to 7 are k 2^-133, below the smallest normal number and
// one binade above it.  So the code in bits 0 to 3 is c 2^-133 and the one in bits 4 to 7
// 16 c 2^-133 as they stand, and an fma with s 2^113 (s 2^109) and -8 s 2^-20 makes
// (c - 8) s 2^-20 of them, exactly: one shift for four codes.  fp16 has no room for that:
// c - 8 first, then s.
template <bool kF16>
constexpr float kOperandScale = kF16 ? 1.f : 0x1p-20f;

template <bool kF16>
struct OperandScale {
    uint32_t low, high, bias;  // fp16: low alone, s
};

template <bool kF16>
__device__ __forceinline__ OperandScale<kF16> operand_scale(float lo, float hi)
{
    OperandScale<kF16> r;
    if constexpr (kF16) {
        r.low = pack_pair<true>(lo, hi);
        r.high = r.bias = 0;
    } else {
        const uint32_t s = pack_pair<false>(lo, hi);
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r.low) : "r"(s), "r"(0x78007800u));   // 2^113
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r.high) : "r"(s), "r"(0x76007600u));  // 2^109
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r.bias) : "r"(s), "r"(0xb700b700u));  // -2^-17
    }
    return r;
}

// The elements whose codes stand at bits 0, 4, 8 and 12 of both halves of w.
template <bool kF16>
__device__ __forceinline__ void dequant_four(uint32_t w, const OperandScale<kF16> &s, uint32_t (&e)[4])
{
    const uint32_t v = w >> 8;
    if constexpr (kF16) {
        uint32_t x[4];
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[0]) : "r"(w), "r"(0x000f000fu), "r"(0x64006400u));
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[1]) : "r"(w), "r"(0x00f000f0u), "r"(0x64006400u));
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[2]) : "r"(v), "r"(0x000f000fu), "r"(0x64006400u));
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[3]) : "r"(v), "r"(0x00f000f0u), "r"(0x64006400u));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i % 2 == 0)
                asm("add.rn.f16x2 %0, %1, %2;" : "=r"(x[i]) : "r"(x[i]), "r"(0xe408e408u));  // 1024 + c - 1032
            else
                asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(x[i]) : "r"(x[i]), "r"(0x2c002c00u), "r"(0xd480d480u));  // / 16 - 72
            asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(e[i]) : "r"(x[i]), "r"(s.low));
        }
    } else {
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(e[0]) : "r"(w & 0x000f000fu), "r"(s.low), "r"(s.bias));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(e[1]) : "r"(w & 0x00f000f0u), "r"(s.high), "r"(s.bias));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(e[2]) : "r"(v & 0x000f000fu), "r"(s.low), "r"(s.bias));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(e[3]) : "r"(v & 0x00f000f0u), "r"(s.high), "r"(s.bias));
    }
}

}  // namespace tv
