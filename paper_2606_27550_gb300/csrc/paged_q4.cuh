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

// The scale byte of a group whose largest magnitude has the bits `top`.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    if (top >= 0x7f800000u)
        return kNanScaleByte;
    const float t = __fdiv_rn(__uint_as_float(top), 7.f);
    // up to 4 significant bits; below 2^-14 (byte 8) up to a multiple of 2^-17
    const uint32_t normal = ((__float_as_uint(t) + 0xfffffu) >> 20) - ((127 - 15) << 3);
    const uint32_t b = t > 0x1p-14f ? normal : (uint32_t)ceilf(t * 0x1p17f);
    return min(b, (uint32_t)kMaxScaleByte);
}

// Codes of 8 elements, the first in the lowest 4 bits; inv = 1 / s rounded (0 where s is 0).
__device__ __forceinline__ uint32_t quantize8(const float (&x)[8], float s, float inv)
{
    // adding 1.5 * 2^23 + 8 leaves rint(y) + 8 in the low bits, ties to even
    constexpr float kRound = 12582912.f + 8.f;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float y = fmaxf(fminf(x[i] * inv, 7.f), -7.f);
        float f = __fadd_rn(y, kRound);
        // x * inv is x / s but for its last bits: where those decide, the quotient itself
        if (fabsf(fabsf(__fsub_rn(y, __fsub_rn(f, kRound))) - 0.5f) < 1e-5f && s > 0.f) {
            y = fmaxf(fminf(__fdiv_rn(x[i], s), 7.f), -7.f);
            f = __fadd_rn(y, kRound);
        }
        w |= (__float_as_uint(f) & 15u) << (4 * i);
    }
    return w;
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

}  // namespace tv
