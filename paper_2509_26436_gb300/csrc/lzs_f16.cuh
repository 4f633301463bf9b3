// QuaRTZ codes as fp16 values without a conversion, for the attention kernels
// over encoded pages: a nibble with its sign bit flipped (c + 8) in the mantissa
// of a constant, and one fused multiply-add that takes the constant and 8 off
// and multiplies by 2^FLAG, exactly.
#pragma once

#include <cstdint>

namespace quartz {

__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// (x & mask) ^ flip in one instruction.
__device__ __forceinline__ uint32_t and_xor(uint32_t x, uint32_t mask, uint32_t flip)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(x), "r"(mask), "r"(flip));
    return d;
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// What a key's codes with FLAG F take: pairs of 2^F, 2^F / 16, -1032 2^F and
// -72 2^F (all exact; by fp16 products rather than integer sums, since the
// logic pipe is the busiest).
struct KeyFlag {
    uint32_t m0, m1, a0, a1;
    __device__ __forceinline__ explicit KeyFlag(uint32_t f)
    {
        m0 = f * 0x04000400u + 0x3C003C00u;
        m1 = mul_f16x2(m0, 0x2C002C00u);
        a0 = mul_f16x2(m0, 0xE408E408u);
        a1 = mul_f16x2(m0, 0xD480D480u);
    }
};

// The eight codes of a word (code k in bits 4k ..) times 2^F as fp16 pairs
// (k, k + 4): f = 1024 + (c + 8), or 1024 + 16 (c + 8) for the odd nibbles of
// each byte; f 2^F - 1032 2^F, f 2^F / 16 - 72 2^F.
__device__ __forceinline__ void key_codes(uint32_t w, const KeyFlag &f, uint32_t (&k)[4])
{
    const uint32_t w8 = w >> 8;
    k[0] = fma_f16x2(and_xor(w, 0x000F000Fu, 0x64086408u), f.m0, f.a0);
    k[1] = fma_f16x2(and_xor(w, 0x00F000F0u, 0x64806480u), f.m1, f.a1);
    k[2] = fma_f16x2(and_xor(w8, 0x000F000Fu, 0x64086408u), f.m0, f.a0);
    k[3] = fma_f16x2(and_xor(w8, 0x00F000F0u, 0x64806480u), f.m1, f.a1);
}

}  // namespace quartz
