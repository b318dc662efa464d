// What the kernels that attend over a pool held in 4 bits share: where a key lies, and codes as numbers.
#ifndef KVC_Q4_DEVICE_H
#define KVC_Q4_DEVICE_H

#include "kvc_attention.h"

// Codes as numbers, two a word.  Bits that lie in the lowest eight of a 16-bit float are a number as they stand: that many of
// the type's smallest, the step from the subnormal numbers to the first binade included.  So the codes in bits 0-3 of either
// half are that many times TINY, and those in bits 4-7 sixteen times as much: one instruction, and the matrix
// instructions, which take subnormal numbers for what they are, can have them.  A word's third and fourth pair are
// eight bits further up.
__device__ __forceinline__ uint32_t kvc_q4_low(uint32_t x) { return x & 0x000F000Fu; }
__device__ __forceinline__ uint32_t kvc_q4_high(uint32_t x) { return x & 0x00F000F0u; }

__device__ __forceinline__ uint32_t kvc_mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// And as values: offset + step * code, rounded once, of two groups a word.
// bf16: as many TINYs times a step that makes up for them, by fma: two instructions for two values.  The step has to stay
// in the type's range, so the values come out as SCALE of what they are, which their product's sums, of 32 bits, do
// not mind (values above 2^60 are none then, and differences below 2^-69 are lost).
// fp16's range is too small for that: the codes go under an exponent that makes them 1024 + code or 64 + code / 16, less that,
// which is exact, then fma.
template <typename T>
struct KvcQ4Values;
template <>
struct KvcQ4Values<__nv_bfloat16> {
    static constexpr float SCALE = 0x1p-64f;
    uint32_t low, high, offset;
    __device__ __forceinline__ KvcQ4Values(uint32_t step, uint32_t off)
        : low(kvc_mul_bf16x2(step, 0x62006200u)),    // 2^(133 - 64)
          high(kvc_mul_bf16x2(step, 0x60006000u)),   // 2^(129 - 64)
          offset(kvc_mul_bf16x2(off, 0x1F801F80u))   // 2^-64
    {
    }
    template <bool HIGH>
    __device__ __forceinline__ uint32_t of(uint32_t x) const
    {
        uint32_t r;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(HIGH ? kvc_q4_high(x) : kvc_q4_low(x)), "r"(HIGH ? high : low), "r"(offset));
        return r;
    }
};
template <>
struct KvcQ4Values<__half> {
    static constexpr float SCALE = 1.f;
    uint32_t step, offset;
    __device__ __forceinline__ KvcQ4Values(uint32_t s, uint32_t off) : step(s), offset(off) {}
    template <bool HIGH>
    __device__ __forceinline__ uint32_t of(uint32_t x) const
    {
        uint32_t r;
        if (HIGH)
            asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(kvc_q4_high(x) | 0x64006400u), "r"(0x2C002C00u), "r"(0xD400D400u));
        else
            asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(kvc_q4_low(x) | 0x64006400u), "r"(0x64006400u));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(r), "r"(step), "r"(offset));
        return r;
    }
};

#endif
