// What the kernels that attend over a pool held in 4 bits share: where a key lies, and codes as numbers.
#ifndef KVC_Q4_DEVICE_H
#define KVC_Q4_DEVICE_H

#include "kvc_attention.h"

// A key that is on its way: its position and its block's id, which nothing looks at until the copies are issued, so
// that the table's latency passes meanwhile.
struct KvcQ4Next {
    int32_t j;
    uint32_t id;
    bool asked;  // whether j is a key of the pair at all
};

__device__ __forceinline__ KvcQ4Next kvc_q4_look(const KvcAttn &a, const KvcSeq &q, const KvcRange &r, int32_t j)
{
    KvcQ4Next n;
    n.j = j;
    n.id = ~0u;
    n.asked = j < r.hi && (j >= r.lo || j < r.sink_end);
    if (n.asked)
        n.id = (uint32_t)a.tables[(int64_t)q.table * a.table_stride + kvc_div((uint32_t)j, a.block_size, a.block_shift)];
    return n;
}

__device__ __forceinline__ uint32_t kvc_bytes(uint32_t a, uint32_t b, uint32_t which)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(which));
    return r;
}
// The low and the high halves of two words.
__device__ __forceinline__ uint32_t kvc_lows(uint32_t a, uint32_t b) { return kvc_bytes(a, b, 0x5410u); }
__device__ __forceinline__ uint32_t kvc_highs(uint32_t a, uint32_t b) { return kvc_bytes(a, b, 0x7632u); }

// Codes as numbers, two a word.  Bits that lie in the lowest eight of a 16-bit float are a number as they stand: that many of
// the type's smallest, the step from the subnormal numbers to the first binade included.  So the codes in bits 0-3 of either
// half are that many times TINY, and those in bits 4-7 sixteen times as much: one instruction, and the matrix
// instructions, which take subnormal numbers for what they are, can have them.  A word's third and fourth pair are
// eight bits further up.
__device__ __forceinline__ uint32_t kvc_q4_low(uint32_t x) { return x & 0x000F000Fu; }
__device__ __forceinline__ uint32_t kvc_q4_high(uint32_t x) { return x & 0x00F000F0u; }

// And as values: offset + step * code, rounded once.  The codes are brought into the type's range first -- bf16: times a
// power of two, fp16 (whose range is too small for the step to make up for TINY): under an exponent that makes them 1024 + code
// or 64 + code / 16, less that -- which is exact, then fma.  `step` is kvc_q4_step's.
template <typename T>
__device__ __forceinline__ uint32_t kvc_q4_step(uint32_t step);
template <typename T, bool HIGH>
__device__ __forceinline__ uint32_t kvc_q4_code(uint32_t x);
template <typename T>
__device__ __forceinline__ uint32_t kvc_q4_value(uint32_t code, uint32_t step, uint32_t offset);

__device__ __forceinline__ uint32_t kvc_mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_step<__nv_bfloat16>(uint32_t step)
{
    return kvc_mul_bf16x2(step, 0x42804280u);  // 2^6
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_code<__nv_bfloat16, false>(uint32_t x)
{
    return kvc_mul_bf16x2(kvc_q4_low(x), 0x7F007F00u);  // 2^127 * 2^-133
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_code<__nv_bfloat16, true>(uint32_t x)
{
    return kvc_mul_bf16x2(kvc_q4_high(x), 0x7D007D00u);  // 2^123 * 2^-129
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_value<__nv_bfloat16>(uint32_t code, uint32_t step, uint32_t offset)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(code), "r"(step), "r"(offset));
    return r;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_step<__half>(uint32_t step)
{
    return step;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_code<__half, false>(uint32_t x)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(kvc_q4_low(x) | 0x64006400u), "r"(0x64006400u));
    return r;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_code<__half, true>(uint32_t x)
{
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(kvc_q4_high(x) | 0x64006400u), "r"(0x2C002C00u), "r"(0xD400D400u));
    return r;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_value<__half>(uint32_t code, uint32_t step, uint32_t offset)
{
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(code), "r"(step), "r"(offset));
    return r;
}

#endif
