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

// A key's codes relative to its plane's base (negative: not there), and its scales relative to them.
struct KvcQ4Key {
    int64_t codes;
    uint32_t scales;
};

template <int D>
__device__ __forceinline__ KvcQ4Key kvc_q4_key(const KvcAttn &a, const KvcQ4Next &n, uint32_t h)
{
    KvcQ4Key k;
    k.codes = -1;
    k.scales = 0;
    if (n.id < a.num_blocks) {
        const uint32_t in = (uint32_t)n.j - kvc_div((uint32_t)n.j, a.block_size, a.block_shift) * a.block_size;
        k.codes = (int64_t)((uint64_t)n.id * a.block_stride + (uint64_t)h * a.block_size * KVC_Q4_ROW_BYTES(D) + in * (D / 2u));
        k.scales = a.block_size * (D / 2u) - in * (D / 2u - D / 8u);
    }
    return k;
}

// Codes as numbers.  The low four bits of either half of a word, put under an exponent whose last place is one, are
// that power of two (BIAS) plus the code: two codes an instruction.  (bf16's 7 bits behind the point reach to 128.)
template <typename T>
struct KvcQ4;
template <>
struct KvcQ4<__nv_bfloat16> {
    static constexpr uint32_t EXPONENT = 0x43004300u;
    static constexpr float BIAS = 128.f;
};
template <>
struct KvcQ4<__half> {
    static constexpr uint32_t EXPONENT = 0x64006400u;
    static constexpr float BIAS = 1024.f;
};

__device__ __forceinline__ uint32_t kvc_bytes(uint32_t a, uint32_t b, uint32_t which)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(which));
    return r;
}
// The low and the high halves of two words.
__device__ __forceinline__ uint32_t kvc_lows(uint32_t a, uint32_t b) { return kvc_bytes(a, b, 0x5410u); }
__device__ __forceinline__ uint32_t kvc_highs(uint32_t a, uint32_t b) { return kvc_bytes(a, b, 0x7632u); }

// BIAS + code of the low four bits of either half.
template <typename T>
__device__ __forceinline__ uint32_t kvc_q4_biased(uint32_t x)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(r) : "r"(x), "n"(KvcQ4<T>::EXPONENT));
    return r;
}
// Without the bias: exact.
template <typename T>
__device__ __forceinline__ uint32_t kvc_q4_plain(uint32_t biased);
template <>
__device__ __forceinline__ uint32_t kvc_q4_plain<__nv_bfloat16>(uint32_t biased)
{
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(biased), "r"(KvcQ4<__nv_bfloat16>::EXPONENT));
    return r;
}
template <>
__device__ __forceinline__ uint32_t kvc_q4_plain<__half>(uint32_t biased)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(biased), "r"(KvcQ4<__half>::EXPONENT));
    return r;
}
// offset + step * code, rounded once.
template <typename T>
__device__ __forceinline__ uint32_t kvc_q4_value(uint32_t code, uint32_t step, uint32_t offset);
template <>
__device__ __forceinline__ uint32_t kvc_q4_value<__nv_bfloat16>(uint32_t code, uint32_t step, uint32_t offset)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(code), "r"(step), "r"(offset));
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
