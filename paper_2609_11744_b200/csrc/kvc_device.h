// Device helpers shared by the kernels that compute on the pool's elements.
#ifndef KVC_DEVICE_H
#define KVC_DEVICE_H

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

// Programmatic dependent launch: the grid may be scheduled while the stream's previous kernel
// drains; nothing in global memory is touched before this returns, and every block calls it, so a
// later kernel that waits for this one has waited for the earlier ones too.
__device__ __forceinline__ void kvc_pdl_wait()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// The same for a kernel that shares nothing with the one before it on the stream, and may run beside it
// (`beside`): the kernel before has itself waited for all that came earlier, and kvc_pdl_end() makes
// this one's end stand for the other's end too.  Every block calls both.
__device__ __forceinline__ void kvc_pdl_begin(uint32_t beside)
{
    if (!beside)
        asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void kvc_pdl_end(uint32_t beside)
{
    if (beside)
        asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <typename A>
inline cudaError_t kvc_launch_pdl(void (*kernel)(const A), const A &a, dim3 grid, uint32_t threads, uint32_t smem,
                                  cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Division by a number that is nearly always a power of two: `shift` is its logarithm, or KVC_NO_SHIFT.
// (An integer division is some 25 instructions, and the kernels have several between their start and
// their first load.)
#define KVC_NO_SHIFT 32u
inline uint32_t kvc_shift_of(uint32_t d)
{
    uint32_t s = 0;
    while (s < 31 && (1u << s) < d)
        ++s;
    return (1u << s) == d ? s : KVC_NO_SHIFT;
}
__device__ __forceinline__ uint32_t kvc_div(uint32_t x, uint32_t d, uint32_t shift)
{
    return shift != KVC_NO_SHIFT ? x >> shift : x / d;
}

// Two 32-bit floats in one 64-bit register pair, for the two-wide arithmetic.
__device__ __forceinline__ uint64_t kvc_pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 kvc_unpair(uint64_t v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t kvc_fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t kvc_add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ uint64_t kvc_mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Two 16-bit elements <-> two floats.
template <typename T>
__device__ __forceinline__ float2 kvc_to_float2(uint32_t v);
template <>
__device__ __forceinline__ float2 kvc_to_float2<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float2 kvc_to_float2<__half>(uint32_t v)
{
    __half2 h;
    memcpy(&h, &v, 4);
    return __half22float2(h);
}
template <typename T>
__device__ __forceinline__ uint32_t kvc_from_float2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t kvc_from_float2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    uint32_t v;
    memcpy(&v, &h, 4);
    return v;
}
template <>
__device__ __forceinline__ uint32_t kvc_from_float2<__half>(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    uint32_t v;
    memcpy(&v, &h, 4);
    return v;
}

#endif
