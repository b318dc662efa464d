// Attention over the paged pool for few query rows (decode): at most 16 rows share a KV head's keys.
//
// Per row: s_j = scale * q . k_j over the keys it sees, o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m).
// One pass over K and V with the running maximum m and sum of a softmax, in 32 bits and base 2; the
// weights are rounded to the pool's type for the second product only, whose instruction takes 16-bit operands of one
// type (the sum is taken before that).  Against 64 bits the result is off by 0.0021 in bf16 (0.0017 with weights in 32
// bits: the result's own rounding).
//
// Bound by memory: 2 * D * 2 bytes per key and KV head against 4 * D * 16 operations -- far below
// what even mma.sync offers, so the tensor work is small and the kernel is built around loads in
// flight.  A block is four warps; each walks its own 16 keys of every 64-key tile through its own
// ring of shared-memory stages filled by 16-byte asynchronous copies, with its own running maximum
// and sum, so nothing but the end of a pair needs a block-wide barrier.  Measured: 64 requests of 128 to
// 32768 tokens (64 and 8 heads of 128), 827 MB of keys and values, in 131 us = 6.3 TB/s.  The ring runs ahead of the
// arithmetic across pairs: the load cursor walks the same units as the compute cursor.
#include "kvc_attention.h"

namespace {

constexpr int WARPS = 4;
constexpr int THREADS = WARPS * 32;
constexpr int TK = 64;             // keys per unit
constexpr int WK = TK / WARPS;     // keys per warp and unit
constexpr int ROWS = KVC_ATTN_SMALL_ROWS;
constexpr int HEAD = 1;            // what a pair costs besides its units, in units
constexpr int LEAST = 2;           // units of a run at least

template <int D>
struct Shape {
    static constexpr int ROW = D * 2;                // bytes of a key
    static constexpr int CHUNKS = ROW / 16;          // 16-byte pieces of a key
    static constexpr int STAGE = 2 * WK * ROW;       // K and V of one warp's share of a unit
    static constexpr int STAGES = D == 128 ? 2 : 4;  // 64 KiB a block, two blocks a SM (three and six: the same rate, a longer start)
    static constexpr int MERGE = 2 * ROWS * D * 4;   // two warps' sums
    static constexpr int SMEM = WARPS * STAGES * STAGE + MERGE;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Where this lane's key of the cursor's unit lies, or -1; lanes 16 and up the same keys again.
template <int D>
__device__ __forceinline__ int64_t look_up(const KvcAttn &a, const KvcCursor &c, uint32_t warp, uint32_t lane)
{
    const int32_t j = (int32_t)(kvc_tile(c.r, c.t) * TK + warp * WK + (lane & 15u));
    int64_t off = -1;
    if (j < c.r.hi && (j >= c.r.lo || j < c.r.sink_end)) {
        off = kvc_key_offset(a, c.q.table, j, c.h, Shape<D>::ROW);
        if (off < 0 && lane < 16)
            atomicAdd(a.status, 1u);
    }
    return off;
}

// Issues the copies of this warp's keys of one unit; returns which of the 16 are there.
template <int D>
__device__ __forceinline__ uint32_t load_unit(const KvcAttn &a, int64_t off, uint32_t lane, uint32_t stage)
{
    using S = Shape<D>;
    const uint32_t there = __ballot_sync(~0u, off >= 0) & 0xFFFFu;
    constexpr int PER = 32 / S::CHUNKS;  // keys per round
    const uint32_t chunk = lane % S::CHUNKS, sub = lane / S::CHUNKS;
#pragma unroll
    for (int i = 0; i < WK / PER; ++i) {
        const uint32_t row = i * PER + sub;
        const int64_t o = __shfl_sync(~0u, off, row);
        const uint32_t bytes = o >= 0 ? 16u : 0u;  // 0: the destination is filled with zeros
        const uint64_t at = (o >= 0 ? (uint64_t)o : 0ull) + chunk * 16u;
        // 16-byte pieces are swapped within a row by its number so that eight rows' pieces of one
        // column, which a matrix load reads together, lie in different banks
        const uint32_t dst = stage + row * S::ROW + ((chunk ^ (row & 7u)) << 4);
        copy16(dst, a.k + at, bytes);
        copy16(dst + WK * S::ROW, a.v + at, bytes);
    }
    return there;
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 2) kvc_attn_rows_kernel(const KvcAttn a)
{
    using S = Shape<D>;
    constexpr int KS = D / 16;  // steps along the head, and 16-wide column tiles of the output
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint32_t s_there[WARPS][S::STAGES];
    __shared__ float s_m[WARPS][ROWS], s_l[WARPS][ROWS];
    kvc_pdl_begin(a.beside);

    const uint32_t n_seq = a.phase == KVC_PHASE_PREFIX ? a.n_groups : a.n_requests;
    const KvcRun run = kvc_find_run<ROWS, TK, HEAD, LEAST, THREADS>(a, n_seq);
    if (!run.any) {
        kvc_pdl_end(a.beside);
        return;
    }
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t ring = smem_addr(smem) + warp * S::STAGES * S::STAGE;
    float *merge = reinterpret_cast<float *>(smem + WARPS * S::STAGES * S::STAGE);
    const uint32_t gr = lane >> 2, gc = lane & 3u;  // row and column pair of an accumulator

    KvcCursor ld = run.at, c = run.at;
    unsigned long long ld_at = run.units_at, units_at = run.units_at;  // where their pairs' units lie on the line
    uint32_t pair = run.pair;
    // the load cursor's unit, if it is in the run, and one step on.  Places are looked up a unit ahead, so
    // that the table's latency and the copies' follow one another only once
    bool more = true;
    int64_t off = look_up<D>(a, ld, warp, lane);
    const auto load = [&](uint32_t stage) {
        if (more) {
            const int64_t now = off;
            const uint32_t n = ld.r.n;
            kvc_next<ROWS, TK>(a, n_seq, ld);
            if (ld.t == 0)
                ld_at += n + HEAD;
            more = ld.s < n_seq && ld_at + ld.t < run.end;
            if (more)
                off = look_up<D>(a, ld, warp, lane);
            const uint32_t there = load_unit<D>(a, now, lane, ring + stage * S::STAGE);
            if (lane == 0)
                s_there[warp][stage] = there;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (uint32_t i = 0; i < S::STAGES - 1; ++i)
        load(i);
    uint32_t stage = 0;

    for (uint32_t n_units; c.s < n_seq && (n_units = run.count(c, units_at)) != 0;) {
        // ---- a new pair (or the rest of one): its queries as matrix operands, 16 rows x D
        const uint32_t row0 = c.rt * ROWS, rows = min((uint32_t)ROWS, (uint32_t)c.q.rows - row0);
        uint32_t qf[KS][4];
        int32_t pos[2];
        const bool real[2] = {gr < rows, gr + 8 < rows};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t row = row0 + gr + 8 * half, tok = kvc_div_g(a, row);
            const unsigned char *src = a.q;
            pos[half] = -1;
            if (real[half]) {
                pos[half] = kvc_row_pos(a, c.q, row);
                src += (int64_t)(c.q.qa + (int32_t)tok) * a.q_tok + (int64_t)(c.h * a.g + (row - tok * a.g)) * a.q_head;
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qf[k][half] = real[half] ? *reinterpret_cast<const uint32_t *>(src + k * 32 + gc * 4) : 0u;
                qf[k][2 + half] = real[half] ? *reinterpret_cast<const uint32_t *>(src + k * 32 + 16 + gc * 4) : 0u;
            }
        }
        float o[2 * KS][4];
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n)
            o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        const bool from_start = c.t == 0;
        const bool to_end = c.t + n_units == c.r.n;

        for (uint32_t i = 0; i < n_units; ++i) {
            // the stage that the previous unit used is free once every lane is past its reads
            __syncwarp();
            load(stage == 0 ? S::STAGES - 1 : stage - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
            __syncwarp();

            const uint32_t kb = ring + stage * S::STAGE, vb = kb + WK * S::ROW;
            const uint32_t there = s_there[warp][stage];
            const int32_t j0 = (int32_t)(kvc_tile(c.r, c.t + i) * TK + warp * WK);
            if (there != 0) {
                float s[2][4] = {};
                const uint32_t krow = (lane & 7u) + ((lane >> 4) << 3), kc = (lane >> 3) & 1u;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t b[4];
                    ldsm4(b, kb + krow * S::ROW + (((k * 2 + kc) ^ (krow & 7u)) << 4));
                    mma<T>(s[0], qf[k], b[0], b[1]);
                    mma<T>(s[1], qf[k], b[2], b[3]);
                }
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = n * 8 + (int)gc * 2 + (e & 1);
                        const bool see = (there >> key & 1u) && kvc_sees(a, pos[e >> 1], j0 + key);
                        s[n][e] = see ? s[n][e] * a.scale_log2 : -INFINITY;
                        top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
                    }
                float base[2];
                bool moved = false;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    top[half] = fmaxf(top[half], __shfl_xor_sync(~0u, top[half], 1));
                    top[half] = fmaxf(top[half], __shfl_xor_sync(~0u, top[half], 2));
                    moved |= top[half] > m[half];
                }
                if (__any_sync(~0u, moved)) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const float now = fmaxf(m[half], top[half]);
                        const float f = m[half] == -INFINITY ? 0.f : exp2f(m[half] - now);
                        m[half] = now;
                        l[half] *= f;
#pragma unroll
                        for (int n = 0; n < 2 * KS; ++n) {
                            o[n][2 * half] *= f;
                            o[n][2 * half + 1] *= f;
                        }
                    }
                }
                base[0] = m[0] == -INFINITY ? 0.f : m[0];
                base[1] = m[1] == -INFINITY ? 0.f : m[1];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[n][e] = exp2f(s[n][e] - base[e >> 1]);
                        l[e >> 1] += s[n][e];
                    }
                const uint32_t p[4] = {kvc_from_float2<T>(s[0][0], s[0][1]), kvc_from_float2<T>(s[0][2], s[0][3]),
                                       kvc_from_float2<T>(s[1][0], s[1][1]), kvc_from_float2<T>(s[1][2], s[1][3])};
                const uint32_t vrow = (lane & 7u) + (((lane >> 3) & 1u) << 3), vc = lane >> 4;
#pragma unroll
                for (int n = 0; n < KS; ++n) {
                    uint32_t b[4];
                    ldsm4t(b, vb + vrow * S::ROW + (((n * 2 + vc) ^ (vrow & 7u)) << 4));
                    mma<T>(o[2 * n], p, b[0], b[1]);
                    mma<T>(o[2 * n + 1], p, b[2], b[3]);
                }
            }
            stage = stage == S::STAGES - 1 ? 0 : stage + 1;
        }

        // ---- end of the pair, or of the run: join the four warps' parts
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(~0u, l[half], 1);
            l[half] += __shfl_xor_sync(~0u, l[half], 2);
        }
        __syncthreads();  // the join before this one is over
        if (gc == 0) {
            s_m[warp][gr] = m[0];
            s_m[warp][gr + 8] = m[1];
            s_l[warp][gr] = l[0];
            s_l[warp][gr + 8] = l[1];
        }
        __syncthreads();
        float tm[2], tl[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t row = gr + 8 * half;
            tm[half] = s_m[0][row];
#pragma unroll
            for (int w = 1; w < WARPS; ++w)
                tm[half] = fmaxf(tm[half], s_m[w][row]);
            const float ref = tm[half] == -INFINITY ? 0.f : tm[half];
            tl[half] = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w)
                tl[half] += s_l[w][row] * exp2f(s_m[w][row] - ref);
            const float f = exp2f(m[half] - ref);
#pragma unroll
            for (int n = 0; n < 2 * KS; ++n) {
                o[n][2 * half] *= f;
                o[n][2 * half + 1] *= f;
            }
        }
        // 3 + 2 -> 1 + 0 -> 0, each lane reading back the places that its partner's lane wrote
#pragma unroll
        for (uint32_t step = 2; step; step /= 2) {
            if (warp >= step && warp < 2 * step) {
                float4 *dst = reinterpret_cast<float4 *>(merge) + (warp - step) * (ROWS * D / 4) + lane;
#pragma unroll
                for (int n = 0; n < 2 * KS; ++n)
                    dst[n * 32] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
            }
            __syncthreads();
            if (warp < step) {
                const float4 *src = reinterpret_cast<const float4 *>(merge) + warp * (ROWS * D / 4) + lane;
#pragma unroll
                for (int n = 0; n < 2 * KS; ++n) {
                    const float4 v = src[n * 32];
                    o[n][0] += v.x;
                    o[n][1] += v.y;
                    o[n][2] += v.z;
                    o[n][3] += v.w;
                }
            }
            if (step > 1)
                __syncthreads();
        }
        if (warp == 0) {
            if (a.phase == KVC_PHASE_WHOLE && from_start && to_end) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (real[half]) {
                        const uint32_t row = row0 + gr + 8 * half, t = kvc_div_g(a, row);
                        const int64_t tok = c.q.qa + (int32_t)t;
                        const uint32_t head = c.h * a.g + (row - t * a.g);
                        const float inv = tl[half] == 0.f ? 0.f : 1.f / tl[half];  // a row that sees nothing: zeros
                        unsigned char *dst = a.out + tok * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
                        for (int n = 0; n < 2 * KS; ++n)
                            *reinterpret_cast<uint32_t *>(dst + n * 16 + gc * 4) =
                                kvc_from_float2<T>(o[n][2 * half] * inv, o[n][2 * half + 1] * inv);
                        if (a.lse && gc == 0)
                            a.lse[tok * a.hq + head] = (tm[half] + log2f(tl[half])) * 0.693147180559945309f;
                    }
            } else if (a.phase == KVC_PHASE_WHOLE || pair < a.parts.max_pairs) {
                const uint64_t slot = a.phase == KVC_PHASE_WHOLE ? 2ull * blockIdx.x + (from_start ? 1 : 0)
                                                                 : (uint64_t)blockIdx.x + pair;
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (real[half]) {
                        const uint64_t at = slot * ROWS + gr + 8 * half;
#pragma unroll
                        for (int n = 0; n < 2 * KS; ++n)
                            *reinterpret_cast<float2 *>(a.parts.o + at * D + n * 8 + gc * 2) =
                                make_float2(o[n][2 * half], o[n][2 * half + 1]);
                        if (gc == 0)
                            a.parts.ml[at] = make_float2(tm[half], tl[half]);
                    }
                if (a.phase != KVC_PHASE_WHOLE && from_start && lane == 0)
                    a.parts.range[pair] = make_ulonglong2(units_at, units_at + c.r.n);
            }
        }
        if (to_end) {
            units_at += c.r.n + HEAD;
            ++pair;
        }
        c.t += n_units - 1;
        kvc_next<ROWS, TK>(a, n_seq, c);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    kvc_pdl_end(a.beside);
}

template <typename T, int D>
cudaError_t launch(const KvcAttn &a, uint32_t blocks, cudaStream_t st)
{
    const cudaError_t e = cudaFuncSetAttribute(kvc_attn_rows_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               Shape<D>::SMEM);
    if (e != cudaSuccess)
        return e;
    return kvc_launch_pdl(kvc_attn_rows_kernel<T, D>, a, dim3(blocks), THREADS, Shape<D>::SMEM, st);
}

}  // namespace

// Two blocks a SM.  Beside a shared prefix, whose blocks hold some SMs for a part of the time, three, so that
// equal runs still end together (64 requests on a 1024-token prefix: 88 us with two, 76 with three, 86 with four).
uint32_t kvc_attn_rows_blocks(const kvc_layout *lay, bool shared) { return (shared ? 3u : 2u) * (uint32_t)lay->sm_count; }

cudaError_t kvc_launch_attn_rows(const KvcAttn &a, uint32_t dtype, uint32_t head_dim, uint32_t blocks, cudaStream_t st)
{
    if (dtype == KVC_DTYPE_BF16)
        return head_dim == 128 ? launch<__nv_bfloat16, 128>(a, blocks, st) : launch<__nv_bfloat16, 64>(a, blocks, st);
    return head_dim == 128 ? launch<__half, 128>(a, blocks, st) : launch<__half, 64>(a, blocks, st);
}
