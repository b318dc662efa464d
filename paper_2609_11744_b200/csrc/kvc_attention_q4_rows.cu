// Attention over a pool held in 4 bits for few query rows (decode): at most 16 rows share a KV head's keys.
//
// The mathematics of kvc_attention_rows.cu: one pass with the running maximum and sum of a softmax, in 32 bits and base
// 2.  What differs is where the values come from.  With codes c, step s and offset f of each group of 32,
//     q . k = sum over groups of (s * sum_d q_d c_d + f * sum_d q_d):
// the codes are exact in the model's 16-bit type, so the first product runs on them, the steps multiply its 32-bit sums,
// four a key, and offsets times sums of the query are a product of their own with the sums in three parts, which hold all
// of their bits.  (Each query row comes times a power of two of its own, so that small ones are none of the type's smallest
// numbers.)  The sum of values is over keys, each with its own step, so there a step would have to go into the weights, an
// operand for each group; instead values become f + s * c in that type (rounded once, as a 16-bit pool would hold
// them).  Against 64 bits the result is off by 0.0027 in bf16 and 0.0003 in fp16: the values' rounding, the weights' (the matrix unit takes 16-bit operands of one type) and
// the result's own, 0.0017.
//
// Keys are the rows of the matrix instruction and queries its columns (16 x 8), since a KV head has 4 or 8 queries where
// one token is decoded: no half of a product is wasted, and a code made into a number serves all columns.  Any order of
// the head's values does for a product as long as both operands have it, so a word of eight codes is taken as
// the pairs (0,4) (1,5) (2,6) (3,7) that its two halves hold side by side: an instruction for two codes.  For
// values the pairs are two keys, from the halves of two keys' words.  Scores go from accumulator to operand
// through a transposition of 8 x 8 in registers.
//
// A block is four warps, each with its own 32 keys of every 128-key unit and its own ring of three stages filled by
// asynchronous copies; the run of units that a block has, parts and joins are kvc_attention.h's.  A unit's weighted sum of
// values is made beside the next unit's scores.  Measured: 64 requests of 128 to 32768 tokens (64 and 8 heads of 128), 282 MB
// of codes and scales, in 86 us with the join (16-bit pool: 146); 16 requests of 80,000, 1.64 GB, in 376 us = 4.4 TB/s.
// Bound by what a warp does for its keys, some 650 instructions a unit at 0.6 an issue slot: with three blocks a SM no unit
// waits for its copies, and without the copies the call takes 7 % less.  Four blocks with two stages and 128 registers
// (no such overlap): 92 us; keys in units of 64: 101; blocks of eight or sixteen warps: 97 and 123.
#include "kvc_q4_device.h"

namespace {

constexpr int WARPS = 4;
constexpr int THREADS = WARPS * 32;
constexpr int WK = 32;             // keys per warp and unit
constexpr int TK = WK * WARPS;     // keys per unit
constexpr int KT = WK / 16;        // key tiles of the matrix instruction
constexpr int HEAD = 2;            // what a pair costs besides its units, in units (64 decode requests: 93, 86, 88, 91 us with 1 to 4)
constexpr int LEAST = 2;           // units of a run at least (one request of 8192: 18.1, 17.5, 17.1 us with 1 to 3; 32 on a 32,000-token prefix 58, 58, 62)

template <int D, int NT>
struct Shape {
    static constexpr int ROWS = 8 * NT;
    static constexpr int GROUPS = D / 32;
    static constexpr int CODES = D / 2;              // bytes of a key's codes
    static constexpr int SCALES = D / 8;             // and of its steps and offsets, which lie behind them
    static constexpr int PITCH = D == 128 ? 80 : 48;  // of a key in shared memory: eight keys' words in different banks
    static constexpr int STAGE = 2 * WK * PITCH;     // K and V of one warp's share of a unit
    static constexpr int STAGES = 3;                 // one that is loaded, one whose keys are used, one whose values are
    static constexpr int BLOCKS = (NT == 1 ? 3 : 2) + (D == 64 ? 1 : 0);  // a SM
    static constexpr int MERGE = 2 * ROWS * D * 4;   // two warps' sums
    static constexpr int SMEM = WARPS * STAGES * STAGE + MERGE;
    static constexpr int MT = D / 16;                // tiles of the second product
    static constexpr int WORDS = D / 64;             // of codes that a lane takes of a value
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Words of shared memory.
__device__ __forceinline__ uint32_t word(const unsigned char *at) { return *reinterpret_cast<const uint32_t *>(at); }
template <int N>
__device__ __forceinline__ void words(uint32_t (&r)[N], const unsigned char *at)
{
    if constexpr (N == 4) {
        const uint4 x = *reinterpret_cast<const uint4 *>(at);
        r[0] = x.x, r[1] = x.y, r[2] = x.z, r[3] = x.w;
    } else if constexpr (N == 2) {
        const uint2 x = *reinterpret_cast<const uint2 *>(at);
        r[0] = x.x, r[1] = x.y;
    } else {
        r[0] = word(at);
    }
}

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 8 x 8 of 16-bit elements: a lane's two are row lane / 4, columns 2 * (lane % 4) and the next, before and after.
__device__ __forceinline__ uint32_t transpose(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Issues the copies of this warp's keys of one unit; returns which of the 32 are there.  Keys that are not
// become zeros, steps and offsets too.  `k`: where the head's rows begin in the plane's first block.  `near`: every place of
// the plane is fewer than 2^32 steps of 16 bytes from its beginning, so a place is one register until its address is
// made, by one multiply-add.
template <int D, int NT>
__device__ __forceinline__ uint32_t load_unit(const KvcAttn &a, int32_t j, uint32_t id, bool asked, const unsigned char *k, bool near,
                                              uint32_t lane, uint32_t stage)
{
    using S = Shape<D, NT>;
    constexpr uint32_t CHUNKS = S::CODES / 16, PER = 32 / CHUNKS;  // pieces of a key's codes, keys per round
    const uint32_t chunk = lane % CHUNKS, sub = lane / CHUNKS;
    const uint32_t there = __ballot_sync(~0u, id < a.num_blocks);
    const uint32_t in = a.block_shift != KVC_NO_SHIFT ? (uint32_t)j & (a.block_size - 1u) : (uint32_t)j % a.block_size;
    const int64_t to_v = a.v - a.k;
    const uint32_t dst = stage + sub * S::PITCH + chunk * 16u, scale_dst = stage + lane * S::PITCH + S::CODES;
    const auto scales = [&](const unsigned char *at, uint32_t bytes) {
        if (S::SCALES == 16) {
            copy16(scale_dst, at, bytes);
            copy16(scale_dst + WK * S::PITCH, at + to_v, bytes);
        } else {
            copy8(scale_dst, at, bytes);
            copy8(scale_dst + WK * S::PITCH, at + to_v, bytes);
        }
    };
    const uint32_t to_scales = a.block_size * S::CODES - in * (S::CODES - S::SCALES);
    if (there == ~0u && near) {
        const uint32_t mine = id * (uint32_t)(a.block_stride >> 4) + in * (S::CODES / 16);
        const unsigned char *kc = k + chunk * 16u, *vc = kc + to_v;
#pragma unroll
        for (uint32_t i = 0; i < WK / PER; ++i) {
            const uint32_t at = __shfl_sync(~0u, mine, i * PER + sub);
            copy16(dst + i * PER * S::PITCH, kc + (uint64_t)at * 16u, 16);
            copy16(dst + (i * PER + WK) * S::PITCH, vc + (uint64_t)at * 16u, 16);
        }
        scales(k + (uint64_t)mine * 16u + to_scales, S::SCALES);
    } else {
        if (asked && id >= a.num_blocks)
            atomicAdd(a.status, 1u);
        const uint64_t mine = id < a.num_blocks ? (uint64_t)id * a.block_stride + (uint64_t)in * S::CODES : 0ull;
#pragma unroll 1
        for (uint32_t i = 0; i < WK / PER; ++i) {
            const uint32_t row = i * PER + sub, bytes = there >> row & 1u ? 16u : 0u;
            const uint64_t at = __shfl_sync(~0u, mine, row);
            const unsigned char *src = bytes ? k + at + chunk * 16u : a.k;
            copy16(dst + i * PER * S::PITCH, src, bytes);
            copy16(dst + (i * PER + WK) * S::PITCH, src + to_v, bytes);
        }
        const bool is = there >> lane & 1u;
        scales(is ? k + mine + to_scales : a.k, is ? (uint32_t)S::SCALES : 0u);
    }
    return there;
}

// Powers of two that queries take with them into the first product.  Each row has one of its own, which brings its largest
// element near 2^TOP and is undone in the scores (exactly, like all of these): so queries of any size keep all of their bits.
// Another one is for all: QUERY, for codes in the low bits, and QUERY / 16 for those in the high ones, so that products with
// codes as numbers as they stand (bf16: 2^-133 each) are none of the smallest; BACK is 1 / QUERY / (what a code in the low bits
// is worth).  fp16: the row's power is two factors, since one ends at 2^15.
template <typename T>
struct Scaling;
template <>
struct Scaling<__nv_bfloat16> {
    static constexpr int TOP = 0, LEAST = -126, MOST = 126, FIRST = 126;
    static constexpr int QUERY = 64;
    static constexpr float BACK = 0x1p69f;  // 2^(133 - 64)
    static constexpr float SUM = 1.f;
    static __device__ __forceinline__ uint32_t power(int e) { return (uint32_t)(e + 127) * 0x00800080u; }
    static __device__ __forceinline__ uint32_t times(uint32_t x, uint32_t f) { return kvc_mul_bf16x2(x, f); }
};
template <>
struct Scaling<__half> {
    static constexpr int TOP = 13, LEAST = -2, MOST = 30, FIRST = 15;
    static constexpr int QUERY = 0;
    static constexpr float BACK = 0x1p24f;
    static constexpr float SUM = 0x1p-6f;  // of a query's sums, which may leave the type's range
    static __device__ __forceinline__ uint32_t power(int e) { return (uint32_t)(e + 15) * 0x04000400u; }
    static __device__ __forceinline__ uint32_t times(uint32_t x, uint32_t f)
    {
        uint32_t r;
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(f));
        return r;
    }
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(THREADS, Shape<D, NT>::BLOCKS) kvc_attn_q4_rows_kernel(const KvcAttn a)
{
    using S = Shape<D, NT>;
    constexpr int ROWS = S::ROWS, G = S::GROUPS;
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
    const bool near = a.block_stride < (1ull << 36) && ((uint64_t)a.num_blocks * (a.block_stride >> 4)) >> 32 == 0;
    // The next unit to load is one of a stretch of key tiles that follow one another; what they have in common is found
    // once a stretch.  `left`: of the stretch, that one among them (0: the run has no more).
    uint32_t left = 0, tiles = 0;
    int32_t ld_j = 0;                // this lane's key
    uint32_t ld_id = ~0u;            // the id of its block, looked up a unit ahead, so that the table's latency passes meanwhile
    bool ld_asked = false;           // whether it is a key of the pair at all
    const int32_t *ld_table = a.tables;
    const unsigned char *ld_k = a.k;
    const auto look = [&] {
        ld_asked = ld_j < ld.r.hi && (ld_j >= ld.r.lo || ld_j < ld.r.sink_end);
        ld_id = ~0u;
        if (ld_asked)
            ld_id = (uint32_t)ld_table[kvc_div((uint32_t)ld_j, a.block_size, a.block_shift)];
    };
    const auto stretch = [&] {  // from the unit at `ld`
        tiles = left = 0;
        if (ld.s < n_seq)
            tiles = left = min(run.count(ld, ld_at), (ld.t < ld.r.sink_tiles ? ld.r.sink_tiles : ld.r.n) - ld.t);
        if (left) {
            ld_j = (int32_t)(kvc_tile(ld.r, ld.t) * TK + warp * WK + lane);
            ld_table = a.tables + (int64_t)ld.q.table * a.table_stride;
            ld_k = a.k + (uint64_t)ld.h * a.block_size * KVC_Q4_ROW_BYTES(D);
            look();
        }
    };
    stretch();
    const auto load = [&](uint32_t stage) {
        if (left) {
            const int32_t j = ld_j;
            const uint32_t id = ld_id;
            const bool asked = ld_asked;
            const unsigned char *k = ld_k;
            if (--left) {
                ld_j += TK;
                look();
            } else {
                const uint32_t n = ld.r.n;
                ld.t += tiles - 1;
                kvc_next<ROWS, TK>(a, n_seq, ld);
                if (ld.t == 0)
                    ld_at += n + HEAD;
                stretch();
            }
            const uint32_t there = load_unit<D, NT>(a, j, id, asked, k, near, lane, ring + stage * S::STAGE);
            if (lane == 0)
                s_there[warp][stage] = there;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    load(0);
    uint32_t stage = 0;

    for (uint32_t n_units; c.s < n_seq && (n_units = run.count(c, units_at)) != 0;) {
        // ---- a new pair (or the rest of one): its queries as matrix operands, D x 8 NT
        const uint32_t row0 = c.rt * ROWS, rows = min((uint32_t)ROWS, (uint32_t)c.q.rows - row0);
        using F = Scaling<T>;
        uint32_t qf[NT][2 * G][2], qs[NT][2];
        int32_t pos[NT][2];
        float scale[NT][2];  // from products to scores, base 2: with the power of two of the column's row
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t i = n * 8 + gr;
            const bool real = i < rows;
            const unsigned char *src = a.q;
            if (real) {
                const uint32_t row = row0 + i, tok = kvc_div_g(a, row);
                src += (int64_t)(c.q.qa + (int32_t)tok) * a.q_tok + (int64_t)(c.h * a.g + (row - tok * a.g)) * a.q_head;
            }
            uint4 x[G];
            uint32_t top = 0;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                x[g] = make_uint4(0, 0, 0, 0);
                if (real)
                    x[g] = *reinterpret_cast<const uint4 *>(src + g * 64 + gc * 16);
                top = __vmaxu2(__vmaxu2(__vmaxu2(top, x[g].x & 0x7FFF7FFFu), __vmaxu2(x[g].y & 0x7FFF7FFFu, x[g].z & 0x7FFF7FFFu)),
                               x[g].w & 0x7FFF7FFFu);
            }
            // the row's power of two, from its largest element (none for infinity and NaN)
            top = max(top & 0xFFFFu, top >> 16);
            top = max(top, __shfl_xor_sync(~0u, top, 1));
            top = max(top, __shfl_xor_sync(~0u, top, 2));
            const int32_t size = (int32_t)(__float_as_uint(kvc_to_float2<T>(top).x) >> 23) - 127;
            const int32_t power = size == 128 ? 0 : kvc_clamp(F::TOP - size, F::LEAST, F::MOST), first_power = min(power, F::FIRST);
            const uint32_t first_by = F::power(first_power), low_by = F::power(power - first_power + F::QUERY),
                           high_by = F::power(power - first_power + F::QUERY - 4);
            float sums[G];
            const float sum_by = __int_as_float((127 + power - first_power) << 23) * F::SUM;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                x[g] = make_uint4(F::times(x[g].x, first_by), F::times(x[g].y, first_by), F::times(x[g].z, first_by), F::times(x[g].w, first_by));
                qf[n][2 * g][0] = F::times(kvc_lows(x[g].x, x[g].z), low_by);
                qf[n][2 * g][1] = F::times(kvc_highs(x[g].x, x[g].z), high_by);
                qf[n][2 * g + 1][0] = F::times(kvc_lows(x[g].y, x[g].w), low_by);
                qf[n][2 * g + 1][1] = F::times(kvc_highs(x[g].y, x[g].w), high_by);
                const float2 p = kvc_to_float2<T>(x[g].x), q = kvc_to_float2<T>(x[g].y), u = kvc_to_float2<T>(x[g].z), v = kvc_to_float2<T>(x[g].w);
                float sum = ((p.x + p.y) + (q.x + q.y)) + ((u.x + u.y) + (v.x + v.y));
                sum += __shfl_xor_sync(~0u, sum, 1);
                sums[g] = (sum + __shfl_xor_sync(~0u, sum, 2)) * sum_by;
            }
            // (a scale that no float is, of queries or scales at the end of the range, becomes the last that is one)
            const float by = fminf(fmaxf(a.scale_log2 * __int_as_float((127 - power) << 23), 0x1p-126f), 0x1p125f);
            scale[n][0] = __shfl_sync(~0u, by, gc * 8u);
            scale[n][1] = __shfl_sync(~0u, by, gc * 8u + 4u);
            // The product of offsets and a query's sums: places 0-3 of the operand take the groups' sums rounded to the type, 4-7
            // and 8-11 what that leaves, twice over: all 24 bits.  This lane holds places 2 gc, 2 gc + 1 and the same + 8.
            const float s0 = G == 4 && (gc & 1u) ? sums[G / 2] : sums[0], s1 = G == 4 && (gc & 1u) ? sums[G - 1] : sums[1];
            const uint32_t first = kvc_from_float2<T>(s0, s1);
            float2 left = kvc_to_float2<T>(first);
            left = make_float2(s0 - left.x, s1 - left.y);
            const uint32_t second = kvc_from_float2<T>(left.x, left.y);
            const float2 then = kvc_to_float2<T>(second);
            const uint32_t third = kvc_from_float2<T>(left.x - then.x, left.y - then.y);
            const bool has = G == 4 || (gc & 1u) == 0;  // (two groups: every second pair of places is empty)
            qs[n][0] = !has ? 0u : gc < 2 ? first : second;
            qs[n][1] = !has || gc >= 2 ? 0u : third;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // (a column of no row sees what the last row does, so that it holds up no check whether all see a unit's keys)
                pos[n][e] = kvc_row_pos(a, c.q, row0 + min(n * 8 + gc * 2 + e, rows - 1u));
            }
        }
        float o[NT][S::MT][4];
        float m[NT][2], l[NT][2], limit[NT][2];  // the maximum in use, base 2; the sum; the score that would move the maximum
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int t = 0; t < S::MT; ++t)
                o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.f;
            m[n][0] = m[n][1] = limit[n][0] = limit[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.f;
        }
        const bool from_start = c.t == 0;
        const bool to_end = c.t + n_units == c.r.n;

        // The weights of one unit and where its values are: their product is made beside the next unit's scores, which have
        // nothing to do with one another, so that the instructions of either fill the waits of the other.
        uint32_t p[KT][NT][2];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                p[t][n][0] = p[t][n][1] = 0;
        const auto products = [&](const unsigned char *vb) {
            // ---- values: of keys 2 gc, 2 gc + 1 and the same + 8, the codes of words WORDS * gr ..
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                uint32_t w[4][S::WORDS], sc[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const unsigned char *at = vb + (t * 16 + gc * 2 + (r & 1) + (r >> 1) * 8) * S::PITCH;
                    words<S::WORDS>(w[r], at + gr * (4 * S::WORDS));
                    sc[r] = word(at + S::CODES + gr * S::WORDS / 4 * 4);
                }
                const KvcQ4Values<T> v0(kvc_lows(sc[0], sc[1]), kvc_highs(sc[0], sc[1])), v1(kvc_lows(sc[2], sc[3]), kvc_highs(sc[2], sc[3]));
#pragma unroll
                for (int u = 0; u < S::WORDS; ++u) {
                    const uint32_t x0 = kvc_lows(w[0][u], w[1][u]), y0 = kvc_highs(w[0][u], w[1][u]);
                    const uint32_t x1 = kvc_lows(w[2][u], w[3][u]), y1 = kvc_highs(w[2][u], w[3][u]);
                    const auto tile = [&](auto high, uint32_t far, int k) {
                        constexpr bool HIGH = decltype(high)::value;
                        const uint32_t f[4] = {v0.template of<HIGH>(x0 >> far), v0.template of<HIGH>(y0 >> far),
                                               v1.template of<HIGH>(x1 >> far), v1.template of<HIGH>(y1 >> far)};
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma<T>(o[n][u * 4 + k], f, p[t][n][0], p[t][n][1]);
                    };
                    tile(std::false_type(), 0, 0);
                    tile(std::true_type(), 0, 1);
                    tile(std::false_type(), 8, 2);
                    tile(std::true_type(), 8, 3);
                }
            }
        };
        uint32_t before = stage;  // (the first unit's own values, with weights of zero)
        for (uint32_t i = 0; i < n_units; ++i) {
            // the stage of the unit before the last is free once every lane is past its reads
            __syncwarp();
            load(stage == S::STAGES - 1 ? 0 : stage + 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();

            const unsigned char *kb = smem + (warp * S::STAGES + stage) * S::STAGE;
            const uint32_t there = s_there[warp][stage];
            const int32_t j0 = (int32_t)(kvc_tile(c.r, c.t + i) * TK + warp * WK);
            float s[KT][NT][4];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const unsigned char *at = kb + (t * 16 + gr) * S::PITCH;
                uint32_t sc[2][G];
                words<G>(sc[0], at + S::CODES);
                words<G>(sc[1], at + 8 * S::PITCH + S::CODES);
                uint32_t f[4];
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    f[r] = f[r + 2] = G == 4 && (gc & 1u) ? kvc_highs(sc[r][G / 2], sc[r][G - 1]) : kvc_highs(sc[r][0], sc[r][1]);
                float codes[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s[t][n][0] = s[t][n][1] = s[t][n][2] = s[t][n][3] = 0.f;
                    codes[n][0] = codes[n][1] = codes[n][2] = codes[n][3] = 0.f;
                    mma<T>(s[t][n], f, qs[n][0], qs[n][1]);
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t w0 = word(at + g * 16 + gc * 4), w1 = word(at + 8 * S::PITCH + g * 16 + gc * 4);
                    float acc[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t y0 = k ? w0 >> 8 : w0, y1 = k ? w1 >> 8 : w1;
                        const uint32_t f[4] = {kvc_q4_low(y0), kvc_q4_low(y1), kvc_q4_high(y0), kvc_q4_high(y1)};
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma<T>(acc[n], f, qf[n][2 * g + k][0], qf[n][2 * g + k][1]);
                    }
                    const float x0 = kvc_to_float2<T>(sc[0][g]).x, x1 = kvc_to_float2<T>(sc[1][g]).x;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            codes[n][e] = fmaf(e < 2 ? x0 : x1, acc[n][e], codes[n][e]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[t][n][e] = fmaf(codes[n][e], Scaling<T>::BACK, Scaling<T>::SUM == 1.f ? s[t][n][e] : s[t][n][e] * (1.f / Scaling<T>::SUM));
            }
            products(smem + (warp * S::STAGES + before) * S::STAGE + WK * S::PITCH);
            before = stage;
            // where some row does not see all of the warp's keys, the scores of those it does not become -inf
            bool all = there == ~0u;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    all = all && j0 + WK - 1 <= pos[n][e] && (a.window == 0 || pos[n][e] - j0 < a.window || j0 + WK <= a.sinks);
            all = __all_sync(~0u, all);
            // The maximum in use need not be the largest score: it moves when a score is more than 2^8 times its weight, which
            // neither type nor the sums mind, and else the lanes of a row have nothing to tell one another
            float top[NT][2];
            bool move = false;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!all) {
                            const int k = t * 16 + (e >> 1) * 8 + (int)gr;
                            if (!((there >> k & 1u) && kvc_sees(a, pos[n][e & 1], j0 + k)))
                                s[t][n][e] = -INFINITY;
                        }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(s[0][n][e], s[0][n][e + 2]);
#pragma unroll
                    for (int t = 1; t < KT; ++t)
                        x = fmaxf(x, fmaxf(s[t][n][e], s[t][n][e + 2]));
                    top[n][e] = x;
                    move |= x > limit[n][e];
                }
            }
            if (__any_sync(~0u, move)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = fmaxf(top[n][e], __shfl_xor_sync(~0u, top[n][e], 4));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                        const float now = fmaxf(m[n][e], x * scale[n][e]);
                        const float f = m[n][e] == -INFINITY ? 0.f : exp2_fast(m[n][e] - now);
                        m[n][e] = now;
                        limit[n][e] = now == -INFINITY ? -INFINITY : __fdividef(now + 8.f, scale[n][e]);
                        l[n][e] *= f;
#pragma unroll
                        for (int t = 0; t < S::MT; ++t) {
                            o[n][t][e] *= f;
                            o[n][t][e + 2] *= f;
                        }
                    }
            }
            #pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float base0 = m[n][0] == -INFINITY ? 0.f : -m[n][0], base1 = m[n][1] == -INFINITY ? 0.f : -m[n][1];
#pragma unroll
                for (int t = 0; t < KT; ++t) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[t][n][e] = exp2_fast(fmaf(s[t][n][e], scale[n][e & 1], e & 1 ? base1 : base0));
                        l[n][e & 1] += s[t][n][e];
                    }
                    p[t][n][0] = transpose(kvc_from_float2<T>(s[t][n][0], s[t][n][1]));
                    p[t][n][1] = transpose(kvc_from_float2<T>(s[t][n][2], s[t][n][3]));
                }
            }
            stage = stage == S::STAGES - 1 ? 0 : stage + 1;
        }
        products(smem + (warp * S::STAGES + before) * S::STAGE + WK * S::PITCH);

        // ---- end of the pair, or of the run: join the four warps' parts
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[n][e] += __shfl_xor_sync(~0u, l[n][e], 4);
                l[n][e] += __shfl_xor_sync(~0u, l[n][e], 8);
                l[n][e] += __shfl_xor_sync(~0u, l[n][e], 16);
            }
        __syncthreads();  // the join before this one is over
        if (gr == 0)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s_m[warp][n * 8 + gc * 2 + e] = m[n][e];
                    s_l[warp][n * 8 + gc * 2 + e] = l[n][e];
                }
        __syncthreads();
        float tm[NT][2], tl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t col = n * 8 + gc * 2 + e;
                tm[n][e] = s_m[0][col];
#pragma unroll
                for (int w = 1; w < WARPS; ++w)
                    tm[n][e] = fmaxf(tm[n][e], s_m[w][col]);
                const float ref = tm[n][e] == -INFINITY ? 0.f : tm[n][e];
                tl[n][e] = 0.f;
#pragma unroll
                for (int w = 0; w < WARPS; ++w)
                    tl[n][e] += s_l[w][col] * exp2f(s_m[w][col] - ref);
                const float f = exp2f(m[n][e] - ref) * (1.f / KvcQ4Values<T>::SCALE);
#pragma unroll
                for (int t = 0; t < S::MT; ++t) {
                    o[n][t][e] *= f;
                    o[n][t][e + 2] *= f;
                }
            }
        // 3 + 2 -> 1 + 0 -> 0, each lane reading back the places that its partner's lane wrote
#pragma unroll
        for (uint32_t step = 2; step; step /= 2) {
            if (warp >= step && warp < 2 * step) {
                float4 *dst = reinterpret_cast<float4 *>(merge) + (warp - step) * (ROWS * D / 4) + lane;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < S::MT; ++t)
                        dst[(n * S::MT + t) * 32] = make_float4(o[n][t][0], o[n][t][1], o[n][t][2], o[n][t][3]);
            }
            __syncthreads();
            if (warp < step) {
                const float4 *src = reinterpret_cast<const float4 *>(merge) + warp * (ROWS * D / 4) + lane;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < S::MT; ++t) {
                        const float4 v = src[(n * S::MT + t) * 32];
                        o[n][t][0] += v.x;
                        o[n][t][1] += v.y;
                        o[n][t][2] += v.z;
                        o[n][t][3] += v.w;
                    }
            }
            if (step > 1)
                __syncthreads();
        }
        if (warp == 0) {
            const bool whole = a.phase == KVC_PHASE_WHOLE && from_start && to_end;
            const bool room = a.phase == KVC_PHASE_WHOLE || pair < a.parts.max_pairs;
            const uint64_t slot = a.phase == KVC_PHASE_WHOLE ? 2ull * blockIdx.x + (from_start ? 1 : 0) : (uint64_t)blockIdx.x + pair;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t col = n * 8 + gc * 2 + e;
                    if (col >= rows)
                        continue;
                    // words WORDS * gr ..: value k of a word is in tile k, row gr, value 4 + k in row gr + 8
                    if (whole) {
                        const uint32_t row = row0 + col, t = kvc_div_g(a, row);
                        const int64_t tok = c.q.qa + (int32_t)t;
                        const uint32_t head = c.h * a.g + (row - t * a.g);
                        const float inv = tl[n][e] == 0.f ? 0.f : 1.f / tl[n][e];  // a row that sees nothing: zeros
                        unsigned char *dst = a.out + tok * a.o_tok + (int64_t)head * a.o_head + gr * (16 * S::WORDS);
#pragma unroll
                        for (int u = 0; u < S::WORDS; ++u) {
                            const auto x = [&](int k) { return o[n][u * 4 + (k & 3)][e + (k >> 2) * 2] * inv; };
                            *reinterpret_cast<uint4 *>(dst + u * 16) =
                                make_uint4(kvc_from_float2<T>(x(0), x(1)), kvc_from_float2<T>(x(2), x(3)),
                                           kvc_from_float2<T>(x(4), x(5)), kvc_from_float2<T>(x(6), x(7)));
                        }
                        if (a.lse && gr == 0)
                            a.lse[tok * a.hq + head] = (tm[n][e] + log2f(tl[n][e])) * 0.693147180559945309f;
                    } else if (room) {
                        const uint64_t at = slot * ROWS + col;
                        float *dst = a.parts.o + at * D + gr * (8 * S::WORDS);
#pragma unroll
                        for (int u = 0; u < S::WORDS; ++u) {
                            const auto x = [&](int k) { return o[n][u * 4 + (k & 3)][e + (k >> 2) * 2]; };
                            *reinterpret_cast<float4 *>(dst + u * 8) = make_float4(x(0), x(1), x(2), x(3));
                            *reinterpret_cast<float4 *>(dst + u * 8 + 4) = make_float4(x(4), x(5), x(6), x(7));
                        }
                        if (gr == 0)
                            a.parts.ml[at] = make_float2(tm[n][e], tl[n][e]);
                    }
                }
            if (a.phase != KVC_PHASE_WHOLE && room && from_start && lane == 0)
                a.parts.range[pair] = make_ulonglong2(units_at, units_at + c.r.n);
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

template <typename T, int D, int NT>
cudaError_t launch(const KvcAttn &a, uint32_t blocks, cudaStream_t st)
{
    using S = Shape<D, NT>;
    const cudaError_t e = cudaFuncSetAttribute(kvc_attn_q4_rows_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess)
        return e;
    return kvc_launch_pdl(kvc_attn_q4_rows_kernel<T, D, NT>, a, dim3(blocks), THREADS, S::SMEM, st);
}

template <typename T>
cudaError_t launch_type(const KvcAttn &a, uint32_t head_dim, uint32_t blocks, cudaStream_t st)
{
    if (a.parts.rows == KVC_ATTN_FEW_ROWS)
        return head_dim == 128 ? launch<T, 128, 1>(a, blocks, st) : launch<T, 64, 1>(a, blocks, st);
    return head_dim == 128 ? launch<T, 128, 2>(a, blocks, st) : launch<T, 64, 2>(a, blocks, st);
}

}  // namespace

// As many blocks as are resident.
uint32_t kvc_attn_q4_rows_blocks(const kvc_layout *lay, uint32_t rows)
{
    const int few = kvc_q4_head_dim(lay) == 128 ? Shape<128, 1>::BLOCKS : Shape<64, 1>::BLOCKS;
    const int more = kvc_q4_head_dim(lay) == 128 ? Shape<128, 2>::BLOCKS : Shape<64, 2>::BLOCKS;
    return (uint32_t)(rows == KVC_ATTN_FEW_ROWS ? few : more) * (uint32_t)lay->sm_count;
}

cudaError_t kvc_launch_attn_q4_rows(const KvcAttn &a, uint32_t dtype, uint32_t head_dim, uint32_t blocks, cudaStream_t st)
{
    return dtype == KVC_DTYPE_BF16 ? launch_type<__nv_bfloat16>(a, head_dim, blocks, st) : launch_type<__half>(a, head_dim, blocks, st);
}
