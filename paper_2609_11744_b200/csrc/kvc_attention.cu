// Entry points of attention over the paged pool (kvc_attention, kvc_attention_shared, and the same over a
// pool held in 4 bits), the layout of their workspace, and the kernels that join the parts of a pair.
#include <string.h>

#include <algorithm>

#include "kvc_attention.h"

namespace {

// ------------------------------------------------------------------------------------ joining parts
//
// A part is (weighted sum o, maximum m, sum l) of a row over some of its keys; the whole is
// sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i with M the largest m_i.  WPR warps serve a row: they
// take the parts in turn, and their sums are added in a fixed order.  Bound by the latency of the
// parts' loads, so a row with many parts gets a whole block.
template <int D>
struct Vec {
    static constexpr int N = D / 32;  // floats per lane
    float v[N];
};

template <int D, int WPR, typename Get>
__device__ __forceinline__ void join_row(uint32_t n, const Get &get, Vec<D> &sum, float &m, float &l)
{
    constexpr int N = Vec<D>::N;
    const uint32_t lane = threadIdx.x & 31u, w = (threadIdx.x >> 5) % WPR;
    const float2 none = make_float2(-INFINITY, 0.f);
    if (WPR == 1 && n <= 4) {  // the usual case: everything at once, no lane needs another's
        float2 x[4];
        float v[4][N];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            x[i] = none;
#pragma unroll
            for (int e = 0; e < N; ++e)
                v[i][e] = 0.f;
            if (i < n) {
                const auto part = get(i);
                x[i] = part.ml();
                if (N == 4)
                    *reinterpret_cast<float4 *>(v[i]) = *reinterpret_cast<const float4 *>(part.o() + lane * N);
                else
                    *reinterpret_cast<float2 *>(v[i]) = *reinterpret_cast<const float2 *>(part.o() + lane * N);
            }
        }
        m = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
        const float ref = m == -INFINITY ? 0.f : m;
        l = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e)
            sum.v[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = exp2f(x[i].x - ref);
            l += x[i].y * f;
#pragma unroll
            for (int e = 0; e < N; ++e)
                sum.v[e] += f * v[i][e];
        }
        return;
    }
    const float2 mine = lane < n ? get(lane).ml() : none;  // the first 32 parts' (m, l), a lane each
    m = mine.x;
    for (uint32_t i = lane + 32; i < n; i += 32)
        m = fmaxf(m, get(i).ml().x);
#pragma unroll
    for (uint32_t o = 16; o; o /= 2)
        m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e)
        sum.v[e] = 0.f;
    for (uint32_t first = 0; first < n; first += 32) {
        const float2 x = first == 0 ? mine : first + lane < n ? get(first + lane).ml() : none;
        const float f = exp2f(x.x - ref);
        l += x.y * f;
        const uint32_t end = min(n - first, 32u);
#pragma unroll 4
        for (uint32_t i = w; i < end; i += WPR) {
            const auto part = get(first + i);
            const float fi = __shfl_sync(~0u, f, i);
            const float *src = part.o() + lane * N;
            float v[N];
            if (N == 4)
                *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(src);
            else
                *reinterpret_cast<float2 *>(v) = *reinterpret_cast<const float2 *>(src);
#pragma unroll
            for (int e = 0; e < N; ++e)
                sum.v[e] += fi * v[e];
        }
    }
#pragma unroll
    for (uint32_t o = 16; o; o /= 2)
        l += __shfl_xor_sync(~0u, l, o);
}

template <int D>
struct Part {
    const KvcParts *p;
    uint64_t at;  // slot * ROWS + row
    __device__ float2 ml() const { return p->ml[at]; }
    __device__ const float *o() const { return p->o + at * D; }
};

template <typename T, int D>
__device__ __forceinline__ void write_row(const KvcAttn &a, int64_t tok, uint32_t head, const Vec<D> &sum, float m, float l)
{
    const uint32_t lane = threadIdx.x & 31u;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    unsigned char *dst = a.out + tok * a.o_tok + (int64_t)head * a.o_head + lane * Vec<D>::N * 2;
#pragma unroll
    for (int e = 0; e < Vec<D>::N; e += 2)
        *reinterpret_cast<uint32_t *>(dst + e * 2) = kvc_from_float2<T>(sum.v[e] * inv, sum.v[e + 1] * inv);
    if (a.lse && lane == 0)
        a.lse[tok * a.hq + head] = (m + log2f(l)) * 0.693147180559945309f;
}

// Whole sequences: block x looks at the boundary between runs x and x + 1.  The first boundary inside
// a pair's units joins that pair: the part of the run before it, then those of the runs after it that begin
// inside the pair.
constexpr int JOIN_WARPS = 8;

template <typename T, int D, int WPR>
__global__ void __launch_bounds__(JOIN_WARPS * 32) kvc_join_split_kernel(const KvcAttn a)
{
    __shared__ float s_sum[JOIN_WARPS][D];
    kvc_pdl_wait();
    const uint32_t c = blockIdx.x + 1;
    const KvcSplit sp = a.parts.split[c];
    if (sp.end == sp.begin || kvc_cut(c - 1, sp.length, sp.runs) > sp.begin)
        return;
    const uint32_t last = kvc_run_of(sp.end - 1, sp.length, sp.runs);  // the run that holds the pair's last unit
    const uint32_t n = last - c + 2;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    // a warp's rows are summed BATCH at a time before any is written, so that their loads overlap
    constexpr int BATCH = WPR == 1 ? 2 : 1;
    constexpr uint32_t STEP = JOIN_WARPS / WPR;
    for (uint32_t row0 = blockIdx.y * STEP * BATCH + warp / WPR; row0 < sp.rows; row0 += gridDim.y * STEP * BATCH) {
        Vec<D> sum[BATCH];
        float m[BATCH], l[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const uint32_t row = min(row0 + b * STEP, sp.rows - 1);
            const auto get = [&](uint32_t i) {
                Part<D> p;
                const uint32_t run = c - 1 + i;
                p.p = &a.parts;
                p.at = (2ull * run + (i == 0 ? 1 : 0)) * a.parts.rows + row;
                return p;
            };
            join_row<D, WPR>(n, get, sum[b], m[b], l[b]);
        }
        if (WPR > 1) {  // one row a block at a time: all warps take the same turns
            __syncthreads();
#pragma unroll
            for (int e = 0; e < Vec<D>::N; ++e)
                s_sum[warp][lane * Vec<D>::N + e] = sum[0].v[e];
            __syncthreads();
            if (warp == 0)
#pragma unroll
                for (int w = 1; w < WPR; ++w)
#pragma unroll
                    for (int e = 0; e < Vec<D>::N; ++e)
                        sum[0].v[e] += s_sum[w][lane * Vec<D>::N + e];
        }
        if (warp % WPR == 0)
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const uint32_t i = sp.row0 + row0 + b * STEP;
                if (row0 + b * STEP < sp.rows)
                    {
                    const uint32_t tok = kvc_div_g(a, i);
                    write_row<T, D>(a, sp.qa + (int32_t)tok, sp.head * a.g + (i - tok * a.g), sum[b], m[b], l[b]);
                }
            }
    }
}

// The parts of one row in one phase: runs first .. first + n - 1, slot = run + pair.
struct PhaseRow {
    uint32_t first, n;
    uint64_t pair, row;
};

__device__ __forceinline__ PhaseRow phase_row(const KvcParts &p, uint32_t seq, uint32_t head, uint32_t rows, uint32_t i)
{
    PhaseRow r;
    const uint32_t tiles = (rows + p.rows - 1) / p.rows;
    r.pair = (uint64_t)p.base[seq] + (uint64_t)head * tiles + i / p.rows;
    r.row = i % p.rows;
    const unsigned long long length = p.length[0];
    const uint32_t runs = (uint32_t)p.length[1];
    r.first = r.n = 0;
    // what lengths that contradict one another lead to is left out
    if (i >= rows || r.pair >= p.max_pairs || length == 0)
        return r;
    const ulonglong2 u = p.range[r.pair];
    if (u.x >= u.y || u.y > length)
        return r;
    r.first = kvc_run_of(u.x, length, runs);
    r.n = kvc_run_of(u.y - 1, length, runs) - r.first + 1;
    return r;
}

struct JoinShared {
    KvcAttn a;
    KvcParts prefix, suffix;
};

// Shared prefixes: WPR warps join one row's parts of its group's prefix and of its own keys.
template <typename T, int D, int WPR>
__global__ void __launch_bounds__(JOIN_WARPS * 32) kvc_join_shared_kernel(const JoinShared j)
{
    kvc_pdl_wait();
    const KvcAttn &a = j.a;
    const uint32_t top = (uint32_t)kvc_clamp(a.cu_q[a.n_requests], 0, (int32_t)a.n_tokens);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint64_t w = (uint64_t)blockIdx.x * (JOIN_WARPS / WPR) + warp / WPR;
    const uint32_t tok = (uint32_t)(w / a.hq), head = (uint32_t)(w - (uint64_t)tok * a.hq);
    // rows outside the sequences belong to none
    const bool real = w < (uint64_t)top * a.hq && (int32_t)tok >= a.cu_q[0];
    if (WPR == 1 && !real)
        return;
    __shared__ float s_sum[JOIN_WARPS][D];
    Vec<D> sum;
    float m = 0.f, l = 0.f;
    if (real) {
        const uint32_t h = head / a.g, x = head % a.g;
        const uint32_t r = kvc_last_at_most_warp(a.cu_q, a.n_requests, (int32_t)tok);
        const int32_t qa = a.cu_q[r], qe = kvc_clamp(a.cu_q[r + 1], qa, (int32_t)a.n_tokens);
        const PhaseRow s = phase_row(j.suffix, r, h, (uint32_t)(qe - qa) * a.g, (tok - (uint32_t)qa) * a.g + x);
        PhaseRow p;
        p.first = p.n = 0;
        p.pair = p.row = 0;
        const int32_t g = kvc_group_of(a, r);
        if (g >= 0) {
            const int32_t R = (int32_t)a.n_requests;
            const int32_t r0 = kvc_clamp(a.group_starts[g], 0, R), r1 = kvc_clamp(a.group_starts[g + 1], r0, R);
            const int32_t ga = kvc_clamp(a.cu_q[r0], 0, (int32_t)a.n_tokens), ge = kvc_clamp(a.cu_q[r1], ga, (int32_t)a.n_tokens);
            p = phase_row(j.prefix, (uint32_t)g, h, (uint32_t)(ge - ga) * a.g, (tok - (uint32_t)ga) * a.g + x);
        }
        const auto get = [&](uint32_t i) {
            Part<D> q;
            const bool in_prefix = i < p.n;
            const KvcParts &from = in_prefix ? j.prefix : j.suffix;
            const PhaseRow &at = in_prefix ? p : s;
            q.p = &from;
            q.at = (at.first + (in_prefix ? i : i - p.n) + at.pair) * from.rows + at.row;
            return q;
        };
        join_row<D, WPR>(p.n + s.n, get, sum, m, l);
    }
    if (WPR > 1) {
#pragma unroll
        for (int e = 0; e < Vec<D>::N; ++e)
            s_sum[warp][lane * Vec<D>::N + e] = sum.v[e];
        __syncthreads();
        if (!real || warp % WPR != 0)
            return;
#pragma unroll
        for (int i = 1; i < WPR; ++i)
#pragma unroll
            for (int e = 0; e < Vec<D>::N; ++e)
                sum.v[e] += s_sum[warp + i][lane * Vec<D>::N + e];
    }
    write_row<T, D>(a, tok, head, sum, m, l);
}

// ------------------------------------------------------------------------------------ workspace

struct Carver {
    unsigned char *base;
    uint64_t used;
    template <typename P>
    void take(P *&p, uint64_t count)
    {
        p = reinterpret_cast<P *>(base + used);
        used += (count * sizeof(P) + 255) & ~255ull;
    }
};

// The parts that the kernel for pairs of `rows` rows can leave.  With whole sequences: at most two
// a block.  By pair, every pair leaves its parts: run + pair is a slot of its own, since along the
// order of units each new part has a larger run or a larger pair.
struct Shape {
    uint32_t head_dim, hkv, g;
    uint64_t tokens, requests, groups;
    bool q4;
};

void carve(Carver &c, KvcParts &p, const kvc_layout *lay, const Shape &s, uint32_t rows, uint64_t sequences, bool by_pair)
{
    const uint32_t blocks = rows > KVC_ATTN_SMALL_ROWS ? kvc_attn_tiles_blocks(lay)
                            : s.q4                     ? kvc_attn_q4_rows_blocks(lay, rows)
                                                       : kvc_attn_rows_blocks(lay, by_pair);
    const uint32_t head_dim = s.head_dim;
    const uint64_t pairs = by_pair ? kvc_max_pairs(sequences, s.tokens, s.g, s.hkv, rows) : 0;
    const uint64_t slots = pairs ? (uint64_t)blocks + pairs : 2ull * blocks;
    memset(&p, 0, sizeof(p));
    p.blocks = blocks;
    p.rows = rows;
    p.max_pairs = (uint32_t)pairs;
    c.take(p.ml, slots * rows);
    c.take(p.o, slots * rows * head_dim);
    if (pairs) {
        c.take(p.base, sequences);
        c.take(p.range, pairs);
        c.take(p.length, 2);
    } else {
        c.take(p.split, blocks);
    }
}

// Bytes of the parts of one phase, for any kernel that may serve it.
uint64_t phase_bytes(const kvc_layout *lay, const Shape &s, uint64_t sequences, bool pairs)
{
    uint64_t most = 0;
    for (const uint32_t rows : {KVC_ATTN_FEW_ROWS, KVC_ATTN_SMALL_ROWS, KVC_ATTN_TILE_ROWS, KVC_ATTN_MANY_ROWS}) {
        if (rows == KVC_ATTN_FEW_ROWS && !s.q4)
            continue;
        KvcParts p;
        Carver c = {nullptr, 0};
        carve(c, p, lay, s, rows, sequences, pairs);
        most = std::max(most, c.used);
    }
    return most;
}

uint64_t workspace_bytes(const kvc_layout *lay, const Shape &s)
{
    return s.groups ? phase_bytes(lay, s, s.groups, true) + phase_bytes(lay, s, s.requests, true)
                    : phase_bytes(lay, s, s.requests, false);
}

kvc_status check(const kvc_layout *lay, const kvc_attention_desc *d, bool q4)
{
    if (!lay || !d || d->reserved != 0)
        return KVC_ERR_INVALID_ARG;
    const kvc_layout_desc &l = lay->d;
    if (d->layer >= l.num_layers || l.kv_planes != 2 ||
        (q4 ? kvc_q4_head_dim(lay) == 0 : l.elem_bytes != 2 || (l.head_dim != 64 && l.head_dim != 128)) ||
        (d->dtype != KVC_DTYPE_BF16 && d->dtype != KVC_DTYPE_FP16))
        return KVC_ERR_INVALID_ARG;
    if (d->n_q_heads == 0 || d->n_q_heads % l.num_kv_heads || !(d->scale > 0.f) || d->scale > 3.0e38f ||
        d->window > KVC_ATTENTION_MAX_KEYS || d->sinks > KVC_ATTENTION_MAX_KEYS || d->n_requests > 0x7FFFFFFFu)
        return KVC_ERR_INVALID_ARG;
    if ((uint64_t)d->n_tokens * (d->n_q_heads / l.num_kv_heads) > 0x7FFFFFFFull)
        return KVC_ERR_TOO_LARGE;
    if (q4 && d->scale > KVC_Q4_MAX_SCALE)
        return KVC_ERR_INVALID_ARG;
    return q4 && !kvc_q4_aligned(lay) ? KVC_ERR_ALIGNMENT : KVC_OK;
}

template <typename T, int D>
cudaError_t join_split(const KvcAttn &a, cudaStream_t st)
{
    if (a.parts.rows <= KVC_ATTN_SMALL_ROWS)  // few rows, possibly of many parts: a block to a row
        return kvc_launch_pdl(kvc_join_split_kernel<T, D, JOIN_WARPS>, a, dim3(a.parts.blocks - 1, 4), JOIN_WARPS * 32, 0, st);
    return kvc_launch_pdl(kvc_join_split_kernel<T, D, 1>, a, dim3(a.parts.blocks - 1, 16), JOIN_WARPS * 32, 0, st);
}

template <typename T, int D>
cudaError_t join_shared(const JoinShared &j, cudaStream_t st)
{
    // few rows: four warps each, for the SMs would stand idle while a row's parts are summed one after the other
    // (1024 rows of some 20 parts: 15 us with one warp a row, 11 with four)
    const uint64_t rows = (uint64_t)j.a.n_tokens * j.a.hq;
    if (rows <= 2048)
        return kvc_launch_pdl(kvc_join_shared_kernel<T, D, 4>, j, dim3((uint32_t)((rows * 4 + JOIN_WARPS - 1) / JOIN_WARPS)),
                              JOIN_WARPS * 32, 0, st);
    return kvc_launch_pdl(kvc_join_shared_kernel<T, D, 1>, j, dim3((uint32_t)((rows + JOIN_WARPS - 1) / JOIN_WARPS)),
                          JOIN_WARPS * 32, 0, st);
}

kvc_status attention(kvc_layout *lay, const kvc_attention_desc *d, bool shared, bool q4, void *stream)
{
    kvc_status s = check(lay, d, q4);
    if (s != KVC_OK)
        return s;
    if (shared ? (d->window != 0 || d->sinks != 0 || d->n_groups == 0 || d->n_groups > d->n_requests)
               : (d->n_groups != 0 || d->group_starts || d->prefix_lens))
        return KVC_ERR_INVALID_ARG;
    if (d->n_tokens == 0 || d->n_requests == 0)
        return KVC_OK;
    if (!d->q || !d->out || !d->cu_tokens || !d->seq_lens || !d->block_tables || !d->workspace || d->max_blocks == 0 ||
        (d->n_requests > 1 && d->table_stride < d->max_blocks) || (shared && (!d->group_starts || !d->prefix_lens)))
        return KVC_ERR_INVALID_ARG;
    const auto off = [](const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) != 0; };
    if (off(d->q, 16) || off(d->out, 16) || off(d->workspace, 256) || off(d->lse, 4) || off(d->cu_tokens, 4) ||
        off(d->seq_lens, 4) || off(d->block_tables, 4) || off(d->group_starts, 4) || off(d->prefix_lens, 4) ||
        (d->q_token_stride | d->q_head_stride | d->out_token_stride | d->out_head_stride) % 8)
        return KVC_ERR_ALIGNMENT;
    s = kvc_ensure_device(lay);
    if (s != KVC_OK)
        return s;
    const kvc_layout_desc &l = lay->d;
    const uint32_t head_dim = q4 ? kvc_q4_head_dim(lay) : l.head_dim;
    Shape shape;
    shape.q4 = q4;
    shape.head_dim = head_dim;
    shape.hkv = l.num_kv_heads;
    shape.g = d->n_q_heads / l.num_kv_heads;
    shape.tokens = d->n_tokens;
    shape.requests = d->n_requests;
    shape.groups = shared ? d->n_groups : 0;
    if (d->workspace_bytes < workspace_bytes(lay, shape))
        return KVC_ERR_INVALID_ARG;

    KvcAttn a;
    memset(&a, 0, sizeof(a));
    a.k = kvc_plane_ptr(lay, d->layer, 0);
    a.v = kvc_plane_ptr(lay, d->layer, 1);
    a.block_stride = lay->block_stride;
    a.tok_stride = l.num_kv_heads * l.head_dim * 2;
    a.block_size = l.block_size;
    a.num_blocks = l.num_blocks;
    a.max_blocks = d->max_blocks;
    a.tables = d->block_tables;
    a.table_stride = (int64_t)d->table_stride;
    a.seq_lens = d->seq_lens;
    a.cu_q = d->cu_tokens;
    a.group_starts = d->group_starts;
    a.prefix_lens = d->prefix_lens;
    a.n_tokens = d->n_tokens;
    a.n_requests = d->n_requests;
    a.n_groups = d->n_groups;
    a.q = static_cast<const unsigned char *>(d->q);
    a.out = static_cast<unsigned char *>(d->out);
    a.lse = d->lse;
    a.q_tok = 2 * d->q_token_stride;
    a.q_head = 2 * d->q_head_stride;
    a.o_tok = 2 * d->out_token_stride;
    a.o_head = 2 * d->out_head_stride;
    a.hq = d->n_q_heads;
    a.hkv = l.num_kv_heads;
    a.g = shape.g;
    a.g_shift = kvc_shift_of(a.g);
    a.block_shift = kvc_shift_of(a.block_size);
    a.scale_log2 = d->scale * 1.44269504088896341f;
    if (q4)
        a.scale_log2 = std::max(a.scale_log2, 0x1p-126f);  // (powers of two are added to its exponent)
    a.window = (int32_t)d->window;
    a.sinks = (int32_t)d->sinks;
    a.status = lay->d_status;

    cudaStream_t st = (cudaStream_t)stream;
    const bool bf16 = d->dtype == KVC_DTYPE_BF16, wide = head_dim == 128;
    Carver c = {static_cast<unsigned char *>(d->workspace), 0};
    // Sixteen rows or fewer fit the kernel for few rows, which reads the keys once for them; with more
    // it would read them once for every sixteen, and the matrix unit takes over.  Up to 128 rows it gets one
    // row tile and a deeper ring of keys.  (Whatever the lengths turn out to be, any of the three is right.)
    // Over a pool held in 4 bits eight rows or fewer are one tile of columns, of which an SM holds one block more (heads of 128:
    // three and two).  Up to 128 rows whose table or window reaches 128 keys at most are for the kernel for few rows too: it starts
    // sooner (32 requests of up to 5 drafted tokens, 20 rows a KV head, 20 to 128 keys: 19 us against 27).  Over long prompts it
    // takes 4.7 times as long (8192 tokens, window 128: 607 us against 130).
    const uint64_t q_len = std::min<uint64_t>(d->max_q_len ? d->max_q_len : d->n_tokens, d->n_tokens);
    const uint64_t table = (uint64_t)a.max_blocks * a.block_size;
    const uint64_t reach = d->window ? std::min<uint64_t>(table, (uint64_t)d->window + d->sinks) : table;
    const auto kernel_rows = [&](uint64_t tokens) {
        const uint64_t rows = tokens * a.g;
        if (q4 && rows <= KVC_ATTN_FEW_ROWS)
            return KVC_ATTN_FEW_ROWS;
        if (q4 && rows <= KVC_ATTN_TILE_ROWS && reach <= 128)
            return KVC_ATTN_SMALL_ROWS;
        return rows <= KVC_ATTN_SMALL_ROWS ? KVC_ATTN_SMALL_ROWS : rows <= KVC_ATTN_TILE_ROWS ? KVC_ATTN_TILE_ROWS : KVC_ATTN_MANY_ROWS;
    };
    const auto launch = [&]() {
        ++lay->launches;
        const bool few = a.parts.rows <= KVC_ATTN_SMALL_ROWS;
        return (q4 ? (few ? kvc_launch_attn_q4_rows : kvc_launch_attn_q4_tiles) : few ? kvc_launch_attn_rows : kvc_launch_attn_tiles)(
            a, d->dtype, head_dim, a.parts.blocks, st);
    };
    cudaError_t e;
    if (!shared) {
        a.phase = KVC_PHASE_WHOLE;
        carve(c, a.parts, lay, shape, kernel_rows(q_len), d->n_requests, false);
        e = launch();
        if (e == cudaSuccess)
            e = bf16 ? (wide ? join_split<__nv_bfloat16, 128>(a, st) : join_split<__nv_bfloat16, 64>(a, st))
                     : (wide ? join_split<__half, 128>(a, st) : join_split<__half, 64>(a, st));
    } else {
        JoinShared j;
        // a group has at least as many rows as a request, and usually several requests
        const uint64_t group_len = std::max<uint64_t>(q_len, (d->n_tokens + d->n_groups - 1) / d->n_groups);
        a.phase = KVC_PHASE_PREFIX;
        carve(c, a.parts, lay, shape, kernel_rows(group_len), d->n_groups, true);
        j.prefix = a.parts;
        e = launch();
        a.phase = KVC_PHASE_SUFFIX;
        a.beside = 1;  // the two phases share nothing but what they read
        carve(c, a.parts, lay, shape, kernel_rows(q_len), d->n_requests, true);
        j.suffix = a.parts;
        if (e == cudaSuccess)
            e = launch();
        j.a = a;
        if (e == cudaSuccess)
            e = bf16 ? (wide ? join_shared<__nv_bfloat16, 128>(j, st) : join_shared<__nv_bfloat16, 64>(j, st))
                     : (wide ? join_shared<__half, 128>(j, st) : join_shared<__half, 64>(j, st));
    }
    ++lay->launches;
    kvc_step_launched(lay->device, st);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return KVC_ERR_CUDA;
    }
    return KVC_OK;
}

kvc_status workspace(kvc_layout *lay, uint32_t n_tokens, uint32_t n_requests, uint32_t n_q_heads, uint32_t n_groups, bool q4,
                     uint64_t *bytes)
{
    if (!lay || !bytes)
        return KVC_ERR_INVALID_ARG;
    *bytes = 0;
    kvc_attention_desc d;
    memset(&d, 0, sizeof(d));
    d.n_tokens = n_tokens;
    d.n_requests = n_requests;
    d.n_q_heads = n_q_heads;
    d.scale = 1.f;
    kvc_status s = check(lay, &d, q4);
    if (s != KVC_OK)
        return s;
    if (n_groups > n_requests)
        return KVC_ERR_INVALID_ARG;
    s = kvc_ensure_device(lay);
    if (s != KVC_OK)
        return s;
    Shape shape;
    shape.q4 = q4;
    shape.head_dim = q4 ? kvc_q4_head_dim(lay) : lay->d.head_dim;
    shape.hkv = lay->d.num_kv_heads;
    shape.g = n_q_heads / lay->d.num_kv_heads;
    shape.tokens = n_tokens;
    shape.requests = n_requests;
    shape.groups = n_groups;
    *bytes = workspace_bytes(lay, shape);
    return KVC_OK;
}

}  // namespace

extern "C" {

kvc_status kvc_attention_workspace_bytes(kvc_layout *lay, uint32_t n_tokens, uint32_t n_requests, uint32_t n_q_heads,
                                         uint32_t n_groups, uint64_t *bytes)
{
    return workspace(lay, n_tokens, n_requests, n_q_heads, n_groups, false, bytes);
}

kvc_status kvc_attention(kvc_layout *lay, const kvc_attention_desc *d, void *stream)
{
    return attention(lay, d, false, false, stream);
}

kvc_status kvc_attention_shared(kvc_layout *lay, const kvc_attention_desc *d, void *stream)
{
    return attention(lay, d, true, false, stream);
}

kvc_status kvc_attention_q4_workspace_bytes(kvc_layout *lay, uint32_t n_tokens, uint32_t n_requests, uint32_t n_q_heads,
                                            uint32_t n_groups, uint64_t *bytes)
{
    return workspace(lay, n_tokens, n_requests, n_q_heads, n_groups, true, bytes);
}

kvc_status kvc_attention_q4(kvc_layout *lay, const kvc_attention_desc *d, void *stream)
{
    return attention(lay, d, false, true, stream);
}

kvc_status kvc_attention_q4_shared(kvc_layout *lay, const kvc_attention_desc *d, void *stream)
{
    return attention(lay, d, true, true, stream);
}

}  // extern "C"
