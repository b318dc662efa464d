// Shared by the attention kernels: the launch parameters, and how a call's work is cut up.
//
// Rows.  The query heads that share a KV head are packed: row i of a sequence and KV head h is
// token i / G, query head h * G + i % G.  A "pair" is (sequence, KV head, tile of ROWS rows); its
// keys are walked in tiles of TK tokens.
//
// Units.  One (pair, key tile) is a unit.  The pairs of a call, in the order sequence, head, row tile, lie
// behind one another on a line: a stretch of HEAD for what a pair costs whatever its keys (its queries,
// filling the pipeline, its result), then its units.  The line is cut into gridDim.x equal runs, one per
// block, whatever the lengths of the sequences: a block may begin and end inside a pair.  What it has
// then is partial -- weighted sum, running maximum and sum of the rows -- and goes to the workspace; a
// second kernel joins the parts of a pair in the order of its keys, so results do not depend on the
// order in which blocks run.  A cut inside a pair's HEAD leaves the whole pair to the block behind it.
// A short line is cut into fewer runs, of LEAST at least: what a part costs to write and to join is then
// not more than what the cut saves, and the blocks left over end at once.
#ifndef KVC_ATTENTION_H
#define KVC_ATTENTION_H

#include <stdint.h>

#include <type_traits>

#include "kvc_device.h"
#include "kvc_internal.h"

#define KVC_ATTN_SMALL_ROWS 16u   // rows of a pair in the kernel for few rows
#define KVC_ATTN_TILE_ROWS 128u   // and in the kernel for many, with one row tile
#define KVC_ATTN_MANY_ROWS 256u   // or two

enum {
    KVC_PHASE_WHOLE = 0,   // sequences are requests, all of their keys
    KVC_PHASE_PREFIX = 1,  // sequences are groups, the keys of their shared prefix
    KVC_PHASE_SUFFIX = 2   // sequences are requests, the keys behind the shared prefix
};

// What a block records about the pair that its run begins inside of.
struct KvcSplit {
    unsigned long long begin, end;  // where the pair's units lie on the line
    unsigned long long length;      // of the line
    uint32_t runs, reserved;        // that it is cut into
    int32_t qa;                     // first token row of the sequence
    uint32_t row0, rows, head;      // first row, rows of the pair, KV head
};

// Parts of one phase in the workspace.
struct KvcParts {
    float *o;        // [slot][ROWS][D] weighted sums
    float2 *ml;      // [slot][ROWS] running maximum (base 2) and sum
    KvcSplit *split; // [block]                                       (WHOLE)
    uint32_t *base;  // [sequence] index of its first pair            (PREFIX, SUFFIX)
    ulonglong2 *range;  // [pair] where its units lie on the line     (PREFIX, SUFFIX)
    unsigned long long *length;  // of the line, and its runs         (PREFIX, SUFFIX)
    uint32_t blocks; // gridDim.x of the kernel that writes them: runs at most
    uint32_t rows;   // ROWS of that kernel
    uint32_t max_pairs;  // pairs that there is room for (PREFIX, SUFFIX): enough for token rows that
                         // ascend, so only lengths that contradict one another can ask for more
};

struct KvcAttn {
    const unsigned char *k, *v;  // planes of the layer
    uint64_t block_stride;
    uint32_t tok_stride;  // bytes between tokens of a block
    uint32_t block_size, num_blocks, max_blocks;
    const int32_t *tables;
    int64_t table_stride;
    const int32_t *seq_lens, *cu_q, *group_starts, *prefix_lens;
    uint32_t n_tokens, n_requests, n_groups;
    const unsigned char *q;
    unsigned char *out;
    float *lse;
    int64_t q_tok, q_head, o_tok, o_head;  // bytes
    uint32_t hq, hkv, g;
    uint32_t g_shift, block_shift;  // log2 of g and of block_size, or KVC_NO_SHIFT
    float scale_log2;
    int32_t window, sinks;
    uint32_t phase;
    uint32_t beside;  // the kernel may run beside the stream's previous one (see kvc_pdl_begin)
    uint32_t *status;
    KvcParts parts;
};

// Pairs of a phase at most: what the workspace is sized by.
inline uint64_t kvc_max_pairs(uint64_t sequences, uint64_t tokens, uint64_t g, uint64_t hkv, uint64_t rows)
{
    return hkv * (sequences + tokens * g / rows);
}

// Implemented in kvc_attention_rows.cu (few rows) and kvc_attention_tiles.cu (many).
uint32_t kvc_attn_rows_blocks(const kvc_layout *lay, bool shared);
cudaError_t kvc_launch_attn_rows(const KvcAttn &a, uint32_t dtype, uint32_t head_dim, uint32_t blocks, cudaStream_t st);
uint32_t kvc_attn_tiles_blocks(const kvc_layout *lay);
cudaError_t kvc_launch_attn_tiles(const KvcAttn &a, uint32_t dtype, uint32_t head_dim, uint32_t blocks, cudaStream_t st);

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t kvc_div_g(const KvcAttn &a, uint32_t x) { return kvc_div(x, a.g, a.g_shift); }

// Where run c of `runs` begins on a line.  (64-bit divisions are worth avoiding: they are a good part of
// what the kernels do before their first load.)
__device__ __forceinline__ unsigned long long kvc_cut(uint32_t c, unsigned long long length, uint32_t runs)
{
    return length < (1ull << 20) ? c * (uint32_t)length / runs : c * length / runs;
}
// The run that holds place x (the last of those that begin there, which is the one that is not empty).
__device__ __forceinline__ uint32_t kvc_run_of(unsigned long long x, unsigned long long length, uint32_t runs)
{
    return length < (1ull << 20) ? (((uint32_t)x + 1) * runs - 1) / (uint32_t)length
                                 : (uint32_t)(((x + 1) * runs - 1) / length);
}

struct KvcSeq {
    int32_t qa, rows;   // first token row; rows (tokens * G)
    int32_t pos;        // position of the first token (may be negative: tokens before the sequence)
    int32_t skip;       // keys before this one belong to the shared prefix (SUFFIX)
    int32_t len;        // keys of the prefix (PREFIX)
    uint32_t table;     // row of the block tables
};

// Largest i in [0, n) with v[i] <= x, for ascending v; 0 where there is none.
__device__ __forceinline__ uint32_t kvc_last_at_most(const int32_t *v, uint32_t n, int32_t x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (v[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// The same for a whole warp at once: 32 places are looked at in one load.
__device__ __forceinline__ uint32_t kvc_last_at_most_warp(const int32_t *v, uint32_t n, int32_t x)
{
    uint32_t lo = 0;
    while (n > 1) {
        const uint32_t step = (n + 31) / 32, at = (threadIdx.x & 31u) * step;
        const uint32_t hit = __ballot_sync(~0u, at < n && v[lo + at] <= x);
        // (a ballot of ascending values is a run of ones from lane 0; taken as 0 where even the first is larger)
        const uint32_t k = hit ? 31u - __clz(hit) : 0u;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

__device__ __forceinline__ int32_t kvc_clamp(int32_t x, int32_t lo, int32_t hi) { return min(max(x, lo), hi); }

// Keys of a request at most: a quarter of the integers' range, so that sums of a position, a window and a
// tile's width stay inside it.
__device__ __forceinline__ int32_t kvc_key_cap(const KvcAttn &a)
{
    return (int32_t)min((uint64_t)a.max_blocks * a.block_size, (uint64_t)KVC_ATTENTION_MAX_KEYS);
}

// The group that holds request r, or -1.
__device__ __forceinline__ int32_t kvc_group_of(const KvcAttn &a, uint32_t r)
{
    if (a.n_groups == 0 || (int32_t)r < a.group_starts[0] || (int32_t)r >= a.group_starts[a.n_groups])
        return -1;
    return (int32_t)kvc_last_at_most(a.group_starts, a.n_groups, (int32_t)r);
}

__device__ __forceinline__ int32_t kvc_prefix_len(const KvcAttn &a, uint32_t group)
{
    return kvc_clamp(a.prefix_lens[group], 0, kvc_key_cap(a));
}

// Lengths come from device memory: token rows are clamped to the rows that q and out have, keys to
// what the table holds, so no value of theirs leads outside a buffer.
__device__ __forceinline__ KvcSeq kvc_seq(const KvcAttn &a, uint32_t s)
{
    KvcSeq q;
    const int32_t top = (int32_t)a.n_tokens;
    if (a.phase == KVC_PHASE_PREFIX) {
        const int32_t R = (int32_t)a.n_requests;
        const int32_t r0 = kvc_clamp(a.group_starts[s], 0, R), r1 = kvc_clamp(a.group_starts[s + 1], r0, R);
        q.qa = kvc_clamp(a.cu_q[r0], 0, top);
        q.rows = (kvc_clamp(a.cu_q[r1], q.qa, top) - q.qa) * (int32_t)a.g;
        q.pos = 0;
        q.skip = 0;
        q.len = kvc_prefix_len(a, s);
        q.table = min((uint32_t)r0, a.n_requests - 1);
    } else {
        q.qa = kvc_clamp(a.cu_q[s], 0, top);
        const int32_t n = kvc_clamp(a.cu_q[s + 1], q.qa, top) - q.qa;
        q.rows = n * (int32_t)a.g;
        q.pos = kvc_clamp(a.seq_lens[s], 0, (int32_t)KVC_ATTENTION_MAX_KEYS) - n;
        q.skip = 0;
        q.len = 0;
        if (a.phase == KVC_PHASE_SUFFIX) {
            const int32_t g = kvc_group_of(a, s);
            q.skip = g < 0 ? 0 : kvc_prefix_len(a, (uint32_t)g);
        }
        q.table = s;
    }
    return q;
}

// The keys that some row of a pair may see, as key tiles: [0, sink_end) and [lo, hi).
struct KvcRange {
    int32_t lo, hi, sink_end;
    uint32_t sink_tiles, first, n;  // tiles 0 .. sink_tiles-1, then first, first+1, ..; n in all, at least one
};

template <int ROWS, int TK>
__device__ __forceinline__ KvcRange kvc_range(const KvcAttn &a, const KvcSeq &q, uint32_t rt)
{
    KvcRange r;
    r.sink_end = 0;
    if (a.phase == KVC_PHASE_PREFIX) {
        r.lo = 0;
        r.hi = q.len;
    } else {
        const int32_t p0 = q.pos + (int32_t)kvc_div_g(a, rt * ROWS);
        const int32_t p1 = q.pos + (int32_t)kvc_div_g(a, min((uint32_t)q.rows, (rt + 1) * ROWS) - 1);
        r.hi = kvc_clamp(p1 + 1, 0, kvc_key_cap(a));
        r.lo = q.skip;
        if (a.window) {
            r.lo = max(0, p0 - a.window + 1);
            r.sink_end = min(a.sinks, min(r.lo, r.hi));
        }
        r.lo = min(r.lo, r.hi);
    }
    r.first = (uint32_t)r.lo / TK;
    r.sink_tiles = min(((uint32_t)r.sink_end + TK - 1) / TK, r.first);
    r.n = max(1u, r.sink_tiles + ((uint32_t)r.hi + TK - 1) / TK - r.first);
    return r;
}

__device__ __forceinline__ uint32_t kvc_tile(const KvcRange &r, uint32_t t)
{
    return t < r.sink_tiles ? t : r.first + (t - r.sink_tiles);
}

// A place in the order of units.
struct KvcCursor {
    uint32_t s, h, rt, t;
    KvcSeq q;
    KvcRange r;
};

template <int ROWS, int TK>
__device__ __forceinline__ void kvc_next(const KvcAttn &a, uint32_t n_seq, KvcCursor &c)
{
    if (++c.t < c.r.n)
        return;
    c.t = 0;
    if (++c.rt * ROWS >= (uint32_t)c.q.rows) {
        c.rt = 0;
        if (++c.h == a.hkv) {
            c.h = 0;
            do {
                if (++c.s >= n_seq)
                    return;
                c.q = kvc_seq(a, c.s);
            } while (c.q.rows == 0);
        }
    }
    c.r = kvc_range<ROWS, TK>(a, c.q, c.rt);
}

// One block's run: its first unit's place and the end of its stretch of the line.  Every thread of the
// block calls this (THREADS of them) and gets the same answer.
struct KvcRun {
    unsigned long long end;
    unsigned long long units_at;  // where the units of the first unit's pair begin on the line
    uint32_t pair;                // index of that pair
    bool any;                     // whether there is a first unit
    KvcCursor at;
    // units of the pair at `at` that belong to the run, from tile t
    __device__ __forceinline__ uint32_t count(const KvcCursor &c, unsigned long long units_at) const
    {
        const unsigned long long from = units_at + c.t;
        return end <= from ? 0u : (uint32_t)min((unsigned long long)(c.r.n - c.t), end - from);
    }
};

template <int ROWS, int TK, int HEAD, int LEAST, int THREADS>
__device__ __forceinline__ KvcRun kvc_find_run(const KvcAttn &a, uint32_t n_seq)
{
    __shared__ unsigned long long sums[THREADS / 32][2];
    __shared__ KvcRun found;
    // A sequence to a thread; or, where there are few sequences of many row tiles, one to a warp whose
    // lanes take its row tiles in turn (one 8192-token prompt: 24 us for one thread, 4 us for a warp).
    const uint32_t lane = threadIdx.x & 31u, w = threadIdx.x >> 5;
    const bool wide = n_seq <= 4u * (THREADS / 32) && (uint64_t)a.n_tokens * a.g >= 4ull * ROWS * n_seq;
    const uint32_t owners = wide ? THREADS / 32 : THREADS, owner = wide ? w : threadIdx.x;
    const uint32_t rt0 = wide ? lane : 0u, rt_step = wide ? 32u : 1u;
    const uint32_t per = (n_seq + owners - 1) / owners;
    const uint32_t s0 = min(owner * per, n_seq), s1 = min(s0 + per, n_seq);
    unsigned long long units = 0, pairs = 0;
    KvcSeq q0;  // the owner's first sequence, usually its only one, and the range of its first row tile, likewise
    KvcRange r0;
#pragma unroll 1
    for (uint32_t s = s0; s < s1; ++s) {
        const KvcSeq q = kvc_seq(a, s);
        if (s == s0)
            q0 = q;
        unsigned long long sum = 0;
        uint32_t n = 0;
#pragma unroll 1
        for (uint32_t rt = rt0; rt * ROWS < (uint32_t)q.rows; rt += rt_step, ++n) {
            const KvcRange r = kvc_range<ROWS, TK>(a, q, rt);
            sum += HEAD + r.n;
            if (s == s0 && rt == 0)
                r0 = r;
        }
        units += sum * a.hkv;
        pairs += (unsigned long long)n * a.hkv;
    }
    unsigned long long iu = units, ip = pairs;
#pragma unroll
    for (uint32_t o = 1; o < 32; o *= 2) {
        const unsigned long long x = __shfl_up_sync(~0u, iu, o), y = __shfl_up_sync(~0u, ip, o);
        if (lane >= o) {
            iu += x;
            ip += y;
        }
    }
    if (lane == 31) {
        sums[w][0] = iu;
        sums[w][1] = ip;
    }
    __syncthreads();
    unsigned long long bu = 0, bp = 0, total = 0;
    for (uint32_t k = 0; k < THREADS / 32; ++k) {
        if (k < w) {
            bu += sums[k][0];
            bp += sums[k][1];
        }
        total += sums[k][0];
    }
    if (wide) {
        units = sums[w][0];
    } else {
        bu += iu - units;
        bp += ip - pairs;
    }
    const uint32_t runs = (uint32_t)max(1ull, min((unsigned long long)gridDim.x, total / LEAST));
    const unsigned long long begin = blockIdx.x < runs ? kvc_cut(blockIdx.x, total, runs) : total;
    const unsigned long long end = blockIdx.x < runs ? kvc_cut(blockIdx.x + 1, total, runs) : total;
    if (threadIdx.x == 0) {
        found.end = end;
        found.any = begin < end;
    }
    // the owner of the sequence that the run begins in walks to the place (of an empty run too: on a line
    // shorter than the number of blocks, the first boundary inside a pair may be that of an empty run)
    const bool mine = begin >= bu && begin < bu + units;
    const bool table = a.phase != KVC_PHASE_WHOLE && blockIdx.x == 0;
    if (mine || table) {
        unsigned long long u = bu, p = bp;
#pragma unroll 1
        for (uint32_t s = s0; s < s1; ++s) {
            if (table && rt0 == 0)
                a.parts.base[s] = (uint32_t)min(p, 0xFFFFFFFFull);
            const KvcSeq q = s == s0 ? q0 : kvc_seq(a, s);
            const uint32_t n = ((uint32_t)q.rows + ROWS - 1) / ROWS;
            const bool one = !wide && n == 1 && s == s0;
            unsigned long long per_head = one ? HEAD + r0.n : 0;
#pragma unroll 1
            for (uint32_t rt = one ? n : rt0; rt < n; rt += rt_step)
                per_head += HEAD + kvc_range<ROWS, TK>(a, q, rt).n;
            if (wide)
#pragma unroll
                for (uint32_t o = 16; o; o /= 2)
                    per_head += __shfl_xor_sync(~0u, per_head, o);
            if (mine && begin >= u && begin < u + per_head * a.hkv) {
                const uint32_t h = per_head < (1ull << 32) && begin - u < (1ull << 32) ? (uint32_t)(begin - u) / (uint32_t)per_head
                                                                                        : (uint32_t)((begin - u) / per_head);
                unsigned long long b = u + h * per_head;
                KvcRange r;
                uint32_t rt = rt0;
                bool here;
#pragma unroll 1
                for (;; rt += rt_step) {
                    // row tiles rt - lane .. of which the lanes hold one each, or just rt
                    uint32_t own = 0;
                    if (rt < n) {
                        r = one ? r0 : kvc_range<ROWS, TK>(a, q, rt);
                        own = HEAD + r.n;
                    }
                    unsigned long long sum = own;
                    if (wide)
#pragma unroll
                        for (uint32_t o = 1; o < 32; o *= 2) {
                            const unsigned long long x = __shfl_up_sync(~0u, sum, o);
                            if (lane >= o)
                                sum += x;
                        }
                    here = begin >= b + sum - own && begin < b + sum;
                    if (wide ? __any_sync(~0u, here) : here) {
                        b += sum - own + HEAD;
                        break;
                    }
                    b += wide ? __shfl_sync(~0u, sum, 31) : sum;
                }
                if (here) {
                    found.units_at = b;
                    found.pair = (uint32_t)(p + (unsigned long long)h * n + rt);
                    found.at.s = s;
                    found.at.h = h;
                    found.at.rt = rt;
                    found.at.t = begin > b ? (uint32_t)(begin - b) : 0u;
                    found.at.q = q;
                    found.at.r = r;
                }
            }
            u += per_head * a.hkv;
            p += (unsigned long long)n * a.hkv;
        }
    }
    __syncthreads();
    KvcRun run = found;
    run.any = run.any && run.count(run.at, run.units_at) != 0;
    if (threadIdx.x == 0) {
        if (a.phase == KVC_PHASE_WHOLE) {
            KvcSplit sp;
            sp.begin = sp.end = 0;
            sp.length = total;
            sp.runs = runs;
            sp.reserved = 0;
            sp.qa = 0;
            sp.row0 = sp.rows = sp.head = 0;
            if (begin < total && run.at.t > 0) {
                sp.begin = run.units_at;
                sp.end = run.units_at + run.at.r.n;
                sp.qa = run.at.q.qa;
                sp.row0 = run.at.rt * ROWS;
                sp.rows = min((uint32_t)ROWS, (uint32_t)run.at.q.rows - sp.row0);
                sp.head = run.at.h;
            }
            a.parts.split[blockIdx.x] = sp;
        } else if (blockIdx.x == 0) {
            a.parts.length[0] = total;
            a.parts.length[1] = runs;
        }
    }
    return run;
}

// The position of a row, for the mask.  In the PREFIX phase the rows of a group belong to several
// requests, and the row's own is looked up.
__device__ __forceinline__ int32_t kvc_row_pos(const KvcAttn &a, const KvcSeq &q, uint32_t row)
{
    const int32_t tok = (int32_t)kvc_div_g(a, row);
    if (a.phase != KVC_PHASE_PREFIX)
        return q.pos + tok;
    const int32_t t = q.qa + tok;
    const uint32_t r = kvc_last_at_most(a.cu_q, a.n_requests, t);
    const int32_t qa = a.cu_q[r], n = kvc_clamp(a.cu_q[r + 1], qa, (int32_t)a.n_tokens) - qa;
    return kvc_clamp(a.seq_lens[r], 0, (int32_t)KVC_ATTENTION_MAX_KEYS) - n + (t - qa);
}

// Whether the row at position p sees key j (which lies in the pair's range).
__device__ __forceinline__ bool kvc_sees(const KvcAttn &a, int32_t p, int32_t j)
{
    return j <= p && (a.window == 0 || p - j < a.window || j < a.sinks);
}

// Where key j of a sequence lies relative to its plane's base, or -1 (an id outside the pool).
__device__ __forceinline__ int64_t kvc_key_offset(const KvcAttn &a, uint32_t table, int32_t j, uint32_t h, uint32_t head_bytes)
{
    const uint32_t b = kvc_div(j, a.block_size, a.block_shift), off = (uint32_t)j - b * a.block_size;
    const uint32_t id = (uint32_t)a.tables[(int64_t)table * a.table_stride + b];
    if (id >= a.num_blocks)
        return -1;
    return (int64_t)((uint64_t)id * a.block_stride + (uint64_t)off * a.tok_stride + (uint64_t)h * head_bytes);
}

#endif  // __CUDACC__
#endif
