// The step's tokens: block tables and slots built from request lengths (kvc_map_tokens), and the
// per-head norm, rotation and cache write of their queries, keys and values (kvc_append).
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "kvc_internal.h"
#include "kvc_device.h"

namespace {

// ------------------------------------------------------------------------------------ map_tokens
//
// hb = ceil(context / B) blocks are held already, ha = ceil((context + new) / B) are needed; the
// ha - hb new ones come from the free list in request order, so the exclusive prefix sums of `new`
// (token rows) and of ha - hb (free-list positions) give every output independently of the others.
// Every block redoes the two sums over all requests -- 8 bytes each, read from L2 -- instead of
// waiting for another block's result: one launch, no flags, the same integers every time.  What
// bounds the call is that chain (two dependent loads, one block scan, one binary search in shared
// memory, one table read), not the 16 bytes it writes per token.
struct MapArgs {
    const int32_t *context_lens, *new_lens, *free_blocks;
    int32_t *tables;
    int64_t table_stride;
    uint32_t max_blocks, n_requests, n_free, capacity, block_size, block_shift, num_blocks;
    int32_t *cu, *total_lens, *positions, *request, *counts;
    int64_t *slots;
    uint32_t *status;
};

__device__ __forceinline__ int32_t sat32(int64_t v) { return v > 0x7FFFFFFFll ? 0x7FFFFFFF : (int32_t)v; }

struct MapReq {
    int32_t ctx, add;  // tokens held, tokens of this step (ctx + add <= INT32_MAX)
    uint32_t hb, ha;   // blocks held, blocks needed (both at most max_blocks)
};

// Blocks that n tokens (at most 2^31 - 1) take.
__device__ __forceinline__ uint32_t map_blocks(const MapArgs &a, uint32_t n)
{
    const uint32_t q = kvc_div(n, a.block_size, a.block_shift);
    return q + (q * a.block_size != n);
}

__device__ __forceinline__ MapReq map_req(const MapArgs &a, uint32_t r)
{
    MapReq q;
    q.ctx = max(a.context_lens[r], 0);
    q.add = max(min(a.new_lens[r], 0x7FFFFFFF - q.ctx), 0);
    q.ha = min(map_blocks(a, (uint32_t)q.ctx + (uint32_t)q.add), a.max_blocks);
    q.hb = min(map_blocks(a, (uint32_t)q.ctx), q.ha);
    if (q.add == 0)
        q.ha = q.hb;  // nothing is added: nothing is taken
    return q;
}

// Largest r in [0, n) with v[r] <= x (v ascending, v[0] = 0).
__device__ __forceinline__ uint32_t last_at_most(const int32_t *v, uint32_t n, int32_t x)
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

template <uint32_t MAP_THREADS>
__global__ void __launch_bounds__(MAP_THREADS) kvc_map_tokens_kernel(const MapArgs a)
{
    extern __shared__ int32_t sm[];
    const uint32_t R = a.n_requests;
    int32_t *cu = sm;               // [R + 1] first token row of each request
    int32_t *fb = sm + R + 1;       // [R + 1] first free-list position of each request
    int32_t *ctx = sm + 2 * (R + 1);  // [R] tokens held
    __shared__ int64_t warp_sum[2][MAP_THREADS / 32];
    kvc_pdl_wait();

    const uint32_t per = (R + MAP_THREADS - 1) / MAP_THREADS;
    const uint32_t r0 = min(threadIdx.x * per, R), r1 = min(r0 + per, R);
    int64_t st = 0, sb = 0;
    for (uint32_t r = r0; r < r1; ++r) {
        const MapReq q = map_req(a, r);
        st += q.add;
        sb += q.ha - q.hb;
    }
    const uint32_t lane = threadIdx.x & 31u, w = threadIdx.x >> 5;
    int64_t it = st, ib = sb;
#pragma unroll
    for (uint32_t o = 1; o < 32; o *= 2) {
        const int64_t x = __shfl_up_sync(~0u, it, o), y = __shfl_up_sync(~0u, ib, o);
        if (lane >= o) {
            it += x;
            ib += y;
        }
    }
    if (lane == 31) {
        warp_sum[0][w] = it;
        warp_sum[1][w] = ib;
    }
    __syncthreads();
    int64_t bt = 0, bb = 0, tt = 0, tb = 0;  // sums of earlier warps, sums of all
    for (uint32_t k = 0; k < MAP_THREADS / 32; ++k) {
        if (k < w) {
            bt += warp_sum[0][k];
            bb += warp_sum[1][k];
        }
        tt += warp_sum[0][k];
        tb += warp_sum[1][k];
    }
    bt += it - st;
    bb += ib - sb;
    int64_t no_block = 0;
    const bool first = blockIdx.x == 0;
    for (uint32_t r = r0; r < r1; ++r) {
        const MapReq q = map_req(a, r);
        cu[r] = sat32(bt);
        fb[r] = sat32(bb);
        ctx[r] = q.ctx;
        if (first) {
            a.cu[r] = sat32(bt);
            if (a.total_lens)
                a.total_lens[r] = q.ctx + q.add;
            // tokens past the blocks that the table and the free list provide
            const int64_t have = (int64_t)q.hb + min(max((int64_t)a.n_free - bb, (int64_t)0), (int64_t)(q.ha - q.hb));
            const int64_t limit = max(have * a.block_size, (int64_t)q.ctx);
            no_block += max((int64_t)q.ctx + q.add - limit, (int64_t)0);
        }
        bt += q.add;
        bb += q.ha - q.hb;
    }
    if (threadIdx.x == 0) {
        cu[R] = sat32(tt);
        fb[R] = sat32(tb);
    }
    __syncthreads();
    if (first) {
        if (threadIdx.x == 0)
            a.cu[R] = sat32(tt);
        if (a.counts) {
#pragma unroll
            for (uint32_t o = 16; o; o /= 2)
                no_block += __shfl_xor_sync(~0u, no_block, o);
            if (lane == 0)
                warp_sum[0][w] = no_block;
            __syncthreads();
            if (threadIdx.x == 0) {
                int64_t sum = 0;
                for (uint32_t k = 0; k < MAP_THREADS / 32; ++k)
                    sum += warp_sum[0][k];
                a.counts[0] = sat32(tt);
                a.counts[1] = (int32_t)min(tb, (int64_t)a.n_free);
                a.counts[2] = sat32(sum);
            }
        }
    }

    const uint32_t B = a.block_size;
    const uint32_t step = gridDim.x * MAP_THREADS, at = blockIdx.x * MAP_THREADS + threadIdx.x;
    // new table entries
    const uint32_t n_new = (uint32_t)fb[R];
    for (uint64_t i = at; i < n_new; i += step) {
        const uint32_t r = last_at_most(fb, R, (int32_t)i);
        const uint32_t hb = min(map_blocks(a, (uint32_t)ctx[r]), a.max_blocks);
        a.tables[(int64_t)r * a.table_stride + hb + (i - (uint32_t)fb[r])] = i < a.n_free ? a.free_blocks[i] : -1;
    }
    // token rows; the rows behind the last token are marked as holding none
    const uint32_t n_tok = min((uint32_t)cu[R], a.capacity);
    for (uint64_t i = at; i < a.capacity; i += step) {
        int64_t slot = -1;
        int32_t pos = 0, req = -1;
        if (i < n_tok) {
            const uint32_t r = last_at_most(cu, R, (int32_t)i);
            req = (int32_t)r;
            pos = ctx[r] + (int32_t)(i - (uint32_t)cu[r]);
            const uint32_t bi = kvc_div((uint32_t)pos, B, a.block_shift), off = (uint32_t)pos - bi * B;
            if (bi < a.max_blocks) {
                const uint32_t hb = map_blocks(a, (uint32_t)ctx[r]);
                int32_t id = -1;
                bool have = true;
                if (bi < hb) {  // the block that the context's last token lies in
                    id = a.tables[(int64_t)r * a.table_stride + bi];
                } else {
                    const uint32_t f = (uint32_t)fb[r] + (bi - hb);
                    have = f < a.n_free;
                    if (have)
                        id = a.free_blocks[f];
                }
                if ((uint32_t)id < a.num_blocks)
                    slot = (int64_t)id * B + off;
                else if (have)
                    atomicAdd(a.status, 1u);  // an entry that names no block of the pool
            }
        }
        a.slots[i] = slot;
        a.positions[i] = pos;
        if (a.request)
            a.request[i] = req;
    }
}

// ------------------------------------------------------------------------------------ append
//
// y = x * rsqrt(mean(x^2) + eps) * w over each head, then the rotation of its first `rot` values by
// the row of the cos/sin table at the token's position; values are copied.  All in 32 bits, rounded
// once to the pool's type.  Every element is read once and written once, so memory is the bound, and
// the arithmetic has to stay out of its way: with one lane to 16 bytes and the partner of each value
// fetched by shuffle it took 110 instructions a lane and twice the time of the copy.  So a lane holds
// both values of each of its pairs -- for "halves" 8 bytes of either half, four lanes' worth a sector --
// and the weights are folded into the angles once a token: with c, s the angle's and e, o the pair,
//     y_e = inv * ((w_e c) x_e - (w_o s) x_o),   y_o = inv * ((w_o c) x_o + (w_e s) x_e),
// two pairs an instruction.  A team of head_dim / 8 lanes (rounded up to a power of two) holds one head;
// a warp serves several heads of one token and one kind (queries, keys or values).
struct AppendArgs {
    const unsigned char *src[3];          // queries, keys, values
    int64_t src_tok[3], src_head[3];      // strides in bytes
    unsigned char *q_out, *k_plane, *v_plane;
    int64_t o_tok, o_head;
    uint64_t block_stride;
    const int64_t *slots;
    const int32_t *positions;
    const float *cos_sin;
    int64_t cs_stride;  // floats
    const void *weight[2];
    float eps;
    uint32_t n_tokens, heads[2], d, rot, max_pos, block_size, block_shift, num_blocks;  // heads: queries; keys and values
    uint32_t lanes;        // lanes per head: a power of two >= d / 8
    uint32_t chunk;        // heads per warp unit
    uint32_t q_chunks, kv_chunks;  // units per token
    uint32_t *status;
};

#define APPEND_THREADS 64u
// Small blocks, 16 a SM: a block's warps go through the same chain (slot, angles, heads) at the same time, and
// small ones start and end more evenly (16384 tokens of 64 + 16 heads: 153 us with 256 threads, 141 with 128,
// 132 with 64).  Four heads a team and turn, two turns: with one turn the angles are fetched too often, with more
// or wider ones too few warps fit (155 to 260 us).
#define APPEND_BLOCKS 16
#define APPEND_UNROLL 4
#define APPEND_CHUNK 2

// A lane's eight values as two words of either piece, and as two pairs of floats an operand.
struct AppendRaw {
    uint2 a, b;
};

// NEIGHBOURS: pairs are (2n, 2n+1), else (n, n + rot/2).  VEC: rows of the cos/sin table are 16-byte aligned.
// PART: some of a head is not rotated (the choice between the two for every pair is 1.5 % of the time, which calls that
// rotate whole heads need not pay).
template <typename T, bool NEIGHBOURS, bool VEC, bool PART>
__global__ void __launch_bounds__(APPEND_THREADS, APPEND_BLOCKS) kvc_append_kernel(const AppendArgs a)
{
    kvc_pdl_wait();
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t team = lane / a.lanes, teams = 32u / a.lanes, l = lane % a.lanes;
    const bool on = l * 8u < a.d, turned = l * 8u < a.rot;
    // first elements of the lane's two pieces of four
    const uint32_t ea = !NEIGHBOURS && turned ? 4u * l : 8u * l, eb = !NEIGHBOURS && turned ? a.rot / 2 + 4u * l : 8u * l + 4u;
    const uint32_t per_token = a.q_chunks + 2 * a.kv_chunks;
    const uint32_t u = blockIdx.x * (APPEND_THREADS / 32u) + (threadIdx.x >> 5);  // (two warps in 2^31 blocks)
    const uint32_t tok = u / per_token;
    if (tok >= a.n_tokens)
        return;
    uint32_t part = u - tok * per_token, kind = 0;
    if (part >= a.q_chunks) {
        part -= a.q_chunks;
        kind = 1;
        if (part >= a.kv_chunks) {
            part -= a.kv_chunks;
            kind = 2;
        }
    }
    const uint32_t h0 = part * a.chunk, h1 = min(h0 + a.chunk, a.heads[kind != 0]);
    const unsigned char *src = a.src[kind] + tok * a.src_tok[kind];
    const int64_t src_head = a.src_head[kind];
    AppendRaw raw[APPEND_UNROLL];
    const auto load = [&](uint32_t hb) {
#pragma unroll
        for (int i = 0; i < APPEND_UNROLL; ++i) {
            const uint32_t h = hb + i * teams;
            raw[i].a = raw[i].b = make_uint2(0, 0);
            if (h < h1 && on) {
                raw[i].a = __ldcs(reinterpret_cast<const uint2 *>(src + h * src_head + ea * 2u));
                raw[i].b = __ldcs(reinterpret_cast<const uint2 *>(src + h * src_head + eb * 2u));
            }
        }
    };
    // the first heads are on their way before the slot, the position and the angles are
    load(h0 + team);
    const int64_t slot = a.slots[tok];
    if (slot < 0)
        return;  // a row without a token
    const int32_t pos = a.rot ? a.positions[tok] : 0;
    const uint64_t id = (uint64_t)slot < (1ull << 32) ? kvc_div((uint32_t)slot, a.block_size, a.block_shift) : (uint64_t)slot / a.block_size;
    if (id >= a.num_blocks || (a.rot && (uint32_t)pos >= a.max_pos)) {
        if (lane == 0 && u == tok * per_token)
            atomicAdd(a.status, 1u);
        return;
    }
    unsigned char *dst = kind == 0 ? a.q_out + tok * a.o_tok
                                   : (kind == 1 ? a.k_plane : a.v_plane) + id * a.block_stride +
                                         ((uint64_t)slot - id * a.block_size) * a.heads[1] * a.d * sizeof(T);
    const int64_t dst_head = kind == 0 ? a.o_head : (int64_t)(a.d * sizeof(T));
    // w_e c, -w_o s, w_o c, w_e s of the lane's four pairs
    uint64_t ec[2], os[2], oc[2], es[2];
    const void *weight = kind < 2 ? a.weight[kind] : nullptr;
    if (kind < 2) {
        float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f}, we[4] = {1.f, 1.f, 1.f, 1.f}, wo[4] = {1.f, 1.f, 1.f, 1.f};
        if (turned) {
            const float *row = a.cos_sin + (int64_t)pos * a.cs_stride + 4u * l;
            if (VEC) {
                const float4 x = *reinterpret_cast<const float4 *>(row), y = *reinterpret_cast<const float4 *>(row + a.rot / 2);
                c[0] = x.x, c[1] = x.y, c[2] = x.z, c[3] = x.w;
                s[0] = y.x, s[1] = y.y, s[2] = y.z, s[3] = y.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[i] = row[i];
                    s[i] = row[a.rot / 2 + i];
                }
            }
        }
        if (weight && on) {
            const unsigned char *w = static_cast<const unsigned char *>(weight);
            const uint2 x = *reinterpret_cast<const uint2 *>(w + ea * 2u), y = *reinterpret_cast<const uint2 *>(w + eb * 2u);
            const float2 p = kvc_to_float2<T>(x.x), q = kvc_to_float2<T>(x.y), r = kvc_to_float2<T>(y.x), t = kvc_to_float2<T>(y.y);
            if (NEIGHBOURS) {
                we[0] = p.x, wo[0] = p.y, we[1] = q.x, wo[1] = q.y, we[2] = r.x, wo[2] = r.y, we[3] = t.x, wo[3] = t.y;
            } else {
                we[0] = p.x, we[1] = p.y, we[2] = q.x, we[3] = q.y, wo[0] = r.x, wo[1] = r.y, wo[2] = t.x, wo[3] = t.y;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            ec[i] = kvc_pair(we[2 * i] * c[2 * i], we[2 * i + 1] * c[2 * i + 1]);
            oc[i] = kvc_pair(wo[2 * i] * c[2 * i], wo[2 * i + 1] * c[2 * i + 1]);
            es[i] = kvc_pair(we[2 * i] * s[2 * i], we[2 * i + 1] * s[2 * i + 1]);
            os[i] = kvc_pair(-wo[2 * i] * s[2 * i], -wo[2 * i + 1] * s[2 * i + 1]);
        }
    }
    const float inv_d = 1.0f / (float)a.d;
    for (uint32_t hb = h0 + team;;) {
#pragma unroll
        for (int i = 0; i < APPEND_UNROLL; ++i) {
            const uint32_t h = hb + i * teams;
            if (h - team >= h1)  // (whole warps: a team past the unit's heads goes through the shuffles with zeros)
                break;
            AppendRaw res = raw[i];
            if (kind < 2) {
                const float2 p = kvc_to_float2<T>(res.a.x), q = kvc_to_float2<T>(res.a.y), r = kvc_to_float2<T>(res.b.x),
                             t = kvc_to_float2<T>(res.b.y);
                uint64_t e[2], o[2];
                if (NEIGHBOURS) {
                    e[0] = kvc_pair(p.x, q.x), o[0] = kvc_pair(p.y, q.y), e[1] = kvc_pair(r.x, t.x), o[1] = kvc_pair(r.y, t.y);
                } else {
                    e[0] = kvc_pair(p.x, p.y), e[1] = kvc_pair(q.x, q.y), o[0] = kvc_pair(r.x, r.y), o[1] = kvc_pair(t.x, t.y);
                }
                float inv = 1.f;
                if (weight) {
                    const float2 sq = kvc_unpair(kvc_fma2(o[1], o[1], kvc_fma2(o[0], o[0], kvc_fma2(e[1], e[1], kvc_mul2(e[0], e[0])))));
                    float sum = sq.x + sq.y;
                    for (uint32_t n = a.lanes / 2; n; n /= 2)
                        sum += __shfl_xor_sync(~0u, sum, n);
                    inv = rsqrtf(sum * inv_d + a.eps);
                }
                const uint64_t inv2 = kvc_pair(inv, inv);
                float2 ye[2], yo[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    // (a value outside the rotation takes nothing from its neighbour, not even zero times it, which
                    // would turn the neighbour's infinity into NaN here, or -0 into 0)
                    const uint64_t ce = kvc_mul2(ec[n], e[n]), co = kvc_mul2(oc[n], o[n]);
                    ye[n] = kvc_unpair(kvc_mul2(inv2, !PART || turned ? kvc_fma2(os[n], o[n], ce) : ce));
                    yo[n] = kvc_unpair(kvc_mul2(inv2, !PART || turned ? kvc_fma2(es[n], e[n], co) : co));
                }
                if (NEIGHBOURS) {
                    res.a = make_uint2(kvc_from_float2<T>(ye[0].x, yo[0].x), kvc_from_float2<T>(ye[0].y, yo[0].y));
                    res.b = make_uint2(kvc_from_float2<T>(ye[1].x, yo[1].x), kvc_from_float2<T>(ye[1].y, yo[1].y));
                } else {
                    res.a = make_uint2(kvc_from_float2<T>(ye[0].x, ye[0].y), kvc_from_float2<T>(ye[1].x, ye[1].y));
                    res.b = make_uint2(kvc_from_float2<T>(yo[0].x, yo[0].y), kvc_from_float2<T>(yo[1].x, yo[1].y));
                }
            }
            if (h < h1 && on) {
                __stcs(reinterpret_cast<uint2 *>(dst + h * dst_head + ea * 2u), res.a);
                __stcs(reinterpret_cast<uint2 *>(dst + h * dst_head + eb * 2u), res.b);
            }
        }
        hb += teams * APPEND_UNROLL;
        if (hb - team >= h1)
            break;
        load(hb);
    }
}

inline bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

struct Span {
    const void *at;  // or NULL
    uint64_t bytes;
};
inline bool overlap(const Span &a, const Span &b)
{
    const uint64_t x = (uint64_t)(uintptr_t)a.at, y = (uint64_t)(uintptr_t)b.at;
    return x && y && a.bytes && b.bytes && (x < y ? y - x < a.bytes : x - y < b.bytes);
}
// Rows of a table, `stride` bytes apart; what lies between them is not the table's.
struct Rows {
    Span first;
    uint64_t stride, n;
};
inline bool overlap(const Span &a, const Rows &b)
{
    const uint64_t x = (uint64_t)(uintptr_t)a.at, y = (uint64_t)(uintptr_t)b.first.at;
    if (b.n == 0 || x <= y || b.n == 1)
        return b.n && overlap(a, b.first);
    // the row at whose place `a` begins, and the one behind it
    const uint64_t row = b.stride ? (x - y) / b.stride : 0, off = (x - y) - row * b.stride;
    return a.at && b.first.at && a.bytes && b.first.bytes &&
           ((row < b.n && off < b.first.bytes) || (row + 1 < b.n && a.bytes > b.stride - off));
}

}  // namespace

extern "C" {

kvc_status kvc_map_tokens(kvc_layout *lay, const kvc_map_tokens_desc *d, void *stream)
{
    if (!lay || !d || d->reserved != 0)
        return KVC_ERR_INVALID_ARG;
    if (d->n_requests > KVC_MAP_MAX_REQUESTS)
        return KVC_ERR_TOO_LARGE;
    if (!d->cu_tokens || (d->n_requests && (!d->context_lens || !d->new_lens)) || (d->n_free && !d->free_blocks) ||
        (d->token_capacity && (!d->positions || !d->slots)) || (d->n_requests && d->max_blocks && !d->block_tables) ||
        d->token_capacity > 0x7FFFFFFFu || d->n_free > 0x7FFFFFFFu ||
        (d->n_requests > 1 && d->table_stride < d->max_blocks))
        return KVC_ERR_INVALID_ARG;
    if (!aligned(d->cu_tokens, 4) || !aligned(d->context_lens, 4) || !aligned(d->new_lens, 4) ||
        !aligned(d->free_blocks, 4) || !aligned(d->block_tables, 4) || !aligned(d->positions, 4) ||
        !aligned(d->slots, 8) || !aligned(d->token_request, 4) || !aligned(d->total_lens, 4) || !aligned(d->counts, 4))
        return KVC_ERR_ALIGNMENT;
    // Every block reads the lengths, and those that finish early write beside blocks that have not read yet
    const uint64_t r = d->n_requests, t = d->token_capacity;
    const Span outs[] = {{d->cu_tokens, 4 * (r + 1)}, {d->positions, 4 * t}, {d->slots, 8 * t}, {d->token_request, 4 * t},
                         {d->total_lens, 4 * r}, {d->counts, 12}};
    const Span ins[] = {{d->context_lens, 4 * r}, {d->new_lens, 4 * r}, {d->free_blocks, 4ull * d->n_free}};
    const Rows tables = {{d->block_tables, 4ull * d->max_blocks}, 4 * d->table_stride, r};
    for (const Span &o : outs) {
        for (const Span &x : ins)
            if (overlap(o, x))
                return KVC_ERR_INVALID_ARG;
        for (const Span *x = outs; x != &o; ++x)
            if (overlap(o, *x))
                return KVC_ERR_INVALID_ARG;
        if (overlap(o, tables))
            return KVC_ERR_INVALID_ARG;
    }
    for (const Span &x : ins)
        if (overlap(x, tables))
            return KVC_ERR_INVALID_ARG;
    kvc_status s = kvc_ensure_device(lay);
    if (s != KVC_OK)
        return s;
    MapArgs a;
    a.context_lens = d->context_lens;
    a.new_lens = d->new_lens;
    a.free_blocks = d->free_blocks;
    a.tables = d->block_tables;
    a.table_stride = (int64_t)d->table_stride;
    a.max_blocks = d->max_blocks;
    a.n_requests = d->n_requests;
    a.n_free = d->n_free;
    a.capacity = d->token_capacity;
    a.block_size = lay->d.block_size;
    a.block_shift = kvc_shift_of(a.block_size);
    a.num_blocks = lay->d.num_blocks;
    a.cu = d->cu_tokens;
    a.total_lens = d->total_lens;
    a.positions = d->positions;
    a.request = d->token_request;
    a.counts = d->counts;
    a.slots = d->slots;
    a.status = lay->d_status;
    const uint32_t smem = (3 * d->n_requests + 2) * sizeof(int32_t);
    // A small step is the chain of one block's scan, which fewer threads go through faster (64 requests: 3.5 us
    // with blocks of 256, 5.4 with 1024); of a large one every block repeats the scan, so one large block a SM
    // (1001 requests, 270,000 rows: 7.9 us, and 10.7 with 256).
    const auto go = [&](auto kernel, uint32_t threads, uint32_t blocks) {
        if (smem > 48 * 1024 &&
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)((3 * KVC_MAP_MAX_REQUESTS + 2) * sizeof(int32_t))) != cudaSuccess)
            return cudaErrorUnknown;
        const uint32_t want = (d->token_capacity + threads - 1) / threads;
        return kvc_launch_pdl(kernel, a, dim3(std::max<uint32_t>(1u, std::min(want, blocks))), threads, smem, (cudaStream_t)stream);
    };
    const bool small = d->token_capacity <= 256u * (uint32_t)lay->sm_count;
    if ((small ? go(kvc_map_tokens_kernel<256>, 256, (uint32_t)lay->sm_count) : go(kvc_map_tokens_kernel<1024>, 1024, (uint32_t)lay->sm_count)) !=
        cudaSuccess) {
        (void)cudaGetLastError();
        return KVC_ERR_CUDA;
    }
    ++lay->launches;
    kvc_step_launched(lay->device, (cudaStream_t)stream);
    return KVC_OK;
}

kvc_status kvc_append(kvc_layout *lay, const kvc_append_desc *d, void *stream)
{
    if (!lay || !d || d->reserved != 0)
        return KVC_ERR_INVALID_ARG;
    const uint32_t hkv = lay->d.num_kv_heads, dim = lay->d.head_dim;
    if (d->layer >= lay->d.num_layers || lay->d.kv_planes != 2 || lay->d.elem_bytes != 2 ||
        (d->dtype != KVC_DTYPE_BF16 && d->dtype != KVC_DTYPE_FP16))
        return KVC_ERR_INVALID_ARG;
    if (dim % 8 || dim > 256 || d->rot_dim > dim || d->rot_dim % 16 || d->interleaved > 1u ||
        !(d->eps >= 0.f) || d->n_tokens > 0x7FFFFFFFu || d->n_q_heads > 0x10000u)
        return KVC_ERR_INVALID_ARG;
    if (d->n_tokens == 0)
        return KVC_OK;
    if (!d->k || !d->v || !d->slots || (d->n_q_heads && (!d->q || !d->q_out)) ||
        (d->rot_dim && (!d->positions || !d->cos_sin || d->cos_sin_stride < d->rot_dim)))
        return KVC_ERR_INVALID_ARG;
    if (!aligned(d->k, 16) || !aligned(d->v, 16) || !aligned(d->q, 16) || !aligned(d->q_out, 16) ||
        !aligned(d->q_weight, 16) || !aligned(d->k_weight, 16) || !aligned(d->slots, 8) ||
        !aligned(d->positions, 4) || !aligned(d->cos_sin, 4))
        return KVC_ERR_ALIGNMENT;
    if ((d->q_token_stride | d->q_head_stride | d->k_token_stride | d->k_head_stride | d->v_token_stride |
         d->v_head_stride | d->out_token_stride | d->out_head_stride) % 8)
        return KVC_ERR_ALIGNMENT;
    kvc_status s = kvc_ensure_device(lay);
    if (s != KVC_OK)
        return s;
    AppendArgs a;
    a.src[0] = static_cast<const unsigned char *>(d->q);
    a.src[1] = static_cast<const unsigned char *>(d->k);
    a.src[2] = static_cast<const unsigned char *>(d->v);
    const int64_t tok[3] = {d->q_token_stride, d->k_token_stride, d->v_token_stride};
    const int64_t head[3] = {d->q_head_stride, d->k_head_stride, d->v_head_stride};
    for (int i = 0; i < 3; ++i) {
        a.src_tok[i] = 2 * tok[i];
        a.src_head[i] = 2 * head[i];
    }
    a.q_out = static_cast<unsigned char *>(d->q_out);
    a.k_plane = const_cast<unsigned char *>(kvc_plane_ptr(lay, d->layer, 0));
    a.v_plane = const_cast<unsigned char *>(kvc_plane_ptr(lay, d->layer, 1));
    a.o_tok = 2 * d->out_token_stride;
    a.o_head = 2 * d->out_head_stride;
    a.block_stride = lay->block_stride;
    a.slots = d->slots;
    a.positions = d->positions;
    a.cos_sin = d->cos_sin;
    a.cs_stride = (int64_t)d->cos_sin_stride;
    a.weight[0] = d->q_weight;
    a.weight[1] = d->k_weight;
    a.eps = d->eps;
    a.n_tokens = d->n_tokens;
    a.heads[0] = d->n_q_heads;
    a.heads[1] = hkv;
    a.d = dim;
    a.rot = d->rot_dim;
    a.max_pos = d->max_positions;
    a.block_size = lay->d.block_size;
    a.block_shift = kvc_shift_of(a.block_size);
    a.num_blocks = lay->d.num_blocks;
    a.status = lay->d_status;
    a.lanes = 1;
    while (a.lanes * 8 < dim)
        a.lanes *= 2;
    // Heads per warp: the fewest that fill the machine's warps once -- a warp that serves more heads
    // of its token fetches the table row once for them, one that serves fewer spreads a small call
    // over more SMs.
    const uint32_t heads = d->n_q_heads + 2 * hkv, teams = 32 / a.lanes;
    const uint64_t warps = (uint64_t)lay->sm_count * APPEND_BLOCKS * (APPEND_THREADS / 32);
    uint64_t chunk = (uint64_t)d->n_tokens * heads / warps;
    chunk = std::max<uint64_t>((chunk + teams - 1) / teams * teams, teams);
    a.chunk = (uint32_t)std::min<uint64_t>(chunk, (uint64_t)APPEND_CHUNK * APPEND_UNROLL * teams);
    a.q_chunks = (d->n_q_heads + a.chunk - 1) / a.chunk;
    a.kv_chunks = (hkv + a.chunk - 1) / a.chunk;
    const uint64_t units = (uint64_t)d->n_tokens * (a.q_chunks + 2 * a.kv_chunks);
    const uint32_t per_block = APPEND_THREADS / 32;
    if ((units + per_block - 1) / per_block > 0x7FFFFFFFull)
        return KVC_ERR_TOO_LARGE;
    const uint32_t grid = (uint32_t)((units + per_block - 1) / per_block);
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    const bool vec = aligned(d->cos_sin, 16) && d->cos_sin_stride % 4 == 0, part = d->rot_dim < dim;
    const auto go = [&](auto type, auto neighbours, auto v, auto p) {
        return kvc_launch_pdl(kvc_append_kernel<decltype(type), decltype(neighbours)::value, decltype(v)::value, decltype(p)::value>, a,
                              dim3(grid), APPEND_THREADS, 0, st);
    };
    const auto go2 = [&](auto type, auto neighbours) {
        const std::true_type yes;
        const std::false_type no;
        return vec ? (part ? go(type, neighbours, yes, yes) : go(type, neighbours, yes, no))
                   : (part ? go(type, neighbours, no, yes) : go(type, neighbours, no, no));
    };
    const auto pick = [&](auto type) { return d->interleaved ? go2(type, std::true_type()) : go2(type, std::false_type()); };
    e = d->dtype == KVC_DTYPE_BF16 ? pick(__nv_bfloat16()) : pick(__half());
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return KVC_ERR_CUDA;
    }
    ++lay->launches;
    kvc_step_launched(lay->device, (cudaStream_t)stream);
    return KVC_OK;
}

}  // extern "C"
