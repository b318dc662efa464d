// Attention over the paged pool for many query rows (prompts, and the shared prefix of a group): tiles
// of 256 or 128 rows against tiles of 128 keys on the fifth-generation tensor cores.
//
// Per row: s_j = scale * q . k_j, o = sum_j 2^(s_j' - m) v_j / sum_j 2^(s_j' - m), s' in base 2; one pass
// with the running maximum and sum of a softmax in 32 bits.
//
// One block a SM, specialised by warp:
//   warps 0-7, 8-15 softmax of rows 0-127 and 128-255, two threads a row, one for each half of a tile's
//                   keys: read S from tensor memory, agree on the maximum, write the weights P (pool's type)
//                   over S, keep m and l in registers; at the end of a pair each writes half of O's columns.
//                   They also load the queries.
//   warp 16         issues the matrix instructions, one lane each but the whole warp along: S = Q K^T from shared memory, O += P V
//                   with P from tensor memory and V as it lies (keys x head, so head-major for this product)
//   warps 17, 18    load K and V tiles through the block table into rings of shared-memory stages, in the
//                   128-byte swizzle that the matrix unit reads: a tensor copy for the keys of each block, or
//                   16-byte asynchronous copies where a tile is not made of whole blocks
//   warp 19         one thread walks the run's pairs and hands them to the others
// Two row tiles share each K and V tile, and while one is in its softmax the other's products run.  A pair
// of 128 rows or fewer has one row tile; its scores then alternate between the two score buffers, so that
// those of the next tile are made while this one is in its softmax (16 requests of up to 5 drafted tokens
// behind 16,000, 64 and 8 heads of 128: a sixth less time than with one buffer, 204 us).
// Bound by the exponentials and the matrix unit alike: 128 x 128 scores take 1024 cycles on each.  Measured:
// an 8192-token prompt (32 and 8 heads of 128, 550 GFLOP) in 600 us = 916 TFLOP/s in runs of five, and in 666 us =
// 825 TFLOP/s in a loop of seconds, where the power limit holds the clock at 1.76 GHz; either unit is busy 45 % of the
// time.  What is left is the chain scores - maximum - weights - products - next scores of either row tile, with a
// meeting of the two warps of a row in it, and some spills (96 registers a thread, 224 bytes read back).
// Moving a part of the exponentials to the multiply-add pipe, smaller key tiles and one softmax thread a
// row were all slower.
// O is rescaled only when a row's maximum has grown by more than 2^8 over the one in use (a published refinement of the
// online softmax of Milakov and Gimelshein, 2018): weights are then at most 2^8, which neither type nor the 32-bit sums
// mind, and almost all tiles skip the rescaling.
// Weights are rounded to the pool's type, since the matrix unit takes 16-bit operands of one type; a second product
// for what the rounding leaves would be half as much tensor work again.  Against 64 bits the result is off by 0.0021 to
// 0.0023 in bf16 (0.0017 with weights in 32 bits: the result's own rounding) and 0.0003 in fp16 (0.0002).
// Every wait is bounded; one that gives up makes all roles leave and is counted.
#include <cuda.h>
#include <stddef.h>
#include <string.h>

#include "kvc_attention.h"

namespace {

constexpr int TK = 128;             // keys of a K or V stage
constexpr int HK = TK / 2;          // keys of one softmax thread
constexpr int THREADS = 640;
constexpr int HEAD = 3;             // what a pair costs besides its units, in units (8192-token prompt: 670, 621, 601, 607 us with 1 to 4)
constexpr int LEAST = 3;            // units of a run at least (64 requests on a 1024-token prefix: 76, 71, 72 us with 2 to 4)
constexpr uint32_t THERE = 8;  // ring of "which keys are there" words, deeper than the K ring

// ROWS is 256, two row tiles a block, or 128, one: half the queries then make room for a third K stage, which long
// runs of keys gain by (one request of drafted tokens behind 80,000: 85.4 us with 256, 83.6 with 128; 32 questions on a
// 32,000-token document 71.2 and 69.5; but 16 requests of drafted tokens behind 16,000 202.4 and 204.5).
template <int D, int ROWS>
struct Shape {
    static constexpr int TILE = TK * D * 2;           // a K or V tile; also the queries of a row tile
    static constexpr int HALF = TK * 128;             // 64 elements (128 bytes) of 128 rows
    static constexpr int KS = D == 64 ? 4 : ROWS == 128 ? 3 : 2, VS = D == 64 ? 4 : 2;
    static constexpr int Q = 0, K = ROWS / 128 * TILE, V = K + KS * TILE, END = V + VS * TILE;
    static constexpr int SMEM = END + 1024;           // room to align the stages to the swizzle's 1024 bytes
};

// tensor memory columns
constexpr uint32_t COL_S = 0, COL_O = 256, COLS = 512;

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// Bounded wait.  `dead` is set by the first wait of the block that gives up, and ends the others.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *dead, uint32_t *status)
{
    if (bar_try(bar, parity))
        return true;
#pragma unroll 1
    for (uint32_t i = 0; i < KVC_WAIT_LIMIT; ++i) {
        if (bar_try(bar, parity))
            return true;
        if (*dead)
            return false;
    }
    if (!atomicExch(const_cast<uint32_t *>(dead), 1u))
        atomicAdd(status + 1, 1u);
    return false;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Shared-memory operand: 128-byte swizzle, 8-row groups 1024 bytes apart along the rows (or keys), and,
// where the other dimension is the contiguous one, its 64-element blocks `lead` bytes apart.
// The low word is built once for each buffer; a place inside one is 16 bytes a step away, and no sum
// carries, since shared memory ends below the field's 2^18 bytes.
constexpr uint32_t OPERAND_HIGH = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t lead) { return (addr >> 4) | ((lead >> 4) << 16); }

// Instruction descriptor: 32-bit sums, both operands of type T, M = 128, N = n; b_by_column: B's n is contiguous.
template <typename T>
__host__ __device__ constexpr uint32_t kind(uint32_t n, bool b_by_column)
{
    const uint32_t f = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return (1u << 4) | (f << 7) | (f << 10) | ((b_by_column ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

// A value that all lanes hold, known to the compiler as such: matrix instructions take their operands from
// the warp's uniform registers, and moving them there one by one costs more than the instruction.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(~0u, x, 0); }

__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(what), "r"((uint32_t)add), "r"(OPERAND_HIGH) : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 db, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(what), "r"((uint32_t)add), "r"(OPERAND_HIGH) : "memory");
}

// The barrier is arrived at once when all matrix instructions issued so far have completed.
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_ld32(float *x, uint32_t addr)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr) : "memory");
}

// 16 rows x 32 columns: four lanes to a row, x[4 * k + 2 * e + i] is row lane / 4 + 8 * e, column 8 * k + 2 * (lane % 4) + i.
__device__ __forceinline__ void tmem_ld16x256(float *x, uint32_t addr)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(x);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr) : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t addr, const float *x)
{
    const uint32_t *r = reinterpret_cast<const uint32_t *>(x);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
                 "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                   "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void release_tmem(uint32_t tmem)
{
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS));
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A word whose lowest n bits are set (n < 0: none, n > 31: all).
__device__ __forceinline__ uint32_t low_bits(int32_t n) { return n <= 0 ? 0u : n > 31 ? ~0u : (1u << n) - 1u; }

struct Bars {
    // q_full: [row tile].  p_full: [score buffer][half of the keys].  s_full, o_done: scores made, and a row tile's
    // last products of a segment, [0] and [1] of either row tile; with one row tile [0] and [2], scores in either buffer
    // and the products of even and of odd tiles (so that a warp that looks one product late is never two phases
    // behind).  [1] belongs to the second row tile alone: nothing waits for its warps while there is one row tile, and
    // a parity does not tell a warp that comes late how many phases it has missed.
    uint64_t q_full[2], s_full[3], p_full[2][2], o_done[3];
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t seg_full[4], seg_empty[4], drained;
};

// The units of one pair in the block's run, as the scheduling warp hands them to the others: what lies
// between pairs is then in the code once and not in every role.
struct Segment {
    KvcSeq q;
    KvcRange r;
    uint32_t h, rt, t, n;  // KV head, row tile; first tile and number of tiles (0: the run is over)
    uint32_t pair;
    unsigned long long units_at;  // where the pair's units begin on the line
};
constexpr uint32_t SEGMENTS = 4;
constexpr uint32_t SEGMENT_READERS = 19;  // 16 softmax warps, 2 loading warps, the issuing warp

// The next segment, copied to registers.  Every lane of the role's warp calls this.
struct SegmentReader {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ bool next(const Segment *ring, Bars *bars, Segment &out, volatile uint32_t *dead, uint32_t *status)
    {
        if (!__all_sync(~0u, bar_wait(smem_addr(&bars->seg_full[slot]), parity, dead, status)))
            return false;
        out = ring[slot];
        __syncwarp();
        if ((threadIdx.x & 31u) == 0)
            bar_arrive(smem_addr(&bars->seg_empty[slot]));
        if (++slot == SEGMENTS) {
            slot = 0;
            parity ^= 1;
        }
        return out.n != 0;
    }
};

#define BAR(name) ((uint32_t)offsetof(Bars, name))

// A role's count of uses of a ring: stage and parity.
template <int N>
struct Ring {
    uint32_t stage = 0, parity = 0;
    __device__ void next()
    {
        if (++stage == N) {
            stage = 0;
            parity ^= 1;
        }
    }
};

// The launch's parameters: with `boxes` != 0 a tile's keys come in that many boxes of box_keys keys, each
// inside one block of the pool, through a tensor map of the plane.
struct alignas(64) TilesArgs {
    CUtensorMap k_map, v_map;  // [block][token][head][element], boxes of [1][box_keys][1][64]
    KvcAttn a;
    uint32_t boxes, box_keys;
};

__device__ __forceinline__ void box_load(uint32_t dst, const CUtensorMap *map, uint32_t x, uint32_t head, uint32_t tok, uint32_t block,
                                         uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(head), "r"(tok), "r"(block), "r"(bar) : "memory");
}

// One of the two loading warps: all tiles of the block's run, K or V.  A tile comes as boxes, where blocks
// and tiles divide one another; a box's block id is looked up a tile ahead.  What is not a key's may be
// garbage in K, whose scores are replaced; in V it meets a weight of zero, which infinity or NaN would
// survive, so a tile of V that is not all keys is copied key by key, with zeros between.
template <int D, int ROWS, bool KEYS>
__device__ __forceinline__ void load_role(const TilesArgs &args, const Segment *segments, uint32_t tiles, Bars *bars,
                                          uint32_t (*there)[4], volatile uint32_t *dead, uint32_t lane)
{
    using S = Shape<D, ROWS>;
    constexpr int STAGES = KEYS ? S::KS : S::VS;
    constexpr int PER = 512 / (D * 2);  // keys per round of 32 lanes
    constexpr uint32_t NONE = ~0u;
    const KvcAttn &a = args.a;
    const uint32_t full = smem_addr(KEYS ? bars->k_full : bars->v_full), empty = smem_addr(KEYS ? bars->k_empty : bars->v_empty);
    const CUtensorMap *map = KEYS ? &args.k_map : &args.v_map;
    const uint32_t boxes = args.boxes, box_at = (boxes ? lane % boxes : 0u) * args.box_keys;  // this lane's box
    SegmentReader reader;
    Segment c;
    Ring<STAGES> ring;
    uint32_t slot = 0, issued = 0;
    bool ok = true;
#pragma unroll 1
    while (ok && reader.next(segments, bars, c, dead, a.status)) {
        // V may be read past the pair's last key, up to the sequence's: what other rows of the call see is as
        // good as what this pair's do
        const int32_t limit = KEYS || a.phase == KVC_PHASE_PREFIX ? c.r.hi : min(c.q.pos + c.q.rows / (int32_t)a.g, kvc_key_cap(a));
        const int32_t *table = a.tables + (int64_t)c.q.table * a.table_stride;
        const auto look = [&](uint32_t u) {  // the block id of this lane's box of tile u
            const int32_t jb = (int32_t)(kvc_tile(c.r, c.t + u) * TK + box_at);
            return jb < limit && (jb + (int32_t)args.box_keys > c.r.lo || jb < c.r.sink_end) ? (uint32_t)table[kvc_div((uint32_t)jb, a.block_size, a.block_shift)] : NONE;
        };
        uint32_t next_id = boxes ? look(0) : NONE;
#pragma unroll 1
        for (uint32_t u = 0; u < c.n; ++u) {
            const int32_t j0 = (int32_t)(kvc_tile(c.r, c.t + u) * TK);
            const uint32_t id = next_id;
            if (boxes && u + 1 < c.n)
                next_id = look(u + 1);
            const auto key = [&](int32_t j) { return j < c.r.hi && (j >= c.r.lo || j < c.r.sink_end); };
            const uint32_t good = __ballot_sync(~0u, id < a.num_blocks) & ((1u << boxes) - 1u);
            bool boxed = boxes != 0;
            if (boxed && KEYS) {
                const int32_t jb = j0 + (int32_t)box_at;
                if (lane < boxes && id >= a.num_blocks && jb < limit && (jb + (int32_t)args.box_keys > c.r.lo || jb < c.r.sink_end))
                    atomicAdd(a.status, 1u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t at = i * 32 + lane;
                    const uint32_t w = __ballot_sync(~0u, key(j0 + (int32_t)at) && (good >> (at / args.box_keys) & 1u));
                    if (lane == 0)
                        there[slot][i] = w;
                }
            } else if (boxed) {
                boxed = ((j0 >= c.r.lo && j0 + TK <= limit) || j0 + TK <= c.r.sink_end) && good == (1u << boxes) - 1u;
            }
            int64_t off[4];
            if (!boxed) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t j = j0 + i * 32 + (int32_t)lane;
                    off[i] = -1;
                    if (key(j)) {
                        off[i] = kvc_key_offset(a, c.q.table, j, c.h, D * 2);
                        if (KEYS && off[i] < 0)
                            atomicAdd(a.status, 1u);
                    }
                    if (KEYS) {
                        const uint32_t w = __ballot_sync(~0u, off[i] >= 0);
                        if (lane == 0)
                            there[slot][i] = w;
                    }
                }
            }
            slot = (slot + 1) % THERE;
            if (!(ok = __all_sync(~0u, bar_wait(empty + ring.stage * 8u, ring.parity ^ 1u, dead, a.status))))
                break;
            const uint32_t tile = tiles + ring.stage * S::TILE, bar = full + ring.stage * 8u;
            if (boxed) {
                // (the words of `there` are ordered before the barrier's phase by lane 0's arrival)
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                                 "r"((uint32_t)__popc(good) * args.box_keys * (uint32_t)D * 2u) : "memory");
                __syncwarp();
                // a lane a box: the lanes take turns at the copy unit, but their operands are ready (8192-token
                // prompt in 16-token blocks: 7 % more with one lane in a loop of 16 boxes)
                const uint32_t h = boxes * (D / 64) > lane ? lane / boxes : 0u, i = lane - h * boxes;
                if (lane < boxes * (D / 64) && (good >> i & 1u))
                    box_load(tile + h * S::HALF + box_at * 128u, map, h * 64u, c.h, boxes > 1 ? 0u : (uint32_t)j0 % a.block_size, id, bar);
            } else {
                const unsigned char *plane = KEYS ? a.k : a.v;
                const uint32_t chunk = lane % (D / 8), sub = lane / (D / 8);
                const uint32_t base = tile + (chunk >> 3) * S::HALF;
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll 4
                    for (int i = 0; i < 32 / PER; ++i) {
                        const uint32_t row = i * PER + sub;
                        const int64_t o = __shfl_sync(~0u, off[q], row);
                        copy16(base + (q * 32 + row) * 128u + (((chunk & 7u) ^ (row & 7u)) << 4), plane + (o >= 0 ? o : 0) + chunk * 16u,
                               o >= 0 ? 16u : 0u);
                    }
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_async();
                __syncwarp();
                if (lane == 0)
                    bar_arrive(bar);
            }
            ring.next();
            ++issued;
        }
    }
    // no copy of ours runs on when the block ends, on no way out
#pragma unroll 1
    for (uint32_t n = issued < STAGES ? 0u : issued - STAGES; n < issued; ++n)
#pragma unroll 1
        for (uint32_t i = 0; i < KVC_WAIT_LIMIT && !bar_try(full + (n % STAGES) * 8u, n / STAGES & 1u); ++i)
            ;
}

template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(THREADS, 1) kvc_attn_tiles_kernel(const __grid_constant__ TilesArgs args)
{
    using S = Shape<D, ROWS>;
    const KvcAttn &a = args.a;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Bars bars;
    __shared__ __align__(16) uint32_t there[THERE][4];
    __shared__ uint32_t s_dead, s_tmem;
    __shared__ Segment segments[SEGMENTS];
    __shared__ float row_top[2][2][2][128], row_sum[2][2][128];  // ([tile of keys, odd or even])[row tile][half][row]
    // What touches no memory of the caller's comes before the wait for the stream's previous kernel.
    const uint32_t warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31u;
    const uint32_t tiles = (smem_addr(smem_raw) + 1023u) & ~1023u;
    unsigned char *tiles_ptr = smem_raw + (tiles - smem_addr(smem_raw));
    volatile uint32_t *dead = &s_dead;
    if (threadIdx.x == 0) {
        s_dead = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&bars.q_full[i]), 8);
            bar_init(smem_addr(&bars.p_full[i][0]), 128);
            bar_init(smem_addr(&bars.p_full[i][1]), 128);
        }
        for (int i = 0; i < 3; ++i) {
            bar_init(smem_addr(&bars.s_full[i]), 1);
            bar_init(smem_addr(&bars.o_done[i]), 1);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(smem_addr(&bars.k_full[i]), 1);
            bar_init(smem_addr(&bars.k_empty[i]), 1);
            bar_init(smem_addr(&bars.v_full[i]), 1);
            bar_init(smem_addr(&bars.v_empty[i]), 1);
            bar_init(smem_addr(&bars.seg_full[i]), 1);
            bar_init(smem_addr(&bars.seg_empty[i]), SEGMENT_READERS);
        }
        bar_init(smem_addr(&bars.drained), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (args.boxes) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&args.k_map) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&args.v_map) : "memory");
        }
    }
    kvc_pdl_begin(a.beside);
    // Tensor memory is not held while waiting for the kernel before: one that lets this one in early, and allocates
    // on the same SM after that, would wait for this block for ever.
    if (warp == 16)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(COLS) : "memory");
    fence_before();

    const uint32_t n_seq = a.phase == KVC_PHASE_PREFIX ? a.n_groups : a.n_requests;
    const KvcRun run = kvc_find_run<ROWS, TK, HEAD, LEAST, THREADS>(a, n_seq);  // (has block-wide barriers)
    fence_after();
    if (!run.any) {
        if (warp == 16)
            release_tmem(uniform(s_tmem));
        kvc_pdl_end(a.beside);
        return;
    }
    const uint32_t tmem = uniform(s_tmem);

    if (warp < 16) {
        // registers: 512 x 104 + 128 x 64 = 640 x 96 of the launch
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        // ---------------------------------------------------------------- softmax
        const uint32_t sub = warp >> 3, half = warp >> 2 & 1u, tid = threadIdx.x & 127u;  // tid: the row
        const uint32_t lanes = (warp & 3u) << 21;  // this warp's 32 rows of tensor memory
        const uint32_t s_col = tmem + COL_S + lanes, o_col = tmem + COL_O + sub * 128u + half * (D / 2) + lanes;
        const uint32_t bar = smem_addr(&bars);
        // The two warps of the same rows meet here: true where one of them is leaving.  A warp that leaves, at its end
        // or because a wait gave up, meets its partner once more and says so; the partner, wherever it comes to meet,
        // then leaves without another meeting.  So every meeting has two sides, and no warp waits for one that
        // is gone, however far apart the two are when a wait gives up.
        const uint32_t meeting = 1u + sub * 4u + (warp & 3u);
        const auto meet = [&](bool leaving) {
            uint32_t gone;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(gone) : "r"(meeting), "r"((uint32_t)leaving) : "memory");
            return gone != 0;
        };
        bool parted = false;  // the partner has left
        SegmentReader reader;
        Segment c, d;
        uint32_t s_parity = 0, o_parity = 0, slot = 0;  // parities: a bit for each barrier, of those that this warp waits for
        // Queries of a segment: 16 bytes a thread and turn, rows of 128 bytes in the swizzle.  All scores
        // of the segment before have been seen, so their operand may go.
        const auto load_queries = [&](const Segment &c) {
            const uint32_t row0 = c.rt * ROWS + sub * 128u, rows_all = (uint32_t)c.q.rows;
            if (row0 >= rows_all || (ROWS == 128 && sub == 1))
                return;
            constexpr uint32_t STEP = 256u / (D / 8), TURNS = 128u / STEP;
            const uint32_t at = threadIdx.x & 255u, chunk = at % (D / 8), r0 = at / (D / 8);
            uint32_t tok = kvc_div_g(a, row0 + r0), head = row0 + r0 - tok * a.g;
            const uint32_t tok_step = kvc_div_g(a, STEP), head_step = STEP - tok_step * a.g;
            const unsigned char *src = a.q + (int64_t)c.q.qa * a.q_tok + (int64_t)(c.h * a.g) * a.q_head + chunk * 16u;
            unsigned char *dst = tiles_ptr + S::Q + sub * S::TILE + (chunk >> 3) * S::HALF;
            uint4 x[TURNS];
#pragma unroll
            for (uint32_t e = 0; e < TURNS; ++e) {
                x[e] = row0 + r0 + e * STEP < rows_all
                           ? *reinterpret_cast<const uint4 *>(src + (int64_t)tok * a.q_tok + (int64_t)head * a.q_head)
                           : make_uint4(0, 0, 0, 0);
                tok += tok_step;
                head += head_step;
                if (head >= a.g) {
                    head -= a.g;
                    ++tok;
                }
            }
#pragma unroll
            for (uint32_t e = 0; e < TURNS; ++e) {
                const uint32_t r = r0 + e * STEP;
                *reinterpret_cast<uint4 *>(dst + r * 128u + (((chunk & 7u) ^ (r & 7u)) << 4)) = x[e];
            }
            fence_async();
            __syncwarp();
            if (lane == 0)
                bar_arrive(bar + BAR(q_full) + sub * 8u);
        };
        bool ok, open = false;  // open: a segment whose products have been started and whose result is to be written
        uint32_t row0 = 0, last = 0;  // last: the barrier of the open segment's last product
        float m = 0.f, l = 0.f;  // m: the maximum in use, base 2; l: of this thread's keys
        for (;;) {
            // the next segment's queries first, so that its scores run while the one before is written
            ok = reader.next(segments, &bars, d, dead, a.status);
            if (ok)
                load_queries(d);
            if (__any_sync(~0u, *dead)) {
                ok = false;
                break;
            }
            if (open) {
                const bool from_start = c.t == 0, to_end = c.t + c.n == c.r.n, real = row0 + tid < (uint32_t)c.q.rows;
                row_sum[sub][half][tid] = l;
                if ((parted = meet(false)))
                    break;
                l = row_sum[sub][0][tid] + row_sum[sub][1][tid];
                if (!__all_sync(~0u, bar_wait(bar + BAR(o_done) + last * 8u, o_parity >> last & 1u ^ 1u, dead, a.status))) {
                    ok = false;
                    break;
                }
                fence_after();
                // O in the other layout that tensor memory is read in: a lane holds two neighbouring columns of rows
                // lane / 4 and lane / 4 + 8 of 16, so that four lanes write adjacent bytes of one row and a store
                // touches 8 rows and not 32
                const bool whole = a.phase == KVC_PHASE_WHOLE && from_start && to_end;
                const bool room = a.phase == KVC_PHASE_WHOLE || c.pair < a.parts.max_pairs;
                const uint64_t slot_row = (a.phase == KVC_PHASE_WHOLE ? 2ull * blockIdx.x + (from_start ? 1 : 0)
                                                                      : (uint64_t)blockIdx.x + c.pair) * ROWS + sub * 128u;
                const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing: zeros
#pragma unroll 1
                for (uint32_t rows16 = 0; rows16 < 32; rows16 += 16) {
                    unsigned char *dst[2];
                    float f[2];
                    bool write[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t in_warp = rows16 + (lane >> 2) + 8 * e, r = (warp & 3u) * 32u + in_warp;
                        const uint32_t i = row0 + r, tok = kvc_div_g(a, i), head = c.h * a.g + (i - tok * a.g);
                        f[e] = __shfl_sync(~0u, inv, in_warp);
                        write[e] = i < (uint32_t)c.q.rows && room;
                        dst[e] = whole ? a.out + (c.q.qa + (int64_t)tok) * a.o_tok + (int64_t)head * a.o_head + half * D + (lane & 3u) * 4u
                                       : reinterpret_cast<unsigned char *>(a.parts.o + (slot_row + r) * D + half * (D / 2) + (lane & 3u) * 2u);
                    }
#pragma unroll 1
                    for (uint32_t q = 0; q < D / 2; q += 32) {
                        float o[16];
                        tmem_ld16x256(o, o_col + (rows16 << 16) + q);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float x = o[k * 4 + e * 2], y = o[k * 4 + e * 2 + 1];
                                if (!write[e])
                                    continue;
                                if (whole)
                                    *reinterpret_cast<uint32_t *>(dst[e] + (q + k * 8) * 2) =
                                        f[e] == 0.f ? 0u : kvc_from_float2<T>(x * f[e], y * f[e]);
                                else
                                    *reinterpret_cast<float2 *>(dst[e] + (q + k * 8) * 4) = make_float2(x, y);
                            }
                    }
                }
                if (real && half == 0) {
                    if (!whole) {
                        if (room)
                            a.parts.ml[slot_row + tid] = make_float2(m, l);
                        if (a.phase != KVC_PHASE_WHOLE && from_start && sub == 0 && tid == 0 && room)
                            a.parts.range[c.pair] = make_ulonglong2(c.units_at, c.units_at + c.r.n);
                    } else if (a.lse) {
                        const uint32_t i = row0 + tid, tok = kvc_div_g(a, i);
                        a.lse[(c.q.qa + (int64_t)tok) * a.hq + c.h * a.g + (i - tok * a.g)] = (m + log2f(l)) * 0.693147180559945309f;
                    }
                }
            }
            if (!ok)
                break;
            c = d;
            row0 = c.rt * ROWS + sub * 128u;
            open = row0 < (uint32_t)c.q.rows && (ROWS == 256 || sub == 0);
            const bool two = ROWS == 256 && (uint32_t)c.q.rows - c.rt * ROWS > 128u;
            if (open) {
                const int32_t pos = row0 + tid < (uint32_t)c.q.rows ? kvc_row_pos(a, c.q, row0 + tid) : -1;
                const int32_t old = a.window ? pos - a.window : -1;  // the last key behind the row's window
                m = -INFINITY;
                l = 0.f;
#pragma unroll 1
                for (uint32_t i = 0; i < c.n; ++i) {
                    const int32_t j0 = (int32_t)(kvc_tile(c.r, c.t + i) * TK + half * HK);
                    const uint32_t buf = two ? sub : i & 1u, at = two ? sub : buf * 2u, s_at = s_col + buf * 128u;
                    if (!(ok = __all_sync(~0u, bar_wait(bar + BAR(s_full) + at * 8u, s_parity >> at & 1u, dead, a.status))))
                        break;
                    s_parity ^= 1u << at;
                    fence_after();
                    float s[HK];
                    tmem_ld32(s, s_at + half * HK);
                    tmem_ld32(s + 32, s_at + half * HK + 32);
                    uint32_t mask0, mask1;
                    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(mask0), "=r"(mask1) : "r"(smem_addr(&there[(slot + i) % THERE][half * 2])));
                    tmem_wait_ld();
                    if (__any_sync(~0u, (mask0 & mask1) != ~0u || j0 + HK - 1 > pos || (j0 <= old && j0 + HK - 1 >= a.sinks))) {
                        // kvc_sees() for 32 keys at a time: at most pos, and after pos - window or before sinks
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int32_t j = j0 + q * 32;
                            uint32_t see = (q ? mask1 : mask0) & low_bits(pos + 1 - j);
                            if (a.window)
                                see &= ~low_bits(pos - a.window + 1 - j) | low_bits(a.sinks - j);
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                s[q * 32 + k] = see >> k & 1u ? s[q * 32 + k] : -INFINITY;
                        }
                    }
                    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int k = 0; k < HK; k += 8)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            t[e] = fmaxf(t[e], fmaxf(s[k + e], s[k + 4 + e]));
                    float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
                    // the row's other half.  After this both halves of S have been read, so P may go over them.
                    // Odd and even tiles have words of their own: with one row tile the scores of tile i + 1 do not
                    // wait for the weights of tile i, so a warp may be here again before its partner has read.  Those
                    // of tile i + 2 do wait for both halves' weights of tile i, and those are made after the reading
                    row_top[i & 1u][sub][half][tid] = top;
                    if ((parted = meet(false))) {
                        ok = false;
                        break;
                    }
                    top = fmaxf(top, row_top[i & 1u][sub][half ^ 1u][tid]) * a.scale_log2;
                    if (i == 0) {
                        m = top;
                    } else {
                        const bool move = top > m + 8.f || (m == -INFINITY && top != m);
                        if (__any_sync(~0u, move)) {
                            const float f = !move ? 1.f : m == -INFINITY ? 0.f : exp2_fast(m - top);
                            if (move)
                                m = top;
                            l *= f;
                            // the products so far have to be in O.  With two row tiles these scores were issued after
                            // them; with one, only the product before the last is known to be there
                            if (!two) {
                                if (!(ok = __all_sync(~0u, bar_wait(bar + BAR(o_done) + (at ^ 2u) * 8u, o_parity >> (at ^ 2u) & 1u ^ 1u, dead, a.status))))
                                    break;
                                fence_after();
                            }
#pragma unroll 1
                            for (int q = 0; q < D / 2; q += 32) {
                                float o[32];
                                tmem_ld32(o, o_col + q);
                                tmem_wait_ld();
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    o[k] *= f;
                                tmem_st32(o_col + q, o);
                            }
                            // Each half has rescaled its columns of O, and the products of either half's weights add to
                            // all of them: no weights are released before both halves have got here (they take this
                            // branch together, having the same rows, maxima and thus votes)
                            tmem_wait_st();
                            fence_before();
                            if ((parted = meet(false))) {
                                ok = false;
                                break;
                            }
                            fence_after();
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    const uint64_t scale2 = kvc_pair(a.scale_log2, a.scale_log2), base2 = kvc_pair(-base, -base);
                    uint64_t sum2 = 0;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t p[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const float2 x = kvc_unpair(kvc_fma2(kvc_pair(s[q * 32 + 2 * k], s[q * 32 + 2 * k + 1]), scale2, base2));
                            const float y0 = exp2_fast(x.x), y1 = exp2_fast(x.y);
                            sum2 = kvc_add2(sum2, kvc_pair(y0, y1));
                            p[k] = kvc_from_float2<T>(y0, y1);
                        }
                        tmem_st16(s_at + half * (HK / 2) + q * 16, p);
                    }
                    const float2 sum = kvc_unpair(sum2);
                    l += sum.x + sum.y;
                    tmem_wait_st();
                    fence_before();
                    bar_arrive(bar + BAR(p_full) + (buf * 2 + half) * 8u);
                    if (!two)
                        o_parity ^= 1u << at;
                }
                if (!ok)
                    break;
                last = two ? sub : (c.n - 1) % 2u * 2u;
                if (two)
                    o_parity ^= 1u << sub;
            }
            slot = (slot + c.n) % THERE;
        }
        if (!parted)
            meet(true);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 17) {
            load_role<D, ROWS, true>(args, segments, tiles + S::K, &bars, there, dead, lane);
        } else if (warp == 18) {
            load_role<D, ROWS, false>(args, segments, tiles + S::V, &bars, there, dead, lane);
        } else if (warp == 16) {
            // ------------------------------------------------------------ matrix instructions
            // The unit takes few instructions ahead, so what this thread does between them is time that
            // the unit may stand still: addresses and parities live in registers.
            constexpr uint32_t KIND_S = kind<T>(TK, false), KIND_O = kind<T>(D, true);
            const uint32_t q_at = operand(tiles + S::Q, 16), k_at = operand(tiles + S::K, 16), v_at = operand(tiles + S::V, S::HALF);
            const uint32_t bar = smem_addr(&bars);
            SegmentReader reader;
            Segment c;
            Ring<S::KS> k;
            Ring<S::VS> v;
            uint32_t q_parity = 0, p_parity = 0;  // a bit for each row tile
            bool ok = true;
            const auto wait = [&](uint32_t at, uint32_t parity) {
                return ok = __all_sync(~0u, bar_wait(bar + at, parity & 1u, dead, a.status));
            };
            const auto commit = [&](uint32_t at) {
                if (elect_one())
                    mma_commit(bar + at);
            };
            const auto scores = [&](uint32_t sub, uint32_t buf, uint32_t at) {
                const uint32_t qa = q_at + sub * (S::TILE >> 4), ka = k_at + k.stage * (S::TILE >> 4), d = tmem + COL_S + buf * 128u;
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t at = ((i >> 2) * S::HALF + (i & 3) * 32) >> 4;
                        mma_ss(d, qa + at, ka + at, KIND_S, i > 0);
                    }
                    mma_commit(bar + BAR(s_full) + at * 8u);
                }
            };
            // O of row tile `sub` += P V, P from score buffer `buf`, in two halves as they come
            const auto products = [&](uint32_t sub, uint32_t buf, bool first) {
                const uint32_t d = tmem + COL_O + sub * 128u, pa = tmem + COL_S + buf * 128u, va = v_at + v.stage * (S::TILE >> 4);
#pragma unroll
                for (uint32_t half = 0; half < 2; ++half) {
                    if (!ok || !wait(BAR(p_full) + (buf * 2 + half) * 8u, p_parity >> buf))
                        continue;
                    fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t j = half * (HK / 16); j < (half + 1) * (HK / 16); ++j)
                            mma_ts(d, pa + j * 8, va + j * (2048 >> 4), KIND_O, j > 0 || !first);
                    }
                }
                p_parity ^= 1u << buf;
            };
            while (reader.next(segments, &bars, c, dead, a.status)) {
                const bool two = ROWS == 256 && uniform((uint32_t)c.q.rows - c.rt * ROWS > 128u);
                const uint32_t n = uniform(c.n);
                if (!wait(BAR(k_full) + k.stage * 8u, k.parity) || !wait(BAR(q_full), q_parity) ||
                    (two && !wait(BAR(q_full) + 8u, q_parity >> 1)))
                    break;
                q_parity ^= two ? 3u : 1u;
                // scores are made `ahead` tiles ahead of the products that use the same buffer
                const uint32_t ahead = two ? 1u : 2u;
                for (uint32_t i = 0; i < min(ahead, n); ++i) {
                    if (i > 0 && !wait(BAR(k_full) + k.stage * 8u, k.parity))
                        break;
                    scores(0, i, i * 2u);
                    if (two)
                        scores(1, 1, 1);
                    commit(BAR(k_empty) + k.stage * 8u);
                    k.next();
                }
                if (!ok)
                    break;
#pragma unroll 1
                for (uint32_t i = 0; i < n; ++i) {
                    const bool more = i + ahead < n;
                    if (!wait(BAR(v_full) + v.stage * 8u, v.parity))
                        break;
                    if (two) {
#pragma unroll
                        for (uint32_t sub = 0; sub < 2; ++sub) {
                            products(sub, sub, i == 0);
                            if (!ok)
                                break;
                            if (!more)
                                commit(BAR(o_done) + sub * 8u);
                            if (sub == 1)
                                commit(BAR(v_empty) + v.stage * 8u);
                            if (more) {  // these scores' barrier stands for the products before them too
                                if (sub == 0 && !wait(BAR(k_full) + k.stage * 8u, k.parity))
                                    break;
                                scores(sub, sub, sub);
                            }
                        }
                    } else {
                        const uint32_t buf = i & 1u;
                        products(0, buf, i == 0);
                        if (!ok)
                            break;
                        commit(BAR(o_done) + buf * 16u);
                        commit(BAR(v_empty) + v.stage * 8u);
                        if (more && wait(BAR(k_full) + k.stage * 8u, k.parity))
                            scores(0, buf, buf * 2u);
                    }
                    if (!ok)
                        break;
                    v.next();
                    if (more) {
                        commit(BAR(k_empty) + k.stage * 8u);
                        k.next();
                    }
                }
                if (!ok)
                    break;
            }
            // nothing of ours runs on when the block gives tensor memory back, on no way out
            commit(BAR(drained));
#pragma unroll 1
            for (uint32_t i = 0; i < KVC_WAIT_LIMIT && !bar_try(smem_addr(&bars.drained), 0); ++i)
                ;
        }
        if (warp == 19 && lane == 0) {
            // ------------------------------------------------------------ the run, pair by pair
            KvcCursor c = run.at;
            uint32_t slot = 0, parity = 1, pair = run.pair, n;
            unsigned long long units_at = run.units_at;
            do {
                if (!bar_wait(smem_addr(&bars.seg_empty[slot]), parity, dead, a.status))
                    break;
                n = c.s < n_seq ? run.count(c, units_at) : 0u;
                Segment &s = segments[slot];
                s.n = n;
                s.q = c.q;
                s.r = c.r;
                s.h = c.h;
                s.rt = c.rt;
                s.t = c.t;
                s.pair = pair;
                s.units_at = units_at;
                bar_arrive(smem_addr(&bars.seg_full[slot]));
                if (++slot == SEGMENTS) {
                    slot = 0;
                    parity ^= 1;
                }
                // (a run that ends inside the pair ends here: the next count is 0)
                units_at += c.r.n + HEAD;
                ++pair;
                c.t = c.r.n - 1;
                kvc_next<ROWS, TK>(a, n_seq, c);
            } while (n != 0);
        }
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == 16) {
        fence_after();
        release_tmem(tmem);
    }
    kvc_pdl_end(a.beside);
}

// A tensor map of one plane of the pool: [block][token][head][element].
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

bool encode(EncodeTiled fn, CUtensorMap *map, const KvcAttn &a, const unsigned char *plane, uint32_t dtype, uint32_t head_dim,
            uint32_t box_keys)
{
    const cuuint64_t dims[4] = {head_dim, a.hkv, a.block_size, a.num_blocks};
    const cuuint64_t strides[3] = {head_dim * 2ull, a.tok_stride, a.block_stride};
    const cuuint32_t box[4] = {64, 1, box_keys, 1}, steps[4] = {1, 1, 1, 1};
    return fn(map, dtype == KVC_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
              const_cast<unsigned char *>(plane), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int ROWS>
cudaError_t launch(const TilesArgs &args, uint32_t blocks, cudaStream_t st)
{
    const cudaError_t e = cudaFuncSetAttribute(kvc_attn_tiles_kernel<T, D, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               Shape<D, ROWS>::SMEM);
    if (e != cudaSuccess)
        return e;
    return kvc_launch_pdl(kvc_attn_tiles_kernel<T, D, ROWS>, args, dim3(blocks), THREADS, Shape<D, ROWS>::SMEM, st);
}

template <typename T, int D>
cudaError_t launch_rows(const TilesArgs &args, uint32_t blocks, cudaStream_t st)
{
    return args.a.parts.rows == 128 ? launch<T, D, 128>(args, blocks, st) : launch<T, D, 256>(args, blocks, st);
}

}  // namespace

uint32_t kvc_attn_tiles_blocks(const kvc_layout *lay) { return (uint32_t)lay->sm_count; }

cudaError_t kvc_launch_attn_tiles(const KvcAttn &a, uint32_t dtype, uint32_t head_dim, uint32_t blocks, cudaStream_t st)
{
    TilesArgs args;
    memset(&args, 0, sizeof(args));
    args.a = a;
    // Boxes where a tile is made of whole blocks, or a block of whole tiles, eight keys (one period of
    // the swizzle) at least; a map's strides end at 2^40 bytes.  Else the tiles are copied key by key.
    const uint32_t B = a.block_size;
    if (((B >= 8 && B < (uint32_t)TK && TK % B == 0) || B % TK == 0) && a.block_stride < (1ull << 40)) {
        args.box_keys = B < (uint32_t)TK ? B : (uint32_t)TK;
        args.boxes = TK / args.box_keys;
        const EncodeTiled fn = encode_tiled();
        if (!fn)
            return cudaErrorNotSupported;
        if (!encode(fn, &args.k_map, a, a.k, dtype, head_dim, args.box_keys) ||
            !encode(fn, &args.v_map, a, a.v, dtype, head_dim, args.box_keys))
            args.boxes = 0;  // a pool that no map describes
    }
    if (dtype == KVC_DTYPE_BF16)
        return head_dim == 128 ? launch_rows<__nv_bfloat16, 128>(args, blocks, st) : launch_rows<__nv_bfloat16, 64>(args, blocks, st);
    return head_dim == 128 ? launch_rows<__half, 128>(args, blocks, st) : launch_rows<__half, 64>(args, blocks, st);
}
