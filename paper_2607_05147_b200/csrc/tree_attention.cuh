// What the two attention kernels of tree_attention.cu share: the work list, the cache's tiles, PTX.
#pragma once

#include <math.h>

#include "kv_cache.cuh"
#include "tcgen05.cuh"

namespace dspark {

constexpr int kAttnMaxDim = 128;
constexpr int kAttnSms = 148;                    // a B200's: the workspace's size is known without the device
constexpr int kAttnTile = 128;                   // rows of a row tile, positions of a cache tile
constexpr int kChunkBytes = kAttnTile * 128;     // 64 columns of 16 bits of a tile: 128 rows of 128 bytes, swizzled
constexpr int kAttnMaxSlots = 12, kAttnMaxRaw = 12, kAttnScaleTiles = 4;
constexpr int kAttnRingBytes = 6 * 2 * kChunkBytes;           // 192 KB: Q and the rings
// Polls of a wait: 1 s, a poll in vain takes 4 us.  The longest sound one is for walks of kAttnMaxWalk nodes, one after the other for half of
// a unit's 64 rows (few_bad).  The waits of the copies and of the widening warps always have these: with a
// count from memory 128 tokens over int8 took 467 us instead of 440.  The others' can be shortened (AttnParams::polls).
constexpr uint32_t kAttnPolls = 1u << 18;
constexpr int kAttnNarrowBytes = 208 * 1024;                  // with 8-bit caches (4 KB of scales beside it)
constexpr float kAttnLog2e = 1.4426950408889634f;
constexpr float kAttnLazy = 8.f;                 // O is scaled when the maximum rises by more than 2^8
constexpr float kAttnNarrowOffset = 7.f;         // fp16 weights: up to 2^(7 + 8) of 65 504, down to 2^-31 of the largest
constexpr float kAttnUnset = -1e38f;              // a reference that every score is above
constexpr float kAttnLeastFactor = 1.4e-45f;     // the smallest number: -infinity times it is -infinity, a score times it next to nothing
constexpr int kAttnMaxWalk = 65536;              // ancestors of a node outside the chain that its request begins with
constexpr int kAttnNoTree = 0x7fffffff;
// Tiles of a unit that a group adds up in one accumulator.  The tensor cores cut what an fp32 sum cannot hold: positive values came out
// 0.6 % too small after 2^20 positions and 10 % after 2^24.  From time to time the accumulator is therefore added to another, rounded, and
// starts again from zero: 256 tiles of eight products each are off by less than 2^-12.
constexpr int kAttnKeep = 256;
constexpr int kAttnUnitFlags = 8;               // units of one CTA that are under way at a time: at most four

enum AttnKind { kAttnWide = 0, kAttnI8 = 1, kAttnE4M3 = 2 };

struct AttnParams {
    KvView c;
    const unsigned char* q; long long q_row, q_head;          // bytes
    unsigned char* out; long long out_row, out_head;
    float* out_lse;
    const int32_t* first; const int32_t* row_offsets; const int32_t* parents;
    int R, n_rows, q_heads, group;
    float score_factor;                          // |scale| log2(e)
    uint32_t q_sign;                             // sign bits of a pair to flip where scale is negative
    int tile_nodes, unit_nodes;                  // nodes of a row tile, of a unit
    int q_tiles;                                 // row tiles of a unit: 1 or 2
    int chunks;                                  // of 64 columns: 1 or 2
    int k_slots, v_slots;                        // rings: 16-bit tiles of K, of V (behind those of K)
    int raw_k, raw_v;                            // 8-bit tiles, the same way
    int tile_tokens, page_tiles, page_boxes;     // positions of a box; cache tiles of a page (pages above 128) ; boxes of a tile
    uint32_t polls;                              // of a wait of the products' and the softmax's warps, before it gives up
    int page_shift;                              // pages of up to 128: log2 of their size; above: -1
    int part_rows;                               // rows of a partial result
    int32_t* dev_status;
    int4* cuts;                                  // workspace: [kAttnSms] (1 + head, last CTA, first row, nodes); 0: none
    float* parts;                                // [2 kAttnSms][part_rows][d]
    float2* part_stats;                          // [2 kAttnSms][part_rows]
};

// ---- the work list ---------------------------------------------------------------------------------------
// cache tiles that hold positions 0 .. length - 1
__device__ __forceinline__ int attn_tiles(const AttnParams& P, int length)
{
    if (P.c.page_size <= kAttnTile) return (int)(((uint32_t)length + kAttnTile - 1) / kAttnTile);     // (lengths up to 2^31 - 1)
    const int pages = length / P.c.page_size;
    return pages * P.page_tiles + (length - pages * P.c.page_size + kAttnTile - 1) / kAttnTile;
}
// first position of a cache tile and the positions that belong to it
__device__ __forceinline__ void attn_tile_at(const AttnParams& P, int j, int& start, int& len)
{
    if (P.c.page_size <= kAttnTile) { start = j * kAttnTile; len = kAttnTile; return; }
    const int page = j / P.page_tiles, at = (j - page * P.page_tiles) * kAttnTile;
    start = page * P.c.page_size + at;
    len = min(kAttnTile, P.c.page_size - at);
}

// the bit of a cache tile in a set of them that is not exact: there are 32
__device__ __forceinline__ uint32_t attn_tile_bit(int j) { return 1u << (j & 31); }

// page of a request that a position is in
__device__ __forceinline__ int attn_page_of(const AttnParams& P, int position)
{
    return P.page_shift >= 0 ? position >> P.page_shift : position / P.c.page_size;
}

struct AttnUnit {
    int r, head, row_tile;                       // row_tile: of q_tiles tiles
    int row0, n, first;                          // the request
    int node0, length;                           // first node of the unit; positions that any of its nodes may see
    int tiles, j0, j1;                           // cache tiles of the unit; those of this CTA
    bool pair;                                   // the second row tile has nodes
};
// The units of one CTA, in order.
struct AttnIter {
    int r, head, row_tile, j;
    long long left;
    int row0, n, first;                          // of request r
    __device__ __forceinline__ void request(const AttnParams& P)
    {
        for (; r < P.R; ++r) {
            const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, kv_capacity(P.c));
            if (q.n > 0) { row0 = q.row0; n = q.n; first = q.first; return; }
        }
        left = 0;
    }
    __device__ __forceinline__ bool next(const AttnParams& P, AttnUnit& u)
    {
        if (left <= 0) return false;
        const int nodes = P.unit_nodes;
        u.r = r; u.head = head; u.row_tile = row_tile;
        u.row0 = row0; u.n = n; u.first = first;
        u.node0 = row_tile * nodes;
        u.length = first + min(n, u.node0 + nodes);
        u.tiles = attn_tiles(P, u.length);
        u.pair = P.q_tiles == 2 && n > u.node0 + P.tile_nodes;
        u.j0 = j;
        u.j1 = (int)min((long long)u.tiles, j + left);
        left -= u.j1 - u.j0;
        j = 0;
        if (u.node0 + nodes < n) ++row_tile;
        else {
            row_tile = 0;
            if (++head == P.c.kv_heads) { head = 0; ++r; if (left > 0) request(P); }
        }
        return true;
    }
};
// cache tiles of one K/V head of a request
__device__ __forceinline__ long long attn_head_tiles(const AttnParams& P, int first, int n)
{
    long long sum = 0;
    for (int at = 0; at < n; at += P.unit_nodes) sum += attn_tiles(P, first + min(n, at + P.unit_nodes));
    return sum;
}

// This CTA's run of the list, and the unit that it divides first (for the joining kernel).  All threads of the CTA; meets them
// twice, so that what was set up before is seen by all.
struct AttnList { long long scan[32], start_at; int start_r; };
template <int kThreads>
__device__ __forceinline__ AttnIter attn_begin(const AttnParams& P, AttnList& S)
{
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // Every thread sums the tiles of its requests, a scan places them.
    const long long capacity = kv_capacity(P.c);
    const int per = (P.R + kThreads - 1) / kThreads, r_lo = tid * per, r_hi = min(P.R, r_lo + per);
    long long mine = 0;
    int status = 0;
    for (int r = r_lo; r < r_hi; ++r) {
        const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, capacity);
        status |= q.status;
        if (q.n > 0) mine += attn_head_tiles(P, q.first, q.n) * P.c.kv_heads;
    }
    if (status && blockIdx.x == 0) atomicOr(P.dev_status, status);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 31) S.scan[warp] = upto;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    long long total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w == warp) before = total;
        total += S.scan[w];
    }
    before += upto - mine;
    const long long ctas = min((long long)gridDim.x, total);
    const bool busy = (long long)blockIdx.x < ctas;
    // the first `more` CTAs have one tile more than the others
    long long each = 0, more = 0;
    if (busy) {
        if (total >> 32) { each = total / ctas; more = total - each * ctas; }
        else { each = (uint32_t)total / (uint32_t)ctas; more = (uint32_t)total % (uint32_t)ctas; }     // four times as fast
    }
    auto run_start = [&](long long cta) { return each * cta + min(cta, more); };
    const long long x0 = run_start(blockIdx.x), x1 = busy ? run_start(blockIdx.x + 1) : x0;
    if (busy && before <= x0 && x0 < before + mine) {
        long long at = before;
        int r = r_lo;
        for (;; ++r) {
            const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, capacity);
            const long long here = q.n > 0 ? attn_head_tiles(P, q.first, q.n) * P.c.kv_heads : 0;
            if (x0 < at + here) break;
            at += here;
        }
        S.start_r = r;
        S.start_at = x0 - at;
    }
    __syncthreads();
    AttnIter it;
    it.left = x1 - x0;
    int4 cut = make_int4(0, 0, 0, 0);
    if (busy) {
        it.r = S.start_r;
        it.request(P);
        long long at = S.start_at;
        const long long head_tiles = attn_head_tiles(P, it.first, it.n);
        it.head = (at | head_tiles) >> 32 ? (int)(at / head_tiles) : (int)((uint32_t)at / (uint32_t)head_tiles);
        at -= it.head * head_tiles;
        it.row_tile = 0;
        const int nodes = P.unit_nodes;
        int tiles;
        for (;;) {
            tiles = attn_tiles(P, it.first + min(it.n, (it.row_tile + 1) * nodes));
            if (at < tiles) break;
            at -= tiles;
            ++it.row_tile;
        }
        it.j = (int)at;
        // A unit that this CTA's start divides first: CTA blockIdx.x - 1 has its beginning, the others up to `last` go on with it
        // from their starts.
        const long long unit = x0 - at;
        if (tid == 0 && at > 0 && run_start((long long)blockIdx.x - 1) <= unit) {
            int last = blockIdx.x;
            while (run_start(last + 1) < unit + tiles) ++last;
            const int node0 = it.row_tile * nodes;
            cut = make_int4(1 + it.head, last, it.row0 + node0, min(it.n - node0, nodes));
        }
    }
    if (tid == 0) P.cuts[blockIdx.x] = cut;
    return it;
}

// ---- trees -----------------------------------------------------------------------------------------------
// Nodes 0 .. straight - 1 of a request are a chain, whatever comes behind: what a node in it sees is a range, and a walk to the root
// ends where it meets it.  A prompt given with parents is one such chain; walked node by node for each of its tiles 8192 tokens took
// 101 ms instead of 1.3.  Looked for only where a request has more nodes than a tile.  Not inline, like the walks of few rows: with this
// code among the softmax warps' the SM's roles no longer fit its instruction caches (128 tokens over int8: 732 us instead of 443).
constexpr int kAttnStraightLoads = 16;
static __device__ __noinline__ int attn_straight(const int32_t* parents, int n)     // a whole warp
{
    const int lane = threadIdx.x & 31;
    for (int i0 = 1; i0 < n; i0 += kAttnStraightLoads * 32) {
        int p[kAttnStraightLoads];
#pragma unroll
        for (int k = 0; k < kAttnStraightLoads; ++k) {
            const int i = i0 + k * 32 + lane;
            p[k] = i < n ? parents[i] : i - 1;
        }
#pragma unroll
        for (int k = 0; k < kAttnStraightLoads; ++k) {
            const uint32_t off = __ballot_sync(0xffffffffu, p[k] != i0 + k * 32 + lane - 1);
            if (off) return i0 + k * 32 + __ffs(off) - 1;
        }
    }
    return n;
}
// What a warp of the softmax has found of the request it is at; kAttnNoTree where no parents are given.
struct AttnStraight { int of, length; };
__device__ __forceinline__ void attn_look_at_tree(const AttnParams& P, const AttnUnit& u, volatile AttnStraight& S)
{
    if (!P.parents || u.n <= kAttnTile || S.of == u.r) return;
    const int length = attn_straight(P.parents + u.row0, u.n);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) { S.length = length; S.of = u.r; }
    __syncwarp();
}
__device__ __forceinline__ int attn_straight_of(const AttnParams& P, const AttnUnit& u, const volatile AttnStraight& S)
{
    return !P.parents ? kAttnNoTree : u.n <= kAttnTile ? 0 : S.length;
}
// A walk's next node: the parent of a > 0, -1 where there is none (reported)
__device__ __forceinline__ int attn_parent(const AttnParams& P, int row0, int a, int& steps)
{
    const int p = P.parents[row0 + a];
    if (p >= 0 && p < a && ++steps <= kAttnMaxWalk) return p;
    atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE);
    return -1;
}

// ---- PTX -------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Operands in shared memory: 128-byte swizzle, descriptor version 1; groups of 8 rows (k-major) or of 8 k (mn-major) are 1 024
// bytes apart; mn-major: the next 64 mn elements are a chunk further.  The upper half of such a descriptor is a constant, a step
// along k an addition to the lower one: 16 products were issued in 1 700 clocks where each built its descriptors from scratch.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_k_major(uint32_t addr) { return (addr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_mn_major(uint32_t addr) { return (addr >> 4) | ((uint32_t)(kChunkBytes >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh) : "memory");
}
// one lane of a whole warp
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, float (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
                   "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
template <int kCols>
__device__ __forceinline__ void attn_read(uint32_t addr, float (&v)[kCols])
{
    if constexpr (kCols == 8)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(addr) : "memory");
    else if constexpr (kCols == 16) tmem_load16(addr, v);
    else { tmem_load32_issue(addr, v); tmem_load_wait(v); }
}
// Asked for; the values are there after attn_wait(), which waits for all that this thread has asked for.
template <int kCols>
__device__ __forceinline__ void attn_issue(uint32_t addr, float (&v)[kCols])
{
    if constexpr (kCols == 16)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                       "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                     : "r"(addr) : "memory");
    else tmem_load32_issue(addr, v);
}
template <int kCols>
__device__ __forceinline__ void attn_wait(float (&v)[kCols])
{
    if constexpr (kCols == 16)
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                       "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
                     :: "memory");
    else tmem_load_wait(v);
}
template <int kCols>
__device__ __forceinline__ void attn_write(uint32_t addr, const uint32_t (&v)[kCols])
{
    if constexpr (kCols == 8)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    else if constexpr (kCols == 16) tmem_store16(addr, v);
    else
        asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
                     "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                     ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
                       "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
                       "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
                       "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <bool kHalf>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    uint32_t r;
    if (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// 32 columns of scores: -infinity where `on` has no bit, times the column's entry of `by` where `odd` (of those in `on`) has one
template <bool kOdd>
__device__ __forceinline__ void attn_hide(uint32_t addr, uint32_t on, uint32_t odd, const float* by)
{
#pragma unroll 1
    for (int c = 0; c < 32; c += 16, on >>= 16, odd >>= 16) {
        if (__all_sync(0xffffffffu, (on & 0xffffu) == 0xffffu && (!kOdd || (odd & 0xffffu) == 0u))) continue;
        float s[16];
        uint32_t x[16];
        tmem_load16(addr + c, s);
        if (kOdd && __any_sync(0xffffffffu, (odd & 0xffffu) != 0u))
#pragma unroll
            for (int i = 0; i < 16; ++i) if (odd & (1u << i)) s[i] *= by[c + i];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = on & (1u << i) ? __float_as_uint(s[i]) : 0xff800000u;
        tmem_store16(addr + c, x);
    }
    tmem_store_wait();
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// whether one of the kThreads threads that meet at barrier `id` says so
template <int kThreads>
__device__ __forceinline__ bool barrier_any(int id, bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "r"(id), "n"(kThreads) : "memory");
    return r != 0;
}
// the largest magnitude of four scales that is finite
__device__ __forceinline__ float attn_finite_max(float4 x)
{
    const float a = fabsf(x.x), b = fabsf(x.y), c = fabsf(x.z), d = fabsf(x.w);
    return max3(fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f), c < INFINITY ? c : 0.f, d < INFINITY ? d : 0.f);
}
// e with 2^e > x; not below -80, so that the softmax's sum stays in range: a weight before its product with V's scale is at most
// 2^(kAttnNarrowOffset + kAttnLazy + 80) of the reference, 2^31 positions' sum 2^126.  (Scales below 2^-80 shrink the fp16 weights.)
__device__ __forceinline__ float attn_exponent(float x) { return fmaxf((float)((int)(__float_as_uint(x) >> 23) - 126), -80.f); }
// four 8-bit values as fp16, exactly
template <int kKind>
__device__ __forceinline__ uint2 widen4(uint32_t w)
{
    uint2 r;
    if (kKind == kAttnI8) {
        // 0x6400 + b is 1024 + b: with b = value + 128, 1152 is taken off
        const uint32_t x = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r.x) : "r"(a), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r.y) : "r"(b), "r"(0x64806480u));
    } else {
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r.x) : "h"((uint16_t)w));
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r.y) : "h"((uint16_t)(w >> 16)));
    }
    return r;
}

// ---- roles that both kernels have ------------------------------------------------------------------------
// A place in a ring and the parity of its round.  K and V have a ring each: a warp that waits for the tiles of one of them only
// must meet every round of a slot, or a slot that is two rounds on looks like one that is not there yet.
struct RingPlace {
    int s = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void next(int slots) { if (++s == slots) { s = 0; ph ^= 1u; } }
};

// The producer warp: K and V tiles into their rings, K before V, a lane a box.
template <bool kNarrow>
__device__ __forceinline__ void attn_produce(const AttnParams& P, AttnIter it, const CUtensorMap& map_k, const CUtensorMap& map_v, unsigned char* ring,
                                             uint64_t* full, uint64_t* empty, volatile int* abort_flag)
{
    const int lane = threadIdx.x & 31, d = P.c.head_dim;
    const int row_bytes = kNarrow ? d : 128, copies = kNarrow ? 1 : P.chunks, slot_bytes = kNarrow ? kAttnTile * d : P.chunks * kChunkBytes;
    const int box = lane / copies, chunk = lane - box * copies;
    const int k_slots = kNarrow ? P.raw_k : P.k_slots, v_slots = kNarrow ? P.raw_v : P.v_slots;
    RingPlace at[2];
    bool ok = true, bad_page = false;
    AttnUnit u;
    // (a vote: lanes that read the flag at different times must not part, the waits below are the whole warp's)
    while (ok && !__any_sync(0xffffffffu, *abort_flag) && it.next(P, u)) {
        const int32_t* table = P.c.block_table + u.r * P.c.table_stride;
        for (int j = u.j0; ok && j < u.j1; ++j) {
            int start, len;
            attn_tile_at(P, j, start, len);
            const int boxes = P.page_boxes == 1 ? 1 : (min(kAttnTile, u.length - start) + P.tile_tokens - 1) / P.tile_tokens;
            const int page_of = attn_page_of(P, start), y = P.page_boxes == 1 ? start - page_of * P.c.page_size : 0;
            int page = 0;
            if (box < boxes) {
                page = table[page_of + box];
                if (page < 0 || page >= P.c.n_pages) { page = P.c.n_pages; bad_page = true; }     // outside the map: zeros
            }
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                RingPlace& place = at[kv];
                const int s = place.s + (kv ? k_slots : 0);
                ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&empty[s], place.ph ^ 1u, kAttnPolls));
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(&full[s], (uint32_t)(boxes * copies * P.tile_tokens * row_bytes));
                __syncwarp();
                if (box < boxes)
                    tma_load_4d(ring + (size_t)s * slot_bytes + chunk * kChunkBytes + box * P.tile_tokens * row_bytes, kv ? &map_v : &map_k,
                                chunk * 64, y, u.head, page, &full[s]);
                place.next(kv ? v_slots : k_slots);
            }
        }
    }
    if (bad_page) atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);
    if (!ok && lane == 0) { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; }
    // Leave only after every copy has landed: its slot has been announced as free, or, where somebody gave up, is full.
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
        for (int i = 0; i < (kv ? v_slots : k_slots); ++i) {
            const int s = at[kv].s + (kv ? k_slots : 0);
            if (*abort_flag || !mbar_wait_bounded(&empty[s], at[kv].ph ^ 1u, kAttnPolls)) mbar_wait_bounded(&full[s], at[kv].ph ^ 1u, kAttnPolls);
            at[kv].next(kv ? v_slots : k_slots);
        }
}

// Where 16 bytes x of an 8-bit tile of 64 or 128 components come from and go to (and the next 16 beside).  Eight lanes store to eight
// different places of a line of 128 bytes: the pieces of two neighbouring positions, which the swizzle parts by an odd number of
// places; with 128 components one position's lie in the other chunk, so that the loads' banks differ too.
__device__ __forceinline__ void widen_place(int x, int d, int& from, int& to)
{
    int token = x >> 2, piece = x & 3;
    if (d == 128) {
        const int odd = x >> 2 & 1;
        token = (x >> 4) * 2 + odd;
        piece = ((x >> 3 & 1) ^ odd) * 4 + (x & 3);
    }
    from = token * d + piece * 16;
    to = (piece >> 2) * kChunkBytes + token * 128 + ((((piece & 3) * 2) ^ (token & 7)) << 4);
}
template <int kKind>
__device__ __forceinline__ void widen16(uint4 w, unsigned char* dst, int to)
{
    const uint2 a = widen4<kKind>(w.x), b = widen4<kKind>(w.y), c = widen4<kKind>(w.z), e = widen4<kKind>(w.w);
    *reinterpret_cast<uint4*>(dst + to) = make_uint4(a.x, a.y, b.x, b.y);
    *reinterpret_cast<uint4*>(dst + (to ^ 16)) = make_uint4(c.x, c.y, e.x, e.y);
}
// A tile of 64 or 128 components (kDim) by kThreads threads, a thread's pieces a fixed number of positions apart.
template <int kKind, int kThreads, int kDim>
__device__ __forceinline__ void widen_tile(const unsigned char* src, unsigned char* dst, int from0, int to0)
{
    constexpr int kPieces = kAttnTile * kDim / 16 / kThreads, kApart = kThreads * 16 / kDim, kBatch = kPieces < 4 ? kPieces : 4;
#pragma unroll
    for (int i0 = 0; i0 < kPieces; i0 += kBatch) {
        uint4 w[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) w[i] = *reinterpret_cast<const uint4*>(src + from0 + (i0 + i) * kApart * kDim);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) widen16<kKind>(w[i], dst, to0 + (i0 + i) * kApart * 128);
    }
}
// A position of a tile of any width, or of a tile's end: zeros where it does not exist; `look`: NaN becomes zero (true: there was some).
template <int kKind>
__device__ __forceinline__ bool widen_position(const unsigned char* src, unsigned char* dst, int token, int d, bool exists, bool look)
{
    bool any = false;
#pragma unroll 2
    for (int piece = 0; piece < d / 16; ++piece) {
        uint4 x = *reinterpret_cast<const uint4*>(src + token * d + piece * 16);
        if (!exists) x = make_uint4(0, 0, 0, 0);
        if (kKind == kAttnE4M3 && look) {
            uint32_t* w[4] = {&x.x, &x.y, &x.z, &x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // bytes of 0x7f or 0xff: the only ones that carry into their highest bit
                const uint32_t bad = ((*w[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                if (bad) { *w[i] &= ~(bad | (bad - (bad >> 7))); any = true; }
            }
        }
        widen16<kKind>(x, dst, (piece >> 2) * kChunkBytes + token * 128 + ((((piece & 3) * 2) ^ (token & 7)) << 4));
    }
    return any;
}
// A position's components (line: its place in an 8-bit tile) as fp16 into this thread's lane of tensor memory, two a column.  The copy
// engine's swizzle has parted the lines of 64 and 128 bytes, so that eight lanes read different banks.  Of 64 or 128 components
// (kDim) all are asked for first.
template <int kKind, int kDim>
__device__ __forceinline__ void widen_line(const unsigned char* line, int token, int d, uint32_t addr)
{
    constexpr int kBatch = kDim ? 4 : 1, kAll = kDim ? kDim / 16 : 1;
    const int turn = kDim == 128 ? token & 7 : kDim == 64 ? token >> 1 & 3 : 0;
    uint4 w[kAll];
#pragma unroll
    for (int p = 0; p < kAll && kDim; ++p) w[p] = *reinterpret_cast<const uint4*>(line + ((p ^ turn) << 4));
#pragma unroll
    for (int p0 = 0; p0 < (kDim ? kAll : d / 16); p0 += kBatch) {
        uint32_t x[kBatch * 8];
        if (!kDim) w[0] = *reinterpret_cast<const uint4*>(line + (p0 << 4));
#pragma unroll
        for (int p = 0; p < kBatch; ++p) {
            const uint4 v = w[kDim ? p0 + p : 0];
            const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint2 z = widen4<kKind>(y[i]);
                x[p * 8 + 2 * i] = z.x;
                x[p * 8 + 2 * i + 1] = z.y;
            }
        }
        attn_write<kBatch * 8>(addr + p0 * 8, x);
    }
    tmem_store_wait();
    tc_fence_before();
}
// The widths and places that are not those of most calls, out of line: what the SM's roles run at a time then fits its instruction caches
// (128 tokens over int8 445 us, inline 529; 96 components 522 and 596, over e4m3 527 and 586; over e4m3 widen_position is inline: 527 us,
// out of line 650).
template <int kKind>
__device__ __noinline__ void widen_line_any(const unsigned char* line, int token, int d, uint32_t addr) { widen_line<kKind, 0>(line, token, d, addr); }
template <int kKind>
__device__ __noinline__ void widen_line_64(const unsigned char* line, int token, int d, uint32_t addr) { widen_line<kKind, 64>(line, token, d, addr); }
template <int kKind, int kThreads>
__device__ __noinline__ void widen_tile_64(const unsigned char* src, unsigned char* dst, int from0, int to0) { widen_tile<kKind, kThreads, 64>(src, dst, from0, to0); }
static __device__ __noinline__ void widen_position_i8(const unsigned char* src, unsigned char* dst, int token, int d, bool exists)
{
    widen_position<kAttnI8>(src, dst, token, d, exists, false);
}
// kThreads threads: 8-bit tiles as fp16 tiles, as the products read them; K and V (kv 0 and 1), or one of them.  kTensorK: K goes to
// tensor memory at `k_columns`, 64 columns a tile.  tile(unit, j) is called before the waits for a tile's K, ready(number) between
// them and the work.  False: a wait ran out.
template <int kKind, int kThreads, bool kTensorK, typename Tile, typename Ready>
__device__ __forceinline__ bool attn_widen(const AttnParams& P, AttnIter it, int ct, int kv_first, int kv_last, const unsigned char* raw,
                                           unsigned char* ring, int tile_bytes, uint64_t* raw_full, uint64_t* raw_empty, uint64_t* full,
                                           uint64_t* empty, uint32_t k_columns, uint32_t* bad_value, volatile int* abort_flag, Tile tile,
                                           Ready ready)
{
    const int lane = threadIdx.x & 31, d = P.c.head_dim;
    static_assert(kThreads == kAttnTile, "a position a thread");
    int number = 0, unit = 0, from0, to0;
    widen_place(ct, d, from0, to0);
    RingPlace at[2], from_raw[2];
    AttnUnit u;
    while (!__any_sync(0xffffffffu, *abort_flag) && it.next(P, u)) {
        for (int j = u.j0; j < u.j1; ++j, ++number) {
            int start, len;
            attn_tile_at(P, j, start, len);
            const int valid = min(len, u.length - start), tree = u.first - start;   // positions from `tree` on are nodes
            tile(u, j);
            for (int kv = kv_first; kv <= kv_last; ++kv) {
                const int s = kv ? P.k_slots + at[1].s : at[0].s, rs = kv ? P.raw_k + from_raw[1].s : from_raw[0].s;
                const uint32_t ph = kv ? at[1].ph : at[0].ph, rph = kv ? from_raw[1].ph : from_raw[0].ph;
                if (!__all_sync(0xffffffffu, mbar_wait_bounded(&empty[s], ph ^ 1u, kAttnPolls) && mbar_wait_bounded(&raw_full[rs], rph, kAttnPolls))) return false;
                if (kv == 0) ready(number);
                const unsigned char* src = raw + (size_t)rs * kAttnTile * d;
                unsigned char* dst = ring + (size_t)s * tile_bytes;
                if (kTensorK && kv == 0) {               // scores of positions that do not exist are hidden: whatever stands there
                    tc_fence_after();
                    const int token = (threadIdx.x >> 5 & 3) * 32 + lane;   // the lanes of tensor memory that this warp may write
                    const uint32_t to = k_columns + ((uint32_t)(token & ~31) << 16) + at[0].s * 64;
                    if (d == 128) widen_line<kKind, 128>(src + token * d, token, d, to);
                    else if (d == 64) widen_line_64<kKind>(src + token * d, token, d, to);
                    else widen_line_any<kKind>(src + token * d, token, d, to);
                } else {
                    // positions that do not exist: zeros; a NaN among the nodes' values of V: zero here and back in the rows that see
                    // it (attn_bad_values)
                    const bool look = kKind == kAttnE4M3 && kv && tree < kAttnTile;
                    if (d == 128 && valid == kAttnTile && !look) widen_tile<kKind, kThreads, 128>(src, dst, from0, to0);
                    else if (d == 64 && valid == kAttnTile && !look) widen_tile_64<kKind, kThreads>(src, dst, from0, to0);
                    else if constexpr (kKind == kAttnI8) widen_position_i8(src, dst, ct, d, ct < valid);
                    else if (widen_position<kKind>(src, dst, ct, d, ct < valid, look && ct >= tree)) atomicOr(&bad_value[unit % kAttnUnitFlags], attn_tile_bit(j));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&raw_empty[rs]); mbar_arrive(&full[s]); }
                if (kv) { at[1].next(P.v_slots); from_raw[1].next(P.raw_v); }
                else { at[0].next(P.k_slots); from_raw[0].next(P.raw_k); }
            }
        }
        ++unit;
    }
    return true;
}

// One position's line of a bf16 V tile: zeros where it does not exist; NaN and infinities become zeros (true: there were some).
__device__ __forceinline__ bool attn_clean_values(unsigned char* line, int row, int chunks, bool exists)
{
    bool any = false;
    for (int c = 0; c < 8 * chunks; ++c) {
        uint4* p = reinterpret_cast<uint4*>(line + (c >> 3) * kChunkBytes + (((c & 7) ^ (row & 7)) << 4));
        if (!exists) { *p = make_uint4(0, 0, 0, 0); continue; }
        const uint4 x = *p;
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        bool bad = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; bad = true; }
            if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; bad = true; }
        }
        if (bad) { *p = make_uint4(w[0], w[1], w[2], w[3]); any = true; }
    }
    return any;
}
// What was left out of the product for a node's row: the sums of kCount components of V from i on over the nodes that it sees in this
// CTA's part of the unit, where those are NaN or infinities.  tiles: those that hold some.  Seldom done; inline with few rows and a call
// with many, which is what each kernel's other code is fastest with (64 trees of 16: 211 us, with a call 215; 105 trees of 55 nodes over
// e4m3: 278 us with a call, else 311).
struct AttnPart {
    int r, head, row0, first, j0, j1;
    explicit __device__ __forceinline__ AttnPart(const AttnUnit& u) : r(u.r), head(u.head), row0(u.row0), first(u.first), j0(u.j0), j1(u.j1) {}
};
template <bool kNarrow, int kCount>
__device__ __forceinline__ void attn_bad_values(const AttnParams& P, AttnPart u, int node, int straight, uint32_t tiles, int i, float* sum)
{
    for (int c = 0; c < kCount; ++c) sum[c] = 0.f;
    auto tile_of = [&](int position) {
        if (P.c.page_size <= kAttnTile) return position / kAttnTile;
        const int page_of = position / P.c.page_size;
        return page_of * P.page_tiles + (position - page_of * P.c.page_size) / kAttnTile;
    };
    auto add = [&](int position) {
        const int page_of = attn_page_of(P, position), token = position - page_of * P.c.page_size;
        const int page = P.c.block_table[u.r * P.c.table_stride + page_of];
        if (page < 0 || page >= P.c.n_pages) return;
        const unsigned char* v = P.c.v + page * P.c.page_stride + token * P.c.token_stride + u.head * P.c.head_stride;
#pragma unroll
        for (int c = 0; c < kCount; ++c) {
            if (kNarrow) { if ((v[i + c] & 0x7fu) == 0x7fu) sum[c] = NAN; }
            else {
                const uint32_t x = reinterpret_cast<const uint16_t*>(v)[i + c];
                if ((x & 0x7f80u) == 0x7f80u) sum[c] += __uint_as_float(x << 16);
            }
        }
    };
    int a = node, steps = 0;
    while (a >= straight) {
        const int j = tile_of(u.first + a);
        if (j < u.j0) return;
        if (j < u.j1 && (tiles & attn_tile_bit(j))) add(u.first + a);
        if (a == 0) return;
        a = attn_parent(P, u.row0, a, steps);
    }
    if (a < 0) return;
    const int j_first = max(u.j0, tile_of(u.first)), j_last = min(u.j1 - 1, tile_of(u.first + a));
    for (int j = j_first; j <= j_last; ++j) {
        if (!(tiles & attn_tile_bit(j))) continue;
        int start, len;
        attn_tile_at(P, j, start, len);
        const int from = max(start, u.first) - start, to = min(len, u.first - start + a + 1);
#pragma unroll 4
        for (int k = from; k < to; ++k) add(start + k);
    }
}

// the dynamic shared memory of a kernel, once per device
template <typename Kernel>
inline bool attn_allow_smem(Kernel kernel, int bytes, std::atomic<unsigned long long>& ready)
{
    int dev = 0;
    cudaGetDevice(&dev);
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    return true;
}
int attn_few_launch(AttnParams& P, int rows, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s);   // tree_attention_few.cu

}  // namespace dspark
