// dspark_tree_attention: attention of a step's nodes (trees or chains of drafted tokens) over the paged cache.
//
//     out[i] = sum_t w_t v_t,  w = softmax_t(scale q_i . k_t) over the positions before the step, node i and its ancestors.
//
// A row of the products is one node and one of the `group` query heads that share a K/V head: 128 / group nodes make a row tile of
// at most 128 rows, so a cache tile is read once for all of them.  A cache tile is 128 positions (fewer at the end of a page of
// more than 128).  The work is the list of (request, K/V head, pair of row tiles, cache tile), cut into as many equal runs as there
// are SMs: one persistent CTA each, whatever the lengths are.  A unit (request, head, pair of row tiles) that a cut divides leaves
// partial results (running maximum, sum, accumulator) in the workspace, which a second small kernel joins.
//
// Within a CTA:
//   * a producer warp brings K and V tiles into a ring by tensor-map copies, a page a box;
//   * one thread issues tcgen05.mma: S = Q K^T into tensor memory (Q and K in shared memory), then O += P V, with P taken from
//     tensor memory and V as it lies (mn-major);
//   * two groups of four warps do the softmax, one row a thread: they read S, write P over it as 16-bit values, and scale O only
//     when the maximum has risen by more than 2^8 (the reference is any number that keeps the exponentials in range).  The two
//     groups have one S and one O each: with two row tiles they take one of them each; with one they take the even and the odd
//     cache tiles and join at the end.  While one group works on its S the tensor cores do the other's products.
//   * 8-bit caches: four more warps turn the tiles into 16-bit floats (exact for both types) in a second ring.  The scales of K
//     multiply the scores and those of V the weights, so that neither is rounded into the operands.
//
// Bound by the cache's bytes where a K/V head has up to about 128 rows (bf16), by the exponentials and the products beyond.
#include <cuda_bf16.h>
#include <math.h>

#include "kv_cache.cuh"
#include "tcgen05.cuh"

namespace dspark {

constexpr int kAttnMaxDim = 128;
constexpr int kAttnSms = 148;                    // a B200's: the workspace's size is known without the device
constexpr int kAttnTile = 128;                   // rows of a row tile, positions of a cache tile
constexpr int kChunkBytes = kAttnTile * 128;     // 64 columns of 16 bits of a tile: 128 rows of 128 bytes, swizzled
constexpr int kAttnMaxSlots = 12, kAttnMaxRaw = 8, kAttnScaleTiles = 4;
constexpr int kAttnRingBytes = 7 * 2 * kChunkBytes;           // 224 KB: Q and the ring
constexpr int kAttnNarrowBytes = 208 * 1024;                  // with 8-bit caches (4 KB of scales beside it)
constexpr float kAttnLog2e = 1.4426950408889634f;
constexpr float kAttnLazy = 8.f;                 // O is scaled when the maximum rises by more than 2^8
constexpr float kAttnNarrowOffset = 7.f;         // fp16 weights: up to 2^(7 + 8) of 65 504, down to 2^-31 of the largest
constexpr int kSoftmaxWarps = 8;
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
    int q_tiles;                                 // row tiles of a unit: 1 or 2
    int chunks;                                  // of 64 columns: 1 or 2
    int slots, raw_slots;                        // 16-bit tiles of the ring, 8-bit tiles
    int tile_tokens, page_tiles, page_boxes;     // positions of a box; cache tiles of a page (pages above 128) ; boxes of a tile
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
    if (P.c.page_size <= kAttnTile) return (length + kAttnTile - 1) / kAttnTile;
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
        const int tile_nodes = kAttnTile / P.group, nodes = tile_nodes * P.q_tiles;
        u.r = r; u.head = head; u.row_tile = row_tile;
        u.row0 = row0; u.n = n; u.first = first;
        u.node0 = row_tile * nodes;
        u.length = first + min(n, u.node0 + nodes);
        u.tiles = attn_tiles(P, u.length);
        u.pair = P.q_tiles == 2 && n > u.node0 + tile_nodes;
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
    const int nodes = kAttnTile / P.group * P.q_tiles;
    long long sum = 0;
    for (int at = 0; at < n; at += nodes) sum += attn_tiles(P, first + min(n, at + nodes));
    return sum;
}

// ---- PTX -------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 128-byte swizzle, descriptor version 1; groups of 8 rows (k-major) or of 8 k (mn-major) are 1 024 bytes apart.  mn-major:
// the next 64 mn elements are a chunk further.
__device__ __forceinline__ uint64_t attn_desc(uint32_t addr, bool mn_major)
{
    const uint64_t lead = mn_major ? (uint64_t)(kChunkBytes >> 4) : 1ull;
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (lead << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
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
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <bool kHalf>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    uint32_t r;
    if (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// the largest of those of four scales that are finite and asked for
__device__ __forceinline__ float attn_finite_max(float4 x, uint32_t of, float top)
{
    if ((of & 1u) && x.x < INFINITY) top = fmaxf(top, x.x);
    if ((of & 2u) && x.y < INFINITY) top = fmaxf(top, x.y);
    if ((of & 4u) && x.z < INFINITY) top = fmaxf(top, x.z);
    if ((of & 8u) && x.w < INFINITY) top = fmaxf(top, x.w);
    return top;
}
// e with 2^e > x, of a size that keeps the softmax's sum in range
__device__ __forceinline__ float attn_exponent(float x) { return fmaxf((float)((int)(__float_as_uint(x) >> 23) - 126), -60.f); }
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
// ---- the kernel ------------------------------------------------------------------------------------------
struct AttnShared {
    uint64_t full[kAttnMaxSlots], empty[kAttnMaxSlots];       // 16-bit tiles
    uint64_t raw_full[kAttnMaxRaw], raw_empty[kAttnMaxRaw];   // 8-bit tiles
    uint64_t q_full, s_full[2], p_full[2], o_full[2], merge_ready, merge_done, mma_done;
    uint32_t tmem_base;
    int abort, bad_value[kAttnUnitFlags];
    int start_r;
    long long start_left, scan[16], start_at;
    float2 second[kAttnTile];                    // (reference, sum) of the second group
};
template <int kKind>
struct AttnScales { float k[kAttnScaleTiles][kAttnTile], v[kAttnScaleTiles][kAttnTile], q[2][kAttnTile]; };   // q: per row
template <> struct AttnScales<kAttnWide> {};

template <int kKind> constexpr int kAttnThreads = (kSoftmaxWarps + 2 + (kKind == kAttnWide ? 0 : 4)) * 32;

template <int kKind>
__global__ void __launch_bounds__(kAttnThreads<kKind>, 1)
attn_kernel(const __grid_constant__ AttnParams P, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    constexpr bool kNarrow = kKind != kAttnWide;
    constexpr int kThreads = kAttnThreads<kKind>, kProducer = kSoftmaxWarps, kIssuer = kSoftmaxWarps + 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzle atoms: 1 KB
    __shared__ AttnShared S;
    __shared__ __align__(16) AttnScales<kKind> scales;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int d = P.c.head_dim, tile_bytes = P.chunks * kChunkBytes;
    unsigned char* sQ = smem;
    unsigned char* ring = smem + P.q_tiles * tile_bytes;
    unsigned char* raw = ring + P.slots * tile_bytes;

    if (tid == 0) {
        for (int s = 0; s < P.slots; ++s) { mbar_init(&S.full[s], kNarrow ? 4 : 1); mbar_init(&S.empty[s], 1); }
        for (int s = 0; s < P.raw_slots; ++s) { mbar_init(&S.raw_full[s], 1); mbar_init(&S.raw_empty[s], 4); }
        mbar_init(&S.q_full, kSoftmaxWarps);
        for (int t = 0; t < 2; ++t) { mbar_init(&S.s_full[t], 1); mbar_init(&S.p_full[t], 4); mbar_init(&S.o_full[t], 1); }
        for (int i = 0; i < kAttnUnitFlags; ++i) S.bad_value[i] = 0;
        mbar_init(&S.merge_ready, 4); mbar_init(&S.merge_done, 4); mbar_init(&S.mma_done, 1);
        S.abort = 0;
        mbar_fence_init();
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();

    // This CTA's run of the work list: every thread sums the tiles of its requests, a scan places them.
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
    const long long x0 = busy ? total * blockIdx.x / ctas : 0, x1 = busy ? total * (blockIdx.x + 1) / ctas : 0;
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
    const uint32_t tmem = S.tmem_base;
    pdl_trigger();                               // the joining kernel only waits
    volatile int* abort_flag = &S.abort;
    auto give_up = [&]() { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; };

    AttnIter it;
    it.left = x1 - x0;
    int4 cut = make_int4(0, 0, 0, 0);
    if (busy) {
        it.r = S.start_r;
        it.request(P);
        long long at = S.start_at;
        const long long head_tiles = attn_head_tiles(P, it.first, it.n);
        it.head = (int)(at / head_tiles);
        at -= it.head * head_tiles;
        it.row_tile = 0;
        const int nodes = kAttnTile / P.group * P.q_tiles;
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
        if (tid == 0 && at > 0 && total * ((long long)blockIdx.x - 1) / ctas <= unit) {
            const long long end = unit + tiles - 1;
            long long last = end * ctas / total;
            while (total * (last + 1) / ctas <= end) ++last;
            const int node0 = it.row_tile * nodes;
            cut = make_int4(1 + it.head, (int)last, it.row0 + node0, min(it.n - node0, nodes));
        }
    }
    if (tid == 0) P.cuts[blockIdx.x] = cut;
    const int tile_nodes = kAttnTile / P.group;
    AttnUnit u;

    if (warp == kProducer) {
        // ---------------- K and V tiles ---------------------------------------------------------------------
        const int slots = kNarrow ? P.raw_slots : P.slots, row_bytes = kNarrow ? d : 128, copies = kNarrow ? 1 : P.chunks;
        const int slot_bytes = kNarrow ? kAttnTile * d : tile_bytes;
        unsigned char* base = kNarrow ? raw : ring;
        uint64_t* full = kNarrow ? S.raw_full : S.full;
        uint64_t* empty = kNarrow ? S.raw_empty : S.empty;
        const int box = lane / copies, chunk = lane - box * copies;          // a lane brings one box
        int s = 0;
        uint32_t ph = 0;
        bool ok = true, bad_page = false;
        while (ok && !*abort_flag && it.next(P, u)) {
            const int32_t* table = P.c.block_table + u.r * P.c.table_stride;
            for (int j = u.j0; ok && j < u.j1; ++j) {
                int start, len;
                attn_tile_at(P, j, start, len);
                const int boxes = P.page_boxes == 1 ? 1 : (min(kAttnTile, u.length - start) + P.tile_tokens - 1) / P.tile_tokens;
                const int page_of = start / P.c.page_size, y = P.page_boxes == 1 ? start - page_of * P.c.page_size : 0;
                int page = 0;
                if (box < boxes) {
                    page = table[page_of + box];
                    if (page < 0 || page >= P.c.n_pages) { page = P.c.n_pages; bad_page = true; }     // outside the map: zeros
                }
                for (int kv = 0; kv < 2; ++kv) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&empty[s], ph ^ 1u));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(&full[s], (uint32_t)(boxes * copies * P.tile_tokens * row_bytes));
                    __syncwarp();
                    if (box < boxes)
                        tma_load_4d(base + (size_t)s * slot_bytes + chunk * kChunkBytes + box * P.tile_tokens * row_bytes, kv ? &map_v : &map_k,
                                    chunk * 64, y, u.head, page, &full[s]);
                    if (++s == slots) { s = 0; ph ^= 1u; }
                }
            }
        }
        if (bad_page) atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);
        if (!ok && lane == 0) give_up();
        // Leave only after every copy has landed: its slot has been announced as free, or, where somebody gave up, is full.
        for (int i = 0; i < slots; ++i) {
            if (!*abort_flag) mbar_wait_bounded(&empty[s], ph ^ 1u);
            else mbar_wait_bounded(&full[s], ph ^ 1u, 1u << 16);
            if (++s == slots) { s = 0; ph ^= 1u; }
        }
    } else if (warp == kIssuer) {
        // ---------------- products --------------------------------------------------------------------------
        if (lane == 0) {
            const uint32_t type = kNarrow ? 0u : 1u;                        // fp16 or bf16 operands, fp32 sums
            const uint32_t common = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(kAttnTile >> 4) << 24);
            const uint32_t idesc_s = common | ((uint32_t)(kAttnTile >> 3) << 17);
            const uint32_t idesc_o = common | ((uint32_t)(d >> 3) << 17) | (1u << 16);
            const uint32_t q0 = smem_u32(sQ), r0 = smem_u32(ring);
            uint32_t units = 0, items[2] = {0, 0};
            bool ok = true, issued = false;
            // K and V tiles alternate in the ring; the places of the next of each
            int ks = 0, vs = 1;
            uint32_t kph = 0, vph = 0;
            auto advance = [&](int& s, uint32_t& ph) { s += 2; if (s >= P.slots) { s -= P.slots; ph ^= 1u; } };
            while (ok && !*abort_flag && it.next(P, u)) {
                const int n = (u.j1 - u.j0) << (u.pair ? 1 : 0);
                auto scores = [&](int t) {
                    if (!mbar_wait_bounded(&S.full[ks], kph)) return false;
                    tc_fence_after();
                    const uint32_t a = q0 + (u.pair && t ? tile_bytes : 0), b = r0 + ks * tile_bytes;
                    for (int k = 0; k < d / 16; ++k) {
                        const uint32_t at = (uint32_t)((k >> 2) * kChunkBytes + (k & 3) * 32);
                        mma_ss(tmem + t * 128, attn_desc(a + at, false), attn_desc(b + at, false), idesc_s, k > 0);
                    }
                    umma_commit(&S.s_full[t]);
                    if (!u.pair || t) { umma_commit(&S.empty[ks]); advance(ks, kph); }
                    issued = true;
                    return true;
                };
                ok = mbar_wait_bounded(&S.q_full, units & 1u);
                ++units;
                if (!ok) break;
                tc_fence_after();
                ok = scores(0);
                if (ok && n > 1) ok = scores(1);
                for (int i = 0; ok && i < n; ++i) {
                    const int t = i & 1;
                    ok = mbar_wait_bounded(&S.p_full[t], items[t] & 1u) && mbar_wait_bounded(&S.full[vs], vph);
                    ++items[t];
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t b = r0 + vs * tile_bytes;
#pragma unroll
                    for (int k = 0; k < kAttnTile / 16; ++k)
                        mma_ts(tmem + 256 + t * 128, tmem + t * 128 + k * 8, attn_desc(b + k * 2048, true), idesc_o, i > 1 || k > 0);
                    if (!u.pair || t) { umma_commit(&S.empty[vs]); advance(vs, vph); }
                    if (u.pair) { if (i + 2 >= n) umma_commit(&S.o_full[t]); }
                    else if (i + 1 == n) { umma_commit(&S.o_full[0]); umma_commit(&S.o_full[1]); }   // the groups share Q
                    if (i + 2 < n) ok = scores(t);
                }
            }
            if (!ok) give_up();
            if (issued) {
                umma_commit(&S.mma_done);
                mbar_wait_bounded(&S.mma_done, 0u);
            }
        }
        __syncwarp();
    } else if (warp < kSoftmaxWarps) {
        // ---------------- softmax ---------------------------------------------------------------------------
        const int t = warp >> 2, row = tid & 127;                           // group; row of the tile
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_base + t * 128, tO = tmem + lane_base + 256 + t * 128;
        uint32_t units = 0, items = 0, merges = 0;
        uint32_t seq = 0;                        // tiles of the ring used by earlier units
        bool ok = true, merged = false;
        auto wait = [&](uint64_t* bar, uint32_t ph) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, ph));
            return ok;
        };
        auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
        // Row `row` of row tile `tile` of a unit into shared memory; in 8-bit mode as fp16, scaled by a power of two so that no
        // value passes the range and what is lost is below 2^-37 of the row's largest.
        auto load_q = [&](const AttnUnit& w, int tile) {
            const int node = w.node0 + tile * tile_nodes + row / P.group;
            if (row < tile_nodes * P.group && node < w.n) {
                const uint4* src = reinterpret_cast<const uint4*>(P.q + (long long)(w.row0 + node) * P.q_row +
                                                                  (long long)(w.head * P.group + row % P.group) * P.q_head);
                unsigned char* dst = sQ + tile * tile_bytes + row * 128;
                float up = 1.f;
                if constexpr (kNarrow) {
                    float top = 0.f;
#pragma unroll 4
                    for (int c = 0; c < d / 8; ++c) {
                        const uint4 x = src[c];
                        const uint32_t w4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(bf16lo(w4[i])), fabsf(bf16hi(w4[i]))));
                    }
                    // 2^e with the largest value below 2^14: exponent field of top to that of 2^13, within the powers of fp32
                    const int e = min(253, max(1, 254 + 13 - (int)(__float_as_uint(top) >> 23)));
                    up = __uint_as_float((uint32_t)e << 23);
                    scales.q[tile][row] = __uint_as_float((uint32_t)(254 - e) << 23);   // the inverse power
                }
#pragma unroll 4
                for (int c = 0; c < d / 8; ++c) {
                    uint4 x = src[c];
                    if (kNarrow) {
                        x.x = pack16<true>(bf16lo(x.x) * up, bf16hi(x.x) * up);
                        x.y = pack16<true>(bf16lo(x.y) * up, bf16hi(x.y) * up);
                        x.z = pack16<true>(bf16lo(x.z) * up, bf16hi(x.z) * up);
                        x.w = pack16<true>(bf16lo(x.w) * up, bf16hi(x.w) * up);
                    }
                    x.x ^= P.q_sign; x.y ^= P.q_sign; x.z ^= P.q_sign; x.w ^= P.q_sign;
                    *reinterpret_cast<uint4*>(dst + (c >> 3) * kChunkBytes + (((c & 7) ^ (row & 7)) << 4)) = x;
                }
            }
            fence_async_smem();
        };
        bool have = it.next(P, u);
        // Q of the first unit; afterwards each unit's is loaded at the end of the one before
        auto prepare_q = [&](const AttnUnit& w) {
            if (w.pair) load_q(w, t);
            else if (t == 1) load_q(w, 0);
            arrive(&S.q_full);
        };
        if (have) prepare_q(u);
        while (ok && have && !*abort_flag) {
            const int tile = u.pair ? t : 0;
            const int node = u.node0 + tile * tile_nodes + row / P.group;
            const bool live = row < tile_nodes * P.group && node < u.n;
            const bool warp_live = __any_sync(0xffffffffu, live);
            float factor = P.score_factor;       // 8-bit caches: what the row of Q was scaled by (K's scales hold score_factor)
            if (tid == 0) S.bad_value[(units + kAttnUnitFlags / 2) % kAttnUnitFlags] = 0;
            float ref = -INFINITY, sum = 0.f;    // O and the sum are relative to 2^ref
            bool any = false;                    // O holds something
            const int step = u.pair ? 1 : 2;
            const int count = u.j1 - u.j0;
            for (int jj = u.pair ? 0 : t; ok && jj < count; jj += step) {
                int start, len;
                attn_tile_at(P, u.j0 + jj, start, len);
                const int valid = min(len, u.length - start);               // positions of this tile that exist
                const bool masked = start + kAttnTile > u.first || valid < kAttnTile;
                // which positions this row sees, a bit each
                uint32_t seen[4] = {~0u, ~0u, ~0u, ~0u};
                if (masked && warp_live) {
                    const int upto = P.parents ? u.first : u.first + node + 1;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int c = min(min(upto - start, valid) - 32 * w, 32);
                        seen[w] = c <= 0 ? 0u : c == 32 ? ~0u : (1u << c) - 1u;
                    }
                    if (P.parents && live && start + valid > u.first) {
                        int a = node;
                        for (;;) {
                            const int at = u.first + a - start;
                            if (at < 0) break;
                            if (at < valid) {
#pragma unroll
                                for (int w = 0; w < 4; ++w) if ((at >> 5) == w) seen[w] |= 1u << (at & 31);
                            }
                            if (a == 0) break;
                            const int p = P.parents[u.row0 + a];
                            if (p < 0 || p >= a) { atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE); break; }
                            a = p;
                        }
                    }
                }
                if (!wait(&S.s_full[t], items & 1u)) break;
                ++items;
                tc_fence_after();
                const float* fk = nullptr;
                const float* fv = nullptr;
                float v_exp = 0.f;
                if constexpr (kNarrow) {
                    // the scales of this tile have been stored before its K tile was announced
                    const int at = (int)((seq / 2 + jj) % kAttnScaleTiles);
                    fk = scales.k[at];
                    fv = scales.v[at];
                    if (!any) factor = scales.q[tile][row];                 // stored before Q was announced
                    if (!masked) v_exp = attn_exponent(warp_max_f32(attn_finite_max(reinterpret_cast<const float4*>(fv)[lane], ~0u, 0.f)));
                    else {                       // of the positions that this row sees
                        float top = 0.f;
#pragma unroll
                        for (int w = 0; w < 4; ++w)
#pragma unroll
                            for (int i = 0; i < 32; i += 4) top = attn_finite_max(*reinterpret_cast<const float4*>(fv + w * 32 + i), seen[w] >> i, top);
                        v_exp = attn_exponent(top);
                    }
                }
                if (warp_live) {
                    // the largest score, in units of log2
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 4; c += 2) {
                        float a[2][32];
                        tmem_load32_issue(tS + c * 32, a[0]);
                        tmem_load32_issue(tS + c * 32 + 32, a[1]);
                        tmem_load_wait(a[0]);
                        tmem_load_wait(a[1]);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if constexpr (kNarrow) {
#pragma unroll
                                for (int i = 0; i < 32; i += 4) {
                                    const float4 f = *reinterpret_cast<const float4*>(fk + (c + h) * 32 + i);
                                    a[h][i] *= f.x; a[h][i + 1] *= f.y; a[h][i + 2] *= f.z; a[h][i + 3] *= f.w;
                                }
                            }
                            if (masked) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) top = fmaxf(top, (seen[c + h] >> i & 1u) ? a[h][i] : -INFINITY);
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; i += 2) top = fmaxf(top, fmaxf(a[h][i], a[h][i + 1]));
                            }
                        }
                    }
                    top = top * factor + (kNarrow ? v_exp - kAttnNarrowOffset : 0.f);
                    const bool raise = top > ref + kAttnLazy || (ref == -INFINITY && top > -INFINITY);
                    if (__any_sync(0xffffffffu, raise)) {
                        const float f = !raise ? 1.f : ref == -INFINITY ? 0.f : ex2_approx(ref - top);
                        if (raise) { sum *= f; ref = top; }
                        if (any)
                            for (int c = 0; c < d; c += 16) {
                                float o[16];
                                uint32_t w[16];
                                tmem_load16(tO + c, o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * f);
                                tmem_store16(tO + c, w);
                            }
                    }
                    any = true;
                    const float base = ref == -INFINITY ? 0.f : ref;
                    const uint64_t f2 = pack2(factor, factor), b2 = pack2(-base, -base);
                    uint64_t s2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    float a[2][32];
                    tmem_load32_issue(tS, a[0]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float (&x)[32] = a[c & 1];
                        tmem_load_wait(x);
                        if (c < 3) tmem_load32_issue(tS + c * 32 + 32, a[(c + 1) & 1]);
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            uint64_t y = pack2(x[i], x[i + 1]);
                            if constexpr (kNarrow) y = mul2(y, *reinterpret_cast<const uint64_t*>(fk + c * 32 + i));
                            y = fma2(y, f2, b2);
                            float e0, e1;
                            unpack2(y, e0, e1);
                            if (masked) {
                                e0 = (seen[c] >> i & 1u) ? e0 : -INFINITY;
                                e1 = (seen[c] >> (i + 1) & 1u) ? e1 : -INFINITY;
                            }
                            e0 = ex2_approx(e0);
                            e1 = ex2_approx(e1);
                            const uint64_t e = pack2(e0, e1);
                            s2[(i >> 1) & 1] = add2(s2[(i >> 1) & 1], e);
                            if constexpr (kNarrow) {
                                unpack2(mul2(e, *reinterpret_cast<const uint64_t*>(fv + c * 32 + i)), e0, e1);
                                if (masked) {
                                    e0 = (seen[c] >> i & 1u) ? e0 : 0.f;
                                    e1 = (seen[c] >> (i + 1) & 1u) ? e1 : 0.f;
                                }
                            }
                            w[i >> 1] = pack16<kNarrow>(e0, e1);
                        }
                        tmem_store16(tS + c * 16, w);
                    }
                    float s0, s1;
                    unpack2(add2(s2[0], s2[1]), s0, s1);
                    sum += s0 + s1;
                    tmem_store_wait();
                }
                if (!kNarrow && masked && (!u.pair || t == 0)) {
                    // V of positions that no row sees, or that hold NaN or infinities that only some see, must not meet a
                    // weight of zero in the product: zeros here, the latter added to the rows that see them at the end
                    const uint32_t i = seq + 2 * jj + 1, s = i % P.slots;
                    if (!wait(&S.full[s], i / P.slots & 1u)) break;
                    if (start + row >= u.first || row >= valid) {
                        unsigned char* v = ring + (size_t)s * tile_bytes + row * 128;
                        for (int c = 0; c < 8 * P.chunks; ++c) {
                            uint4* p = reinterpret_cast<uint4*>(v + (c >> 3) * kChunkBytes + (((c & 7) ^ (row & 7)) << 4));
                            if (row >= valid) { *p = make_uint4(0, 0, 0, 0); continue; }
                            uint4 x = *p;
                            uint32_t w[4] = {x.x, x.y, x.z, x.w};
                            bool bad = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; bad = true; }
                                if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; bad = true; }
                            }
                            if (bad) {
                                *p = make_uint4(w[0], w[1], w[2], w[3]);
                                S.bad_value[units % kAttnUnitFlags] = 1;
                            }
                        }
                    }
                    fence_async_smem();
                }
                if (merged) {                    // the second group's O of the unit before has been read
                    if (!wait(&S.merge_done, (merges - 1) & 1u)) break;
                    merged = false;
                }
                tc_fence_before();
                arrive(&S.p_full[t]);
            }
            if (!ok || !wait(&S.o_full[t], units & 1u)) break;
            tc_fence_after();
            // Everything of this unit has been multiplied: Q of the next one takes the place of this one's.
            AttnUnit done = u;
            have = it.next(P, u);
            const int done_count = count;
            if (have) prepare_q(u);
            const bool join = !done.pair && done_count > 1;
            if (join && t == 1) {
                if (merged) { if (!wait(&S.merge_done, (merges - 1) & 1u)) break; merged = false; }
                S.second[row] = make_float2(ref, sum);
                tc_fence_before();
                arrive(&S.merge_ready);
                ++merges;
                merged = true;
            } else if (done.pair || t == 0) {
                float ref1 = -INFINITY, f0 = 1.f, f1 = 0.f;
                if (join) {
                    if (!wait(&S.merge_ready, merges & 1u)) break;
                    ++merges;
                    tc_fence_after();
                    const float2 o = S.second[row];
                    ref1 = o.x;
                    const float top = fmaxf(ref, ref1), base = top == -INFINITY ? 0.f : top;
                    f0 = ex2_approx(ref - base);
                    f1 = ex2_approx(ref1 - base);
                    sum = sum * f0 + o.y * f1;
                    ref = top;
                }
                const bool whole = done.j0 == 0 && done.j1 == done.tiles;
                const bool bad_value = kKind != kAttnI8 && *(volatile int*)&S.bad_value[units % kAttnUnitFlags] != 0;
                const long long part = (long long)(2 * blockIdx.x + (done.j0 > 0 ? 0 : 1)) * P.part_rows + tile * kAttnTile + row;
                const int head = done.head * P.group + row % P.group;
                const long long out_row = done.row0 + node;
                const float inverse = 1.f / sum;
                if (warp_live) {
                    for (int c = 0; c < d; c += 16) {
                        float o[16];
                        __syncwarp();
                        tmem_load16(tO + c, o);
                        if (join) {
                            float o1[16];
                            tmem_load16(tO + 128 + c, o1);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = o[i] * f0 + o1[i] * f1;
                        }
                        if (bad_value && live) {
                            int a = node;
                            for (;;) {           // values that were left out of the product, where this row sees them
                                const int position = done.first + a;
                                const int page_of = position / P.c.page_size, token = position - page_of * P.c.page_size;
                                const int j = P.c.page_size <= kAttnTile ? position / kAttnTile : page_of * P.page_tiles + token / kAttnTile;
                                const int page = P.c.block_table[done.r * P.c.table_stride + page_of];
                                if (j >= done.j0 && j < done.j1 && page >= 0 && page < P.c.n_pages) {
                                    const unsigned char* v = P.c.v + page * P.c.page_stride + token * P.c.token_stride + done.head * P.c.head_stride;
#pragma unroll
                                    for (int i = 0; i < 16; ++i) {
                                        if (kNarrow) { if ((v[c + i] & 0x7fu) == 0x7fu) o[i] = NAN; }
                                        else {
                                            const uint32_t x = reinterpret_cast<const uint16_t*>(v)[c + i];
                                            if ((x & 0x7f80u) == 0x7f80u) o[i] += __uint_as_float(x << 16);
                                        }
                                    }
                                }
                                if (a == 0) break;
                                const int p = P.parents ? P.parents[done.row0 + a] : a - 1;
                                if (p < 0 || p >= a) break;
                                a = p;
                            }
                        }
                        if (live && whole) {
                            uint32_t w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = pack16<false>(o[2 * i] * inverse, o[2 * i + 1] * inverse);
                            uint4* dst = reinterpret_cast<uint4*>(P.out + out_row * P.out_row + head * P.out_head + c * 2);
                            dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                            dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        } else if (live) {
                            float4* dst = reinterpret_cast<float4*>(P.parts + part * d + c);
#pragma unroll
                            for (int i = 0; i < 4; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                        }
                    }
                    if (live) {
                        if (!whole) P.part_stats[part] = make_float2(ref, sum);
                        else if (P.out_lse) P.out_lse[out_row * P.q_heads + head] = (ref + log2f(sum)) * 0.6931471805599453f;
                    }
                }
                __syncwarp();
                if (join) { tc_fence_before(); arrive(&S.merge_done); }
            }
            seq += 2 * done_count;
            ++units;
        }
        if (!ok && lane == 0) give_up();
    } else {
        // ---------------- 8-bit tiles to 16 bits --------------------------------------------------------------
        if constexpr (kNarrow) {
            const int ct = tid - (kSoftmaxWarps + 2) * 32;                  // 0 .. 127
            const int pieces = d / 16, inverse = (65536 + pieces - 1) / pieces;   // 16-byte pieces of a position
            int s = 0, rs = 0, tile_no = 0, unit_next = 0;
            uint32_t ph = 0, rph = 0;
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t p) { ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, p)); return ok; };
            // scales of position ct of a tile
            auto load_scales = [&](const AttnUnit& w, int j, float& k, float& v) {
                int start, len;
                attn_tile_at(P, j, start, len);
                k = v = 0.f;
                if (ct >= min(len, w.length - start)) return;
                const int position = start + ct, page_of = position / P.c.page_size, token = position - page_of * P.c.page_size;
                const int page = P.c.block_table[w.r * P.c.table_stride + page_of];
                if (page < 0 || page >= P.c.n_pages) return;
                const long long at = ((long long)page * P.c.kv_heads + w.head) * P.c.page_size + token;
                k = P.c.k_scale[at];
                v = P.c.v_scale[at];
            };
            bool have = it.next(P, u);
            int j = u.j0;
            float ks = 0.f, vs = 0.f;
            if (have) load_scales(u, j, ks, vs);
            while (ok && have && !*abort_flag) {
                int start, len;
                attn_tile_at(P, j, start, len);
                const int valid = min(len, u.length - start);
                const int tree = u.first - start;                           // positions from here on are nodes
                const float k_now = ks * P.score_factor, v_now = vs;
                const int unit_no = unit_next;
                if (++j == u.j1) { have = it.next(P, u); j = u.j0; ++unit_next; }
                if (have) load_scales(u, j, ks, vs);
                for (int kv = 0; kv < 2; ++kv) {
                    if (!wait(&S.raw_full[rs], rph) || !wait(&S.empty[s], ph ^ 1u)) break;
                    if (kv == 0) {
                        // free: the scores of tile_no - 2 are not computed before the weights of tile_no - 4 are there
                        scales.k[tile_no % kAttnScaleTiles][ct] = k_now;
                        scales.v[tile_no % kAttnScaleTiles][ct] = v_now;
                    }
                    const unsigned char* src = raw + (size_t)rs * kAttnTile * d;
                    unsigned char* dst = ring + (size_t)s * tile_bytes;
#pragma unroll 4
                    for (int i = 0; i < pieces; ++i) {
                        const int x = i * 128 + ct, token = x * inverse >> 16, piece = x - token * pieces;
                        const uint4 w = *reinterpret_cast<const uint4*>(src + x * 16);
                        uint2 a = widen4<kKind>(w.x), b = widen4<kKind>(w.y), c = widen4<kKind>(w.z), e = widen4<kKind>(w.w);
                        if (token >= valid) a = b = c = e = make_uint2(0, 0);
                        if (kKind == kAttnE4M3 && kv && token >= tree) {
                            // a NaN among the nodes' values of V: as with 16 bits, zero here and back in the rows that see it
                            uint32_t h[8] = {a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
                            bool bad = false;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                if ((h[k] & 0x7c00u) == 0x7c00u) { h[k] &= 0xffff0000u; bad = true; }
                                if ((h[k] & 0x7c000000u) == 0x7c000000u) { h[k] &= 0xffffu; bad = true; }
                            }
                            if (bad) {
                                a = make_uint2(h[0], h[1]); b = make_uint2(h[2], h[3]); c = make_uint2(h[4], h[5]); e = make_uint2(h[6], h[7]);
                                S.bad_value[unit_no % kAttnUnitFlags] = 1;
                            }
                        }
                        unsigned char* line = dst + (piece >> 2) * kChunkBytes + token * 128;
                        const int at = (piece & 3) * 2, turn = (piece >> 2) & 1;       // the two halves of eight lanes store in turn
                        const uint4 lo = make_uint4(a.x, a.y, b.x, b.y), hi = make_uint4(c.x, c.y, e.x, e.y);
                        *reinterpret_cast<uint4*>(line + (((at + turn) ^ (token & 7)) << 4)) = turn ? hi : lo;
                        *reinterpret_cast<uint4*>(line + (((at + 1 - turn) ^ (token & 7)) << 4)) = turn ? lo : hi;
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&S.raw_empty[rs]); mbar_arrive(&S.full[s]); }
                    if (++rs == P.raw_slots) { rs = 0; rph ^= 1u; }
                    if (++s == P.slots) { s = 0; ph ^= 1u; }
                }
                ++tile_no;
            }
            if (!ok && lane == 0) give_up();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- joining the parts of divided units ------------------------------------------------------------------
// A warp a row: the parts' references and sums first, then the weighted sum of their accumulators, in the order of the CTAs.
constexpr int kJoinThreads = 256;

__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams P, int ctas)
{
    __shared__ int4 s_cut[kAttnSms];
    __shared__ int s_cta[kAttnSms], s_start[kAttnSms + 1], s_cuts;
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid < 32) {
        int n = 0, rows = 0;
        for (int b0 = 0; b0 < ctas; b0 += 32) {
            const int b = b0 + lane;
            int4 cut = make_int4(0, 0, 0, 0);
            if (b < ctas) cut = P.cuts[b];
            const uint32_t some = __ballot_sync(0xffffffffu, cut.x != 0);
            int mine = cut.x ? cut.w * P.group : 0, upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            if (cut.x) {
                const int at = n + __popc(some & ((1u << lane) - 1u));
                s_cut[at] = cut;
                s_cta[at] = b;
                s_start[at] = rows + upto - mine;
            }
            n += __popc(some);
            rows += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) { s_cuts = n; s_start[n] = rows; }
    }
    __syncthreads();
    const int cuts = s_cuts, d = P.c.head_dim, tile_rows = kAttnTile / P.group * P.group;
    const int rows = s_start[cuts];
    int at = 0;
    for (int w = blockIdx.x * (kJoinThreads / 32) + (tid >> 5); w < rows; w += gridDim.x * (kJoinThreads / 32)) {
        while (s_start[at + 1] <= w) ++at;
        const int4 cut = s_cut[at];
        const int b = s_cta[at], i = w - s_start[at], node = i / P.group;
        const int parts = cut.y - b + 2;
        const int row = i < tile_rows ? i : kAttnTile + i - tile_rows;       // its place in a partial result
        auto place = [&](int k) { return (long long)(k == 0 ? 2 * (b - 1) + 1 : 2 * (b - 1 + k)) * P.part_rows + row; };
        float top = -INFINITY;
        for (int k = lane; k < parts; k += 32) top = fmaxf(top, P.part_stats[place(k)].x);
        top = warp_max_f32(top);
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int k0 = 0; k0 < parts; k0 += 32) {
            float2 s = make_float2(-INFINITY, 0.f);
            if (k0 + lane < parts) s = P.part_stats[place(k0 + lane)];
            const float f = ex2_approx(s.x - base);
            sum += s.y * f;
            const int here = min(32, parts - k0);
            for (int k = 0; k < here; k += 4) {
                float4 x[4];
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    if (k + m < here && lane * 4 < d) x[m] = *reinterpret_cast<const float4*>(P.parts + place(k0 + k + m) * d + lane * 4);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float g = __shfl_sync(0xffffffffu, f, (k + m) & 31);
                    if (k + m < here && lane * 4 < d) {
                        o[0] = fmaf(x[m].x, g, o[0]); o[1] = fmaf(x[m].y, g, o[1]);
                        o[2] = fmaf(x[m].z, g, o[2]); o[3] = fmaf(x[m].w, g, o[3]);
                    }
                }
            }
        }
        sum = warp_sum_f32(sum);
        const float inverse = 1.f / sum;
        const int head = (cut.x - 1) * P.group + i % P.group;
        const long long out_row = cut.z + node;
        if (lane * 4 < d)
            *reinterpret_cast<uint2*>(P.out + out_row * P.out_row + head * P.out_head + lane * 8) =
                make_uint2(pack16<false>(o[0] * inverse, o[1] * inverse), pack16<false>(o[2] * inverse, o[3] * inverse));
        if (P.out_lse && lane == 0) P.out_lse[out_row * P.q_heads + head] = (top + log2f(sum)) * 0.6931471805599453f;
    }
}

// ---- host side -------------------------------------------------------------------------------------------
// One K/V array of a layer as [page][head][token][d]; a box is `tokens` positions of one head of a page.
static bool cache_map(CUtensorMap* map, const unsigned char* base, const KvView& c, int tokens)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const bool wide = c.dtype == DSPARK_BF16;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.kv_heads, (cuuint64_t)c.n_pages};
    auto step = [](long long s) { return (cuuint64_t)(s > 16 ? s : 16); };  // of a single entry: any
    const cuuint64_t strides[3] = {step(c.token_stride), step(c.head_stride), step(c.page_stride)};
    const cuuint32_t box[4] = {(cuuint32_t)(wide ? 64 : c.head_dim), (cuuint32_t)tokens, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, wide ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<unsigned char*>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, wide ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static int attn_sms()
{
    static std::atomic<int> sms[64];
    int dev = 0;
    cudaGetDevice(&dev);
    int v = sms[dev & 63].load(std::memory_order_relaxed);
    if (!v) {
        cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
        if (v > kAttnSms) v = kAttnSms;
        sms[dev & 63].store(v, std::memory_order_relaxed);
    }
    return v;
}
struct AttnWs { size_t stats, parts, total; int rows; };
static AttnWs attn_ws(long long n_rows, int group, int d)
{
    AttnWs w;
    const long long rows = n_rows * group;
    w.rows = rows < 2 * kAttnTile ? (rows <= kAttnTile ? (int)rows : 2 * kAttnTile) : 2 * kAttnTile;
    w.stats = ((size_t)kAttnSms * sizeof(int4) + 255) / 256 * 256;
    w.parts = w.stats + ((size_t)2 * kAttnSms * w.rows * sizeof(float2) + 255) / 256 * 256;
    w.total = w.parts + (size_t)2 * kAttnSms * w.rows * d * sizeof(float);
    return w;
}
template <int kKind>
static int attn_launch(AttnParams& P, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    constexpr bool kNarrow = kKind != kAttnWide;
    constexpr int kSmem = (kNarrow ? kAttnNarrowBytes : kAttnRingBytes) + 1024;
    static std::atomic<unsigned long long> ready{0};
    int dev = 0;
    cudaGetDevice(&dev);
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(attn_kernel<kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return launch_status();
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    const int tile = P.chunks * kChunkBytes;
    if (kNarrow) {
        // four 16-bit tiles beside one of Q, three beside two; the rest for 8-bit ones
        P.slots = P.q_tiles == 1 ? 4 : 3;
        P.raw_slots = (kAttnNarrowBytes - (P.q_tiles + P.slots) * tile) / (kAttnTile * P.c.head_dim);
        if (P.raw_slots > kAttnMaxRaw) P.raw_slots = kAttnMaxRaw;
    } else {
        P.slots = kAttnRingBytes / tile - P.q_tiles;
        if (P.slots > kAttnMaxSlots) P.slots = kAttnMaxSlots;
        P.raw_slots = 0;
    }
    KernelTimerScope timer(DSPARK_K_TREE_ATTENTION, s);
    launch_pdl(attn_kernel<kKind>, dim3((unsigned)sms), dim3(kAttnThreads<kKind>), kSmem, s, P, k, v);
    return launch_status();
}

}  // namespace dspark

extern "C" {

size_t dspark_tree_attention_workspace_bytes(int n_rows, int q_heads, int kv_heads, int head_dim)
{
    if (n_rows < 1 || q_heads < 1 || kv_heads < 1 || head_dim < 1 || q_heads % kv_heads != 0) return 0;
    return dspark::attn_ws(n_rows, q_heads / kv_heads, head_dim).total;
}

int dspark_tree_attention(const dspark_kv_cache_t* cache, int layer, const void* q, int64_t q_row_stride, int64_t q_head_stride,
                          int q_heads, const int32_t* first, const int32_t* row_offsets, const int32_t* parents, int R, int n_rows,
                          float scale, void* out, int64_t out_row_stride, int64_t out_head_stride, float* out_lse, int32_t* dev_status,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace dspark;
    if (!q || !out || q_heads < 1 || !isfinite(scale)) return DSPARK_ERR_INVALID_ARG;
    if (int e = kv_cache_check(cache, layer)) return e;
    if (int e = kv_step_check(first, row_offsets, R, n_rows, dev_status)) return e;
    const int d = cache->head_dim;
    if (q_heads % cache->kv_heads != 0) return DSPARK_ERR_INVALID_ARG;
    if (d > kAttnMaxDim || q_heads / cache->kv_heads > 128) return DSPARK_ERR_SHAPE;
    const int64_t strides[4] = {q_row_stride, q_head_stride, out_row_stride, out_head_stride};
    for (int i = 0; i < 4; ++i) {
        if (strides[i] < 0 || (strides[i] < d && ((i & 1) ? q_heads > 1 : n_rows > 1))) return DSPARK_ERR_INVALID_ARG;
        if (strides[i] % 8) return DSPARK_ERR_ALIGNMENT;
    }
    if (((uintptr_t)q | (uintptr_t)out) & 15) return DSPARK_ERR_ALIGNMENT;
    if (((uintptr_t)parents | (uintptr_t)out_lse) & 3) return DSPARK_ERR_ALIGNMENT;
    if (q == out && (q_row_stride != out_row_stride || q_head_stride != out_head_stride)) return DSPARK_ERR_INVALID_ARG;
    AttnParams P = {};
    P.group = q_heads / cache->kv_heads;
    const AttnWs w = attn_ws(n_rows, P.group, d);
    if (!workspace || workspace_bytes < w.total) return DSPARK_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255) return DSPARK_ERR_ALIGNMENT;
    P.c = kv_view(cache, layer);
    P.q = (const unsigned char*)q; P.q_row = q_row_stride * 2; P.q_head = q_head_stride * 2;
    P.out = (unsigned char*)out; P.out_row = out_row_stride * 2; P.out_head = out_head_stride * 2;
    P.out_lse = out_lse;
    P.first = first; P.row_offsets = row_offsets; P.parents = parents;
    P.R = R; P.n_rows = n_rows; P.q_heads = q_heads;
    P.score_factor = fabsf(scale) * kAttnLog2e;
    P.q_sign = scale < 0.f ? 0x80008000u : 0u;
    P.dev_status = dev_status;
    // two row tiles a unit where the requests have more rows than one holds on average: their cache tiles are then read once
    P.q_tiles = (long long)n_rows * P.group > (long long)kAttnTile * R ? 2 : 1;
    P.chunks = d > 64 ? 2 : 1;
    P.tile_tokens = cache->page_size < kAttnTile ? cache->page_size : kAttnTile;
    P.page_boxes = kAttnTile / P.tile_tokens;
    P.page_tiles = (cache->page_size + kAttnTile - 1) / kAttnTile;
    P.part_rows = w.rows;
    unsigned char* ws = (unsigned char*)workspace;
    P.cuts = (int4*)ws;
    P.part_stats = (float2*)(ws + w.stats);
    P.parts = (float*)(ws + w.parts);
    CUtensorMap map_k, map_v;
    if (!cache_map(&map_k, P.c.k, P.c, P.tile_tokens) || !cache_map(&map_v, P.c.v, P.c, P.tile_tokens)) return DSPARK_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int sms = attn_sms();
    int rc;
    if (cache->dtype == DSPARK_BF16) rc = attn_launch<kAttnWide>(P, map_k, map_v, sms, s);
    else if (cache->dtype == DSPARK_I8) rc = attn_launch<kAttnI8>(P, map_k, map_v, sms, s);
    else rc = attn_launch<kAttnE4M3>(P, map_k, map_v, sms, s);
    if (rc) return rc;
    KernelTimerScope timer(DSPARK_K_TREE_COMBINE, s);
    launch_pdl(attn_join_kernel, dim3((unsigned)(2 * sms)), dim3(kJoinThreads), 0, s, P, sms);
    return launch_status();
}

}  // extern "C"
