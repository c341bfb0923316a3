// dspark_tree_attention for requests whose nodes make few rows with a K/V head (up to 64): single tokens, short drafts, trees.
//
// The products are turned round: S^T = K Q^T and O^T = V^T P^T, so that the 128 positions of a cache tile are the 128 rows of the
// tensor cores' tile and the rows of Q are its columns.  With rows as lanes, 8 rows of one decoding token would leave 120 of 128
// threads idle in a softmax of 128 exponentials a thread; here every thread has one position and 8 to 32 exponentials, and what
// belongs to a position (its scales in an 8-bit cache, whether it exists) belongs to a thread.
//
//   * S^T = K Q^T: K as it lies (k-major), Q in shared memory, N = rows rounded up to 16, 32 or 64;
//   * the softmax, two groups of four warps: a thread reads its position's scores, weighs them against one reference a row and
//     writes 16-bit weights, a part of a line of the mn-major operand P^T, to shared memory;
//   * O^T += V^T P^T: V as it lies (mn-major), O^T has a row per component and a column per row of Q.
// Each group has half of the columns of every tile, but for 8-bit caches and up to 16 rows, where the groups take the tiles in turn,
// with an O^T, references and sums each, joined at the end of a unit: a tile's chain of waits and loads is longer than its
// bytes take to arrive (128 tokens over 8192 positions of int8, 8 rows: 454 us when it was made, 536 with halves; over bf16 the same, and a single
// token a microsecond slower; with 32 columns a thread of an 8-bit cache has too few registers, 203 us instead of 193).  A group has two
// S^T and P^T, so that one tile's products run while the next one's weights are made.
//
// The maximum of a row would need a reduction over the threads for every row and tile.  It is not needed: any reference serves
// that keeps the exponentials in range, so the threads only vote whether one of their scores is above its reference by more than
// 2^8; then, seldom, the maxima are found, and O^T and the sums scaled.  The sums of the weights stay in the threads until the
// end of a unit.
//
// Bound by the cache's bytes over bf16: 64 trees of 16 nodes, 4 heads a K/V head, over 4096 positions take 211 us, 5.2 TB/s (one call after
// the other in a replayed graph; 232 us, 4.7 TB/s, where every call finds other inputs), 128 tokens, 8 heads a K/V head, over 8192
// positions 657 us, 6.5 TB/s.  An 8-bit cache has half of the bytes and the same work a tile, and two kinds of warps more: the 128 tokens
// take 460 us over int8, 4.8 TB/s (508 us, 4.4 TB/s), a tile 1 800 clocks: the widening warps' waits, loads and stores, one after
// the other.  The roles' code together is about what the SM's instruction caches hold: code that is seldom run stands out of line or
// inline as measured.
#include <math.h>

#include "tree_attention.cuh"

namespace dspark {

constexpr int kSoftmaxWarps = 8;
constexpr int kFewSmem = 216 * 1024;             // two of P, Q, the ring; tables beside it
template <int kKind, int kN> constexpr bool kFewTurns = kKind != kAttnWide && kN == 16;      // the groups take the tiles in turn
template <int kKind, int kN> constexpr int kFewBuffers = kFewTurns<kKind, kN> ? 4 : 2;
// P^T: a line of 128 bytes a position, of 64 / kN tiles beside one another
constexpr int kFewPBytes = kAttnTile * 128;
template <int kKind, int kN> constexpr int kFewPAll = (kFewBuffers<kKind, kN> * kN + 63) / 64 * kFewPBytes;
template <int kN> __device__ __forceinline__ int few_p_line(uint32_t b) { return (int)(b / (64 / kN)) * kFewPBytes; }
template <int kN> __device__ __forceinline__ int few_p_at(uint32_t b) { return (int)(b % (64 / kN)) * (kN / 8); }      // 16-byte pieces
constexpr float kFewUnset = 1e38f;               // less a reference that every score is above

struct FewShared {
    uint64_t full[kAttnMaxSlots], empty[kAttnMaxSlots], raw_full[kAttnMaxRaw], raw_empty[kAttnMaxRaw];
    uint64_t q_full, q_empty, s_full[4], p_full[4], o_done[4], mma_done[2];
    uint32_t tmem_base;
    int abort;
    uint32_t bad_value[kAttnUnitFlags];          // tiles of a unit whose V had NaN or infinities among the nodes
    AttnStraight straight[8];                    // of each softmax warp
    AttnUnit unit[2];                            // the one that each group is at, for few_bad
    AttnList list;
};
template <int kN>
struct FewTables {
    float less[2][kN];                           // less the references, in units of log2, of either group
    float scale[2][kN];                          // what O^T and the sums are multiplied by when they change, and at the end
    float q[2][kN];                              // 8-bit caches: what a row of Q was divided by, of this unit and the next
    float top[kSoftmaxWarps][kN], sum[kSoftmaxWarps][kN];     // a warp's maxima; its sums at the end
    float kept[2][kN];                           // less the references of what has been put by (few_keep)
    unsigned long long seen[2][kAttnTile];       // rows that see a position (tiles with nodes), for each group
};

// whether one of a group's 128 threads says so
__device__ __forceinline__ bool group_any(int group, bool x) { return barrier_any<128>(group + 1, x); }
__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(group + 1) : "memory"); }
// eight warps widen 8-bit tiles where their registers leave the softmax enough
template <int kKind, int kN> constexpr int kFewConverters = kKind == kAttnWide ? 0 : kN == 64 ? 4 : 8;   // eight: four for K, four for V
template <int kKind, int kN> constexpr int kFewThreads = (kSoftmaxWarps + 3 + kFewConverters<kKind, kN>) * 32;

// The tile's positions that node `self` sees (the unit's node number `place`) get the bits of its rows.  first: where the request's
// nodes begin in the tile.
static __device__ __noinline__ void few_mark(const AttnParams& P, int row0, int first, int self, int place, int straight, int valid,
                                             unsigned long long* seen)
{
    const unsigned long long bits = (P.group == 64 ? ~0ull : (1ull << P.group) - 1) << (place * P.group);
    int a = self, steps = 0;
    for (;;) {
        const int at = first + a;
        if (a < straight) {
            for (int i = max(first, 0); i <= min(at, valid - 1); ++i) atomicOr(&seen[i], bits);
            return;
        }
        if (at < 0) return;
        if (at < valid) atomicOr(&seen[at], bits);
        if (a == 0) return;
        a = attn_parent(P, row0, a, steps);
        if (a < 0) return;
    }
}

// This thread's component of a group's O^T, `columns` of tensor memory at `o`: put by in as many columns at `kept`, and O^T zero again,
// or (back) what was put by added to O^T.  less, kept_less: less the references, now and when it was put by; first: nothing was.
static __device__ __forceinline__ void few_keep(uint32_t o, uint32_t kept, int columns, const float* less, const float* kept_less, bool first, bool back)
{
#pragma unroll 1
    for (int c0 = 0; c0 < columns; c0 += 8) {
        float x[8], k[8];
        attn_read<8>(o + c0, x);
        if (!first) {
            attn_read<8>(kept + c0, k);
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = fmaf(k[c], ex2_approx(less[c0 + c] - kept_less[c0 + c]), x[c]);
        }
        attn_write<8>(back ? o + c0 : kept + c0, reinterpret_cast<const uint32_t (&)[8]>(x));
        if (!back) {
            const uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
            attn_write<8>(o + c0, zero);
        }
    }
    tmem_store_wait();
    tc_fence_before();
}

// Values that were left out of the products, to component `pos` of the rows from e0 on that see them: in the output or, where the unit is
// divided, in the partial result.
template <bool kNarrow, int kE>
__device__ __forceinline__ void few_bad(const AttnParams& P, const AttnUnit& u, const AttnStraight& of, uint32_t tiles, int pos, int e0)
{
    const int straight = attn_straight_of(P, u, of), rows = min(kE, min(P.tile_nodes, u.n - u.node0) * P.group - e0);
    const long long part = (long long)(2 * blockIdx.x + (u.j0 > 0 ? 0 : 1)) * P.part_rows + e0;
    float bad = 0.f;
    for (int c = 0, at = -1; c < rows; ++c) {
        const int r = e0 + c, node = u.node0 + r / P.group;
        if (node != at) attn_bad_values<kNarrow, 1>(P, AttnPart(u), node, straight, tiles, pos, &bad);
        at = node;
        if (bad == 0.f) continue;
        if (u.j0 > 0 || u.j1 < u.tiles) P.parts[(part + c) * P.c.head_dim + pos] += bad;
        else {
            uint16_t* to = reinterpret_cast<uint16_t*>(P.out + (long long)(u.row0 + node) * P.out_row +
                                                       (long long)(u.head * P.group + r % P.group) * P.out_head) + pos;
            *to = (uint16_t)pack16<false>(__uint_as_float((uint32_t)*to << 16) + bad, 0.f);
        }
    }
}

template <int kKind, int kN, bool kLong>         // kLong: units of more than 2 kAttnKeep tiles
__global__ void __launch_bounds__(kFewThreads<kKind, kN>, 1)
attn_few_kernel(const __grid_constant__ AttnParams P, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    constexpr bool kNarrow = kKind != kAttnWide;
    constexpr int kThreads = kFewThreads<kKind, kN>, kProducer = kSoftmaxWarps, kIssuer = kSoftmaxWarps + 1, kIssuerO = kSoftmaxWarps + 2;
    constexpr int kWarps = kFewConverters<kKind, kN>, kOf = kNarrow ? 4 : 1;                 // kOf: warps that make one 16-bit tile
    constexpr bool kTurns = kFewTurns<kKind, kN>;
    constexpr int kBuffers = kFewBuffers<kKind, kN>, kS = 128 / kBuffers;          // kS: columns from one S^T to the next
    constexpr int kE = kN / 2, kC = kTurns ? kN : kE;                       // rows that a group loads and writes; whose weights it makes
    // columns of tensor memory: S^T from 0 on, O^T at 128 (and 160), two K tiles of an 8-bit cache at 192 and 256, O^T put by behind
    constexpr uint32_t kO = 128, kK = 192, kKept = kNarrow ? 320 : 192, kColumns = kNarrow ? 512 : 256;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzle atoms: 1 KB
    __shared__ FewShared S;
    __shared__ __align__(16) FewTables<kN> T;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;    // warp: uniform, and known to be
    const int d = P.c.head_dim, tile_bytes = P.chunks * kChunkBytes;
    unsigned char* sP = smem;
    unsigned char* sQ = sP + kFewPAll<kKind, kN>;     // per 64 components: kN lines of 128 bytes
    const int slots = P.k_slots + P.v_slots;
    unsigned char* ring = sQ + P.chunks * kN * 128 - (kNarrow ? P.k_slots * tile_bytes : 0);       // 8-bit: of V alone
    unsigned char* raw = ring + slots * tile_bytes;

    if (tid == 0) {
        for (int s = 0; s < slots; ++s) { mbar_init(&S.full[s], kOf); mbar_init(&S.empty[s], 1); }
        for (int s = 0; s < P.raw_k + P.raw_v; ++s) { mbar_init(&S.raw_full[s], 1); mbar_init(&S.raw_empty[s], kOf); }
        mbar_init(&S.q_full, kSoftmaxWarps); mbar_init(&S.q_empty, 1);
        for (int b = 0; b < kBuffers; ++b) { mbar_init(&S.s_full[b], 1); mbar_init(&S.p_full[b], kTurns ? 4 : 8); mbar_init(&S.o_done[b], 1); }
        for (int t = 0; t < 2; ++t) mbar_init(&S.mma_done[t], 1);
        for (int i = 0; i < kAttnUnitFlags; ++i) S.bad_value[i] = 0;
        for (AttnStraight& x : S.straight) x.of = -1;
        S.abort = 0;
        mbar_fence_init();
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    AttnIter it = attn_begin<kThreads>(P, S.list);
    const uint32_t tmem = S.tmem_base;
    pdl_trigger();                               // the joining kernel only waits
    volatile int* abort_flag = &S.abort;
    auto give_up = [&]() { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; };
    AttnUnit u;

    if (warp == kProducer) {
        attn_produce<kNarrow>(P, it, map_k, map_v, kNarrow ? raw : ring, kNarrow ? S.raw_full : S.full, kNarrow ? S.raw_empty : S.empty,
                              abort_flag);
    } else if (warp == kIssuer || warp == kIssuerO) {
        // ---------------- products --------------------------------------------------------------------------
        // One warp issues S^T = K Q^T, another O^T += V^T P^T: what a single one has to wait for and to issue for a tile takes it
        // longer than the tile's bytes take to arrive.
        const bool second = warp == kIssuerO;
        const uint32_t type = kNarrow ? 0u : 1u;                            // fp16 or bf16 operands, fp32 sums
        const uint32_t idesc_s = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(kAttnTile >> 4) << 24);
        const uint32_t idesc_o = idesc_s | (1u << 15) | (1u << 16);
        const int first_slot = second ? P.k_slots : 0, ring_slots = second ? P.v_slots : P.k_slots;
        RingPlace place;
        uint32_t units = 0, item = 0;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t p) { ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, p, P.polls)); return ok; };
        while (ok && !__any_sync(0xffffffffu, *abort_flag) && it.next(P, u)) {
            const int n = u.j1 - u.j0;
            if (!second && !wait(&S.q_full, units & 1u)) break;
            ++units;
            for (int i = 0; i < n; ++i, ++item) {
                const uint32_t b = item % kBuffers, turn = item / kBuffers; // which S^T and P^T, for the how-manieth time
                const uint32_t s = (uint32_t)(first_slot + place.s), ph = place.ph;
                if (second) {
                    if (!wait(&S.full[s], ph) || !wait(&S.p_full[b], turn & 1u)) break;
                    tc_fence_after();
                    const uint32_t v = desc_mn_major(smem_u32(ring + s * tile_bytes)), p = desc_mn_major(smem_u32(sP + few_p_line<kN>(b))) + few_p_at<kN>(b);
                    const uint32_t o = tmem + kO + (kTurns ? (item & 1u) * 32 : 0);
                    const bool more = i > (kTurns ? 1 : 0);  // not the first of its O^T
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kAttnTile / 16; ++k) mma_ss(o, v + k * 128, p + k * 128, idesc_o, more || k > 0);
                        umma_commit(&S.empty[s]);
                        umma_commit(&S.o_done[b]);
                    }
                } else {
                    // the scores that were here before have been read
                    if ((turn && !wait(&S.p_full[b], (turn - 1) & 1u)) || !wait(&S.full[s], ph)) break;
                    tc_fence_after();
                    const uint32_t k0 = kNarrow ? 0u : desc_k_major(smem_u32(ring + s * tile_bytes)), q0 = desc_k_major(smem_u32(sQ));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kAttnMaxDim / 16; ++k)
                            if (k >= d / 16) break;
                            else if constexpr (kNarrow)
                                mma_ts(tmem + b * kS, tmem + kK + s * 64 + k * 8, q0 + (k >> 2) * (kN * 8) + (k & 3) * 2, idesc_s, k > 0);
                            else
                                mma_ss(tmem + b * kS, k0 + (k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2, q0 + (k >> 2) * (kN * 8) + (k & 3) * 2, idesc_s, k > 0);
                        umma_commit(&S.s_full[b]);
                        umma_commit(&S.empty[s]);
                        if (i + 1 == n) umma_commit(&S.q_empty);
                    }
                }
                __syncwarp();
                place.next(ring_slots);
            }
        }
        if (!ok && lane == 0) give_up();
        if (units) {                             // tensor memory is returned only after the last product
            if (elect_one()) umma_commit(&S.mma_done[second]);
            __syncwarp();
            mbar_wait_bounded(&S.mma_done[second], 0u);
        }
        __syncwarp();
    } else if (warp < kSoftmaxWarps) {
        // ---------------- softmax ---------------------------------------------------------------------------
        // Within a unit the groups share nothing but the tiles.  A wait that runs out makes `ok` false in its thread; the threads of a
        // group leave together, at the next vote, and where they take turns both groups, at the votes of a unit's start and end.
        const int t = warp >> 2, pos = tid & 127;                           // group; position in a tile, later component
        const int row0 = kTurns ? 0 : t * kC, e0 = t * kE;                  // first of the rows it weighs; of those it loads and writes
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tmem + lane_base + kO, tMine = tO + t * (kTurns ? 32 : kC);          // O^T; that of this group
        constexpr int kStep = kTurns ? 2 : 1;
        auto vote = [&](bool x) { return kTurns ? barrier_any<2 * 128>(3, x) : group_any(t, x); };
        auto first_tile = [&](uint32_t from) { return kTurns ? (int)((from ^ (uint32_t)t) & 1u) : 0; };      // of a unit that starts there
        uint32_t units = 0, item = 0;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t ph) { ok = ok && mbar_wait_bounded(bar, ph, P.polls); };      // each lane for itself
        auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
        // Q of a unit, this group's rows: 128 / kE threads a row, asked for and later stored.
        constexpr int kPer = 128 / kE, kMost = (kAttnMaxDim / 8 + kPer - 1) / kPer;
        const int q_row = e0 + pos / kPer, q_sub = pos % kPer, q_node = q_row / P.group, q_head = q_row - q_node * P.group;
        uint4 x[kMost];
        auto fetch_q = [&](const AttnUnit& w) {
            const bool live = q_row < P.tile_nodes * P.group && w.node0 + q_node < w.n;
            const uint4* src = reinterpret_cast<const uint4*>(P.q + (long long)(w.row0 + w.node0 + q_node) * P.q_row +
                                                              (long long)(w.head * P.group + q_head) * P.q_head);
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                x[i] = make_uint4(0, 0, 0, 0);
                if (live && i * kPer + q_sub < d / 8) x[i] = src[i * kPer + q_sub];
            }
        };
        // With an 8-bit cache as fp16, scaled by a power of two so that no value passes the range and what is lost is below 2^-37
        // of the row's largest (2^-150 at least).
        auto store_q = [&](uint32_t unit) {
            if constexpr (kNarrow) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < kMost; ++i) {
                    const uint32_t w4[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(bf16lo(w4[j])), fabsf(bf16hi(w4[j]))));
                }
#pragma unroll
                for (int o = kPer / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                // 2^e with the largest value below 2^14: exponent field of top to that of 2^13; at most 2^126, whose inverse is no
                // subnormal
                const int e = min(127 + 126, max(1, 254 + 13 - (int)(__float_as_uint(top) >> 23)));
                const float up = __uint_as_float((uint32_t)e << 23);
                if (q_sub == 0) T.q[unit & 1u][q_row] = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
                for (int i = 0; i < kMost; ++i) {
                    x[i].x = pack16<true>(bf16lo(x[i].x) * up, bf16hi(x[i].x) * up);
                    x[i].y = pack16<true>(bf16lo(x[i].y) * up, bf16hi(x[i].y) * up);
                    x[i].z = pack16<true>(bf16lo(x[i].z) * up, bf16hi(x[i].z) * up);
                    x[i].w = pack16<true>(bf16lo(x[i].w) * up, bf16hi(x[i].w) * up);
                }
            }
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const int c = i * kPer + q_sub;
                x[i].x ^= P.q_sign; x[i].y ^= P.q_sign; x[i].z ^= P.q_sign; x[i].w ^= P.q_sign;
                if (c < d / 8) *reinterpret_cast<uint4*>(sQ + (c >> 3) * (kN * 128) + q_row * 128 + (((c & 7) ^ (q_row & 7)) << 4)) = x[i];
            }
            fence_async_smem();
            arrive(&S.q_full);
        };
        // An 8-bit cache's scales of this thread's position, asked for one of the group's tiles ahead, their page two ahead.
        struct Ahead { int page, token; };
        auto page_of = [&](const AttnUnit& w, int jj) {
            Ahead a = {-1, 0};
            if (kNarrow && w.j0 + jj < w.j1 && row0 < min(P.tile_nodes, w.n - w.node0) * P.group) {
                int start, len;
                attn_tile_at(P, w.j0 + jj, start, len);
                if (pos < min(len, w.length - start)) {
                    const int position = start + pos, page = attn_page_of(P, position);
                    a.token = position - page * P.c.page_size;
                    a.page = P.c.block_table[w.r * P.c.table_stride + page];
                }
            }
            return a;
        };
        auto scales_of = [&](const AttnUnit& w, Ahead a) {
            float2 s = make_float2(0.f, 0.f);
            if (kNarrow && a.page >= 0 && a.page < P.c.n_pages) {
                const long long at = ((long long)a.page * P.c.kv_heads + w.head) * P.c.page_size + a.token;
                s = make_float2(P.c.k_scale[at], P.c.v_scale[at]);
            }
            return s;
        };
        Ahead ahead = {-1, 0};
        float2 scale_next = make_float2(0.f, 0.f);
        auto first_scales = [&](uint32_t from) {
            scale_next = scales_of(u, page_of(u, first_tile(from)));
            ahead = page_of(u, first_tile(from) + kStep);
        };
        bool have = it.next(P, u);
        if (have) {
            fetch_q(u);
            store_q(0);
            first_scales(0);
        }
        while (have) {
            if (!kTurns && pos < kC) T.less[t][row0 + pos] = kFewUnset;
            if (tid == 0) S.bad_value[(units + kAttnUnitFlags / 2) % kAttnUnitFlags] = 0;
            if (vote(!ok || *abort_flag)) { ok = false; break; }
            if (kTurns) {                        // both groups have read what there was of the last unit
                if (pos < kC) T.less[t][pos] = kFewUnset;
                group_sync(t);
            }
            uint64_t sums[kC / 2];                                          // of this position's weights, two rows each
#pragma unroll
            for (int c = 0; c < kC / 2; ++c) sums[c] = pack2(0.f, 0.f);
            const int count = u.j1 - u.j0, rows = min(P.tile_nodes, u.n - u.node0) * P.group;
            bool left = false;
            const int first = first_tile(item);
            attn_look_at_tree(P, u, S.straight[warp]);
            if (kKind != kAttnI8 && pos == 0) S.unit[t] = u;
            int jj = first;
            do {
            const int stretch = jj, end = kLong ? min(count, jj + kAttnKeep * kStep) : count;
            for (; jj < end; jj += kStep) {
                const uint32_t number = item + jj, b = number % kBuffers, turn = number / kBuffers;
                const uint32_t tS = tmem + lane_base + b * kS + row0;
                unsigned char* p_line = sP + few_p_line<kN>(b) + pos * 128;
                const int p_at = few_p_at<kN>(b) + row0 / 8;
                int start, len;
                attn_tile_at(P, u.j0 + jj, start, len);
                const int valid = min(len, u.length - start);               // positions of this tile that exist
                const bool masked = start > u.first - kAttnTile || valid < kAttnTile;
                // rows that see this thread's position, a bit each
                unsigned long long seen = ~0ull;
                if (masked) {
                    const int straight = attn_straight_of(P, u, S.straight[warp]);
                    const bool chain = min(u.n, u.node0 + P.unit_nodes) <= straight;        // every node of the unit sees all before it
                    const int node = start - u.first + pos;                 // the node at this position
                    if (pos >= valid) seen = 0;
                    else if (node >= 0 && chain) {
                        const int shift = (node - u.node0) * P.group;
                        seen = shift <= 0 ? ~0ull : shift >= 64 ? 0 : ~0ull << shift;
                    }
                    if (!chain && start + valid > u.first) {
                        T.seen[t][pos] = 0;
                        group_sync(t);
                        if (pos < P.tile_nodes && u.node0 + pos < u.n) few_mark(P, u.row0, u.first - start, u.node0 + pos, pos, straight, valid, T.seen[t]);
                        group_sync(t);
                        if (node >= 0 && pos < valid) seen = T.seen[t][pos];
                    }
                    seen >>= row0;
                }
                float k_scale = P.score_factor, v_scale = scale_next.y;
                const float2 scale = scale_next;
                scale_next = scales_of(u, ahead);
                ahead = page_of(u, jj + 2 * kStep);
                // an 8-bit V: 2^exponent > its scale's size; what a weight may be above its reference depends on it
                float above = 0.f;
                if constexpr (kNarrow) {
                    k_scale *= scale.x;
                    above = attn_exponent(fabsf(scale.y) < INFINITY ? fabsf(scale.y) : 0.f) - kAttnNarrowOffset;
                }
                if (turn) wait(&S.o_done[b], (turn - 1) & 1u);              // P^T that was here before has been multiplied
                wait(&S.s_full[b], turn & 1u);
                __syncwarp();
                tc_fence_after();
                if (row0 < rows) {
                    __syncwarp();
                    if (masked) {
                        // scores of rows that do not see the position: -infinity, in place.  Over an 8-bit cache it has to stay that when
                        // it is multiplied: the others are multiplied here by K's scale up to one and its sign, below by the rest and
                        // the row's factor, whose product is at least 2^-126.  Where a scale is no number the position is NaN for the
                        // rows that see it, and the scales are not used.
                        const bool bad = kNarrow && !(fabsf(scale.x) < INFINITY && fabsf(scale.y) < INFINITY);
                        const float by = fminf(fmaxf(k_scale, -1.f), 1.f);
                        if (kNarrow) k_scale = fmaxf(fabsf(k_scale), 1.f);
#pragma unroll 1
                        for (int c0 = 0; c0 < kC; c0 += 8) {
                            float s[8];
                            attn_read<8>(tS + c0, s);
#pragma unroll
                            for (int c = 0; c < 8; ++c) s[c] = !(seen >> (c0 + c) & 1) ? -INFINITY : bad ? NAN : kNarrow ? s[c] * by : s[c];
                            attn_write<8>(tS + c0, reinterpret_cast<const uint32_t (&)[8]>(s));
                        }
                        tmem_store_wait();
                        if (bad) { k_scale = 1.f; v_scale = 0.f; above = -kAttnNarrowOffset; }
                    }
                    // y = score * factor - reference
                    const uint64_t k2 = pack2(k_scale, k_scale);
                    auto relative = [&](float (&s)[kC]) {
#pragma unroll
                        for (int c = 0; c < kC; c += 2) {
                            uint64_t k = k2;
                            if constexpr (kNarrow) k = mul2(k, *reinterpret_cast<const uint64_t*>(&T.q[units & 1u][row0 + c]));
                            unpack2(fma2(pack2(s[c], s[c + 1]), k, *reinterpret_cast<const uint64_t*>(&T.less[t][row0 + c])), s[c], s[c + 1]);
                        }
                    };
                    float y[kC], tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    attn_read<kC>(tS, y);
                    relative(y);
#pragma unroll
                    for (int c = 0; c < kC; c += 2) tops[c / 2 % 4] = fmaxf(tops[c / 2 % 4], fmaxf(y[c], y[c + 1]));
                    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                    if (group_any(t, !ok || top + above > kAttnLazy)) {
                        // references: the largest score of each row in this tile, where it is that much above
                        if (jj > first) wait(&S.o_done[(number - kStep) % kBuffers], (number - kStep) / kBuffers & 1u);     // O^T of the tile before
                        if (group_any(t, !ok)) { left = true; break; }
                        tc_fence_after();
                        __syncwarp();
#pragma unroll 1
                        for (int c0 = 0; c0 < kC; c0 += 8) {
                            float s[8], mine = -INFINITY;
                            attn_read<8>(tS + c0, s);
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const float z = warp_max_f32(s[c] * (kNarrow ? k_scale * T.q[units & 1u][row0 + c0 + c] : k_scale) + above);
                                if (lane == c) mine = z;
                            }
                            if (lane < 8) T.top[warp][row0 + c0 + lane] = mine;
                            __syncwarp();
                        }
                        group_sync(t);
                        if (pos < kC) {
                            const int r = row0 + pos;
                            const float old = -T.less[t][r], now = fmaxf(fmaxf(T.top[4 * t][r], T.top[4 * t + 1][r]), fmaxf(T.top[4 * t + 2][r], T.top[4 * t + 3][r]));
                            const bool raise = now > old + kAttnLazy;
                            T.scale[t][r] = raise ? ex2_approx(old - now) : 1.f;
                            if (raise) T.less[t][r] = -now;
                        }
                        group_sync(t);
                        __syncwarp();
#pragma unroll
                        for (int c = 0; c < kC / 2; ++c) sums[c] = mul2(sums[c], *reinterpret_cast<const uint64_t*>(&T.scale[t][row0 + 2 * c]));
                        if (jj > first) {
#pragma unroll 1
                            for (int c0 = 0; c0 < kC; c0 += 8) {
                                float o[8];
                                attn_read<8>(tMine + c0, o);
#pragma unroll
                                for (int c = 0; c < 8; ++c) o[c] *= T.scale[t][row0 + c0 + c];
                                attn_write<8>(tMine + c0, reinterpret_cast<const uint32_t (&)[8]>(o));
                            }
                            tmem_store_wait();
                        }
                        attn_read<kC>(tS, y);
                        relative(y);
                    }
                    uint32_t w[kC / 2];
#pragma unroll
                    for (int c = 0; c < kC; c += 2) {
                        float e0 = ex2_approx(y[c]), e1 = ex2_approx(y[c + 1]);
                        const uint64_t e = pack2(e0, e1);
                        sums[c / 2] = add2(sums[c / 2], e);
                        if constexpr (kNarrow) unpack2(mul2(e, pack2(v_scale, v_scale)), e0, e1);
                        w[c / 2] = pack16<kNarrow>(e0, e1);
                    }
#pragma unroll
                    for (int c = 0; c < kC / 8; ++c)
                        *reinterpret_cast<uint4*>(p_line + (((p_at + c) ^ (pos & 7)) << 4)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                }
                if (!kNarrow && masked) {
                    // V of positions that no row sees, or that hold NaN or infinities that only some see, must not meet a
                    // weight of zero in the product: zeros here, the latter added to the rows that see them at the end
                    const uint32_t s = P.k_slots + number % P.v_slots;
                    wait(&S.full[s], number / P.v_slots & 1u);
                    if ((kTurns || (pos & 1) == t) && (pos >= u.first - start || pos >= valid))
                        if (attn_clean_values(ring + (size_t)s * tile_bytes + pos * 128, pos, P.chunks, pos < valid))
                            atomicOr(&S.bad_value[units % kAttnUnitFlags], attn_tile_bit(u.j0 + jj));
                }
                fence_async_smem();
                tc_fence_before();
                arrive(&S.p_full[b]);
            }
            if (kLong && !left && jj < count && row0 < rows) {
                const uint32_t last = item + jj - kStep;
                wait(&S.o_done[last % kBuffers], last / kBuffers & 1u);
                __syncwarp();
                tc_fence_after();
                few_keep(tMine, tMine - kO + kKept, kC, T.less[t] + row0, T.kept[t] + row0, stretch == first, false);
                group_sync(t);
                if (pos < kC) T.kept[t][row0 + pos] = T.less[t][row0 + pos];
            }
            } while (kLong && !left && jj < count);
            if (left) { if (kTurns) vote(true); ok = false; break; }        // all of the group; the other one learns of it
            item += count;
            // The next unit's Q and scales, asked for while the products of this one are finished.
            const AttnUnit done = u;
            have = it.next(P, u);
            if (have) {
                fetch_q(u);
                first_scales(item);
            }
            if (row0 < rows) {
                // sums over the positions of this warp: half of the rows pass to the other half of the lanes, as long as there are
                // rows to part
                float v[kC];
#pragma unroll
                for (int c = 0; c < kC / 2; ++c) unpack2(sums[c], v[2 * c], v[2 * c + 1]);
                int left_rows = kC, row = 0;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    if (left_rows > 1) {
                        left_rows >>= 1;
#pragma unroll
                        for (int c = 0; c < kC / 2; ++c)
                            if (c < left_rows) {
                                const float give = (lane & o) ? v[c] : v[c + left_rows], keep = (lane & o) ? v[c + left_rows] : v[c];
                                v[c] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                            }
                        if (lane & o) row += left_rows;
                    } else
                        v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                }
                T.sum[warp][row0 + row] = v[0];                         // the lanes of a row write the same
            }
            wait(&S.q_empty, units & 1u);        // this unit's Q has been multiplied: the next one's takes its place
            if (have) store_q(units + 1);
            if (first < count) {                 // the group's last tile
                const uint32_t last = item - count + first + (count - 1 - first) / kStep * kStep;
                wait(&S.o_done[last % kBuffers], last / kBuffers & 1u);
            }
            __syncwarp();
            tc_fence_after();
            if (kLong && row0 < rows && (count - 1 - first) / kStep >= kAttnKeep)
                few_keep(tMine, tMine - kO + kKept, kC, T.less[t] + row0, T.kept[t] + row0, false, true);
            if (vote(!ok)) { ok = false; break; }
            tc_fence_after();
            if (e0 < rows) {
                const bool whole = done.j0 == 0 && done.j1 == done.tiles;
                const long long part = (long long)(2 * blockIdx.x + (done.j0 > 0 ? 0 : 1)) * P.part_rows + e0;
                const int mine = min(kE, rows - e0);
                const int node0 = done.node0 + e0 / P.group, head0 = e0 % P.group;              // of the group's first row
                // where the groups took turns: both have had a tile?  (one tile: the other's O^T has not been written)
                const int only = kTurns && count == 1 ? (int)((item - 1) & 1u) : -1;
                if (pos < mine) {
                    const int r = e0 + pos;
                    const int g = kTurns ? 0 : t;
                    float sum = (T.sum[4 * g][r] + T.sum[4 * g + 1][r]) + (T.sum[4 * g + 2][r] + T.sum[4 * g + 3][r]), ref = -T.less[g][r];
                    float f0 = 1.f, f1 = 0.f;
                    if (kTurns) {
                        const float sum1 = (T.sum[4][r] + T.sum[5][r]) + (T.sum[6][r] + T.sum[7][r]), ref1 = -T.less[1][r];
                        const float top = fmaxf(ref, ref1);
                        f0 = ex2_approx(ref - top);
                        f1 = ex2_approx(ref1 - top);
                        sum = sum * f0 + sum1 * f1;
                        ref = top;
                    }
                    const float inverse = whole ? 1.f / sum : 1.f;
                    T.scale[kTurns ? 0 : t][r] = f0 * inverse;
                    if (kTurns) T.scale[1][r] = f1 * inverse;
                    if (!whole) P.part_stats[part + pos] = make_float2(ref, sum);
                    else if (P.out_lse)
                        P.out_lse[(long long)(done.row0 + done.node0 + r / P.group) * P.q_heads + done.head * P.group + r % P.group] =
                            (log2f(sum) + ref) * 0.6931471805599453f;
                }
                group_sync(t);
                unsigned char* to = P.out + (long long)(done.row0 + node0) * P.out_row + (long long)(done.head * P.group + head0) * P.out_head + pos * 2;
                const long long next_node = P.out_row - (P.group - 1) * P.out_head;
                float* to_part = P.parts + part * d + pos;
                int in_group = head0;
                __syncwarp();
#pragma unroll 1
                for (int h = 0; h < mine; h += 8) {
                    float o[8];
                    attn_read<8>(tO + (only == 1 ? 32 : 0) + e0 + h, o);
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[c] *= T.scale[kTurns ? (only == 1 ? 1 : 0) : t][e0 + h + c];
                    if (kTurns && only < 0) {
                        float o1[8];
                        attn_read<8>(tO + 32 + e0 + h, o1);
#pragma unroll
                        for (int c = 0; c < 8; ++c) o[c] = fmaf(o1[c], T.scale[1][e0 + h + c], o[c]);
                    }
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        if (h + c < mine && pos < d) {
                            const float value = o[c];
                            if (whole) *reinterpret_cast<uint16_t*>(to) = (uint16_t)pack16<false>(value, 0.f);
                            else to_part[(h + c) * d] = value;
                        }
                        if (++in_group == P.group) { in_group = 0; to += next_node; } else to += P.out_head;
                    }
                    __syncwarp();
                }
                if (kKind != kAttnI8 && *(volatile uint32_t*)&S.bad_value[units % kAttnUnitFlags] != 0u && pos < d)
                    few_bad<kNarrow, kE>(P, S.unit[t], S.straight[warp], S.bad_value[units % kAttnUnitFlags], pos, e0);
                tc_fence_before();
            }
            ++units;
        }
        if (!ok) give_up();
    } else {
        if constexpr (kNarrow) {
            const int ct = tid - (kSoftmaxWarps + 3) * 32, kv = kWarps == 8 ? ct >> 7 : 0;
            if (!attn_widen<kKind, 128, true>(P, it, ct & 127, kv, kWarps == 8 ? kv : 1, raw, ring, tile_bytes, S.raw_full, S.raw_empty, S.full, S.empty,
                                              tmem + kK, S.bad_value, abort_flag, [](const AttnUnit&, int) {}, [](int) {}) &&
                lane == 0)
                give_up();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kColumns) : "memory");
    }
}

template <int kKind, int kN, bool kLong>
static int few_launch(AttnParams& P, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    static std::atomic<unsigned long long> ready{0};
    constexpr int kSmem = kFewSmem + 1024;
    if (!attn_allow_smem(attn_few_kernel<kKind, kN, kLong>, kSmem, ready)) return launch_status();
    const int tile = P.chunks * kChunkBytes;
    // a chunk is left behind the ring: with up to 64 components the products read one past a tile (and nobody its results)
    int room = kFewSmem - kFewPAll<kKind, kN> - P.chunks * kN * 128 - (P.chunks == 1 ? kChunkBytes : 0);
    // V tiles stay longer than K tiles: until their weights are there.  8-bit caches: two of each as 16 bits (K's in tensor memory),
    // the rest for 8-bit ones on their way: 128 KB of them in flight per SM, or the memory's latency shows.
    const int slots = room / tile < kAttnMaxSlots ? room / tile : kAttnMaxSlots;
    P.k_slots = kKind != kAttnWide ? 2 : slots / 2;
    P.v_slots = kKind != kAttnWide ? 2 : slots - P.k_slots;
    const int raw = (room - P.v_slots * tile) / (kAttnTile * P.c.head_dim), most = raw < kAttnMaxRaw ? raw : kAttnMaxRaw;
    P.raw_k = kKind == kAttnWide ? 0 : most / 2;
    P.raw_v = kKind == kAttnWide ? 0 : most - P.raw_k;
    KernelTimerScope timer(DSPARK_K_TREE_ATTENTION, s);
    launch_pdl(attn_few_kernel<kKind, kN, kLong>, dim3((unsigned)sms), dim3(kFewThreads<kKind, kN>), kSmem, s, P, k, v);
    return launch_status();
}
template <int kKind, int kN>
static int few_launch(AttnParams& P, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    // Room for more than 65536 positions: the kernel that puts its sums by (with that code 128 tokens over 8192 positions of int8 take 467 us,
    // without it 445; trees of 8 nodes, 64 rows 460 and 448).  Without, 512 tiles are cut by less than 2^-11.
    return kv_capacity(P.c) > 2 * kAttnKeep * kAttnTile ? few_launch<kKind, kN, true>(P, k, v, sms, s) : few_launch<kKind, kN, false>(P, k, v, sms, s);
}
template <int kKind>
static int few_rows(AttnParams& P, int rows, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    if (rows <= 16) return few_launch<kKind, 16>(P, k, v, sms, s);
    if (rows <= 32) return few_launch<kKind, 32>(P, k, v, sms, s);
    return few_launch<kKind, 64>(P, k, v, sms, s);
}
int attn_few_launch(AttnParams& P, int rows, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    if (P.c.dtype == DSPARK_BF16) return few_rows<kAttnWide>(P, rows, k, v, sms, s);
    if (P.c.dtype == DSPARK_I8) return few_rows<kAttnI8>(P, rows, k, v, sms, s);
    return few_rows<kAttnE4M3>(P, rows, k, v, sms, s);
}

}  // namespace dspark
