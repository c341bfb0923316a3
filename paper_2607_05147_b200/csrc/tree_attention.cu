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
//   * a producer warp brings K and V tiles into a ring each by tensor-map copies, a page a box;
//   * one thread issues tcgen05.mma: S = Q K^T into tensor memory (Q and K in shared memory), then O += P V, with P taken from
//     tensor memory and V as it lies (mn-major);
//   * two groups of eight warps do the softmax, a row in two threads, half of a tile's positions each: they read S, write P over
//     it as 16-bit values (what the product takes: off by half a step of 2^-8 or 2^-11 each, up as often as down, so that the sum is
//     nearer than the result's own rounding; the sum of the weights is that of the unrounded ones), and scale O only when the maximum has risen by more than 2^8 (the reference is any number that keeps
//     the exponentials in range).  The groups have one S and one O each: with two row tiles they take one of them each; with one
//     they take the even and the odd cache tiles and join at the end.  While one group works on its S the tensor cores do the
//     other's products.
//   * 8-bit caches: four more warps turn the tiles into 16-bit floats (exact for both types) in a second pair of rings.  The scales
//     of K multiply the scores and those of V the weights, so that neither is rounded into the operands.
//
// This kernel is for more than 64 rows with a K/V head; up to there tree_attention_few.cu does the work.
//
// Bound by the cache's bytes up to about 128 rows over bf16 (64 requests of 32 nodes, 4 heads a K/V head, over 4096 positions: 244 us,
// 4.5 TB/s, in a replayed graph like the other times here), beyond by the chain scores -> exponentials -> products of a group, which the other group's covers in part: a tile
// for 256 rows over e4m3 takes 6 800 clocks, of which the exponentials alone are 2 048 and the products 1 500.  64 nodes over 131072
// positions: 236 us, 0.58 PFLOP/s.  A prompt of 8192, 32 heads: 1.28 ms over bf16, 0.43 PFLOP/s of those that are seen.
// Tried and not kept: a warp a group for the products (the groups fall into step, 259 us); the weights made in the pass that finds
// the largest score (32 more registers than there are).
#include "tree_attention.cuh"

namespace dspark {

// ---- the kernel ------------------------------------------------------------------------------------------
struct AttnShared {
    uint64_t full[kAttnMaxSlots], empty[kAttnMaxSlots];       // 16-bit tiles
    uint64_t raw_full[kAttnMaxRaw], raw_empty[kAttnMaxRaw];   // 8-bit tiles
    uint64_t q_full, s_full[2], p_full[2], o_full[2], merge_ready, merge_done, mma_done;
    uint32_t tmem_base;
    int abort;
    uint32_t bad_value[kAttnUnitFlags];          // tiles of a unit whose V had NaN or infinities among the nodes
    AttnStraight straight[16];                   // of each softmax warp
    AttnList list;
    float2 second[kAttnTile];                    // (reference, sum) of the second group
    float of_half[2][2][kAttnTile];              // what the two threads of a row tell one another: largest scores, sums
    float kept[2][2][kAttnTile];                 // reference of what a row's threads have put by (attn_keep)
};
template <int kKind>
struct AttnScales {                              // q: per row
    float k[kAttnScaleTiles][kAttnTile], v[kAttnScaleTiles][kAttnTile], q[2][kAttnTile];
    // Nodes' positions, which some rows do not see, whose K scale is not a positive number: a bit each in odd, the scale here and 1
    // in k.  A score of -infinity has to stay that after the product with k.
    float odd_k[kAttnScaleTiles][kAttnTile];
    uint32_t odd[kAttnScaleTiles][4];
};
template <> struct AttnScales<kAttnWide> {};

constexpr int kRowWarps = 16;                    // of the softmax: two groups of four warps a half
constexpr int kAttnConverters = 4;
template <int kKind> constexpr int kAttnCols = kKind == kAttnWide ? 32 : 16;    // scores in registers at a time
template <int kKind> constexpr int kAttnThreads = (kRowWarps + 2 + (kKind == kAttnWide ? 0 : kAttnConverters)) * 32;

// A row's components [begin, end) of O, at tensor memory `o`: put by in memory and O zero again, or (back) what was put by added to O.
// by: 2 to the reference that it was put by with less the present one; 0: nothing was.  kept: NULL for a row that is none.
static __device__ __noinline__ void attn_keep(uint32_t o, int begin, int end, float* kept, float by, bool back)
{
    for (int c = begin; c < end; c += 16) {
        float x[16];
        tmem_load16(o + c, x);
        if (kept)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float4* at = reinterpret_cast<float4*>(kept + c + i);
                const float4 k = by != 0.f ? *at : make_float4(0.f, 0.f, 0.f, 0.f);
                x[i] = fmaf(k.x, by, x[i]); x[i + 1] = fmaf(k.y, by, x[i + 1]);
                x[i + 2] = fmaf(k.z, by, x[i + 2]); x[i + 3] = fmaf(k.w, by, x[i + 3]);
                if (!back) *at = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
            }
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = back ? __float_as_uint(x[i]) : 0u;
        tmem_store16(o + c, w);
    }
    tmem_store_wait();
}

template <bool kNarrow>
__device__ __noinline__ void attn_bad_row(const AttnParams& P, AttnPart u, int node, int straight, uint32_t tiles, int i, float* sum)
{
    attn_bad_values<kNarrow, 16>(P, u, node, straight, tiles, i, sum);
}

template <int kKind>
__global__ void __launch_bounds__(kAttnThreads<kKind>, 1)
attn_kernel(const __grid_constant__ AttnParams P, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    constexpr bool kNarrow = kKind != kAttnWide;
    constexpr int kThreads = kAttnThreads<kKind>, kProducer = kRowWarps, kIssuer = kRowWarps + 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzle atoms: 1 KB
    __shared__ AttnShared S;
    __shared__ __align__(16) AttnScales<kKind> scales;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;    // warp: uniform, and known to be
    const int d = P.c.head_dim, tile_bytes = P.chunks * kChunkBytes;
    unsigned char* sQ = smem;
    unsigned char* ring = smem + P.q_tiles * tile_bytes;
    const int slots = P.k_slots + P.v_slots;
    unsigned char* raw = ring + slots * tile_bytes;

    if (tid == 0) {
        for (int s = 0; s < slots; ++s) { mbar_init(&S.full[s], kNarrow ? kAttnConverters : 1); mbar_init(&S.empty[s], 1); }
        for (int s = 0; s < P.raw_k + P.raw_v; ++s) { mbar_init(&S.raw_full[s], 1); mbar_init(&S.raw_empty[s], kAttnConverters); }
        mbar_init(&S.q_full, kRowWarps);
        for (int t = 0; t < 2; ++t) { mbar_init(&S.s_full[t], 1); mbar_init(&S.p_full[t], kRowWarps / 2); mbar_init(&S.o_full[t], 1); }
        for (int i = 0; i < kAttnUnitFlags; ++i) S.bad_value[i] = 0;
        mbar_init(&S.merge_ready, kRowWarps / 2); mbar_init(&S.merge_done, kRowWarps / 2); mbar_init(&S.mma_done, 1);
        for (AttnStraight& x : S.straight) x.of = -1;
        S.abort = 0;
        mbar_fence_init();
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();

    AttnIter it = attn_begin<kThreads>(P, S.list);
    const uint32_t tmem = S.tmem_base;
    pdl_trigger();                               // the joining kernel only waits
    volatile int* abort_flag = &S.abort;
    auto give_up = [&]() { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; };
    const int tile_nodes = P.tile_nodes;
    AttnUnit u;

    if (warp == kProducer) {
        attn_produce<kNarrow>(P, it, map_k, map_v, kNarrow ? raw : ring, kNarrow ? S.raw_full : S.full, kNarrow ? S.raw_empty : S.empty,
                              abort_flag);
    } else if (warp == kIssuer) {
        // ---------------- products --------------------------------------------------------------------------
        const uint32_t type = kNarrow ? 0u : 1u;                            // fp16 or bf16 operands, fp32 sums
        const uint32_t common = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(kAttnTile >> 4) << 24);
        const uint32_t idesc_s = common | ((uint32_t)(kAttnTile >> 3) << 17);
        const uint32_t idesc_o = common | ((uint32_t)(d >> 3) << 17) | (1u << 16);
        const uint32_t q0 = desc_k_major(smem_u32(sQ)), k0 = desc_k_major(smem_u32(ring)), v0 = desc_mn_major(smem_u32(ring));
        const uint32_t tile_step = (uint32_t)tile_bytes >> 4;
        const int steps = d / 16;
        uint32_t units = 0, items[2] = {0, 0};
        bool ok = true, issued = false;
        RingPlace k_at, v_at;
        auto wait = [&](uint64_t* bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, ph, P.polls)); return ok; };
        while (ok && !__any_sync(0xffffffffu, *abort_flag) && it.next(P, u)) {
            const int n = (u.j1 - u.j0) << (u.pair ? 1 : 0);
            const bool pair = u.pair;
            auto scores = [&](uint32_t t) {
                const uint32_t ks = (uint32_t)k_at.s;
                if (!wait(&S.full[ks], k_at.ph)) return;
                tc_fence_after();
                const uint32_t a = q0 + (pair && t ? tile_step : 0u), b = k0 + ks * tile_step;
                const bool last = !pair || t;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kAttnMaxDim / 16; ++k)
                        if (k < steps) {
                            const uint32_t at = (uint32_t)((k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2);
                            mma_ss(tmem + t * 128, a + at, b + at, idesc_s, k > 0);
                        }
                    umma_commit(&S.s_full[t]);
                    if (last) umma_commit(&S.empty[ks]);
                }
                __syncwarp();
                if (last) k_at.next(P.k_slots);
                issued = true;
            };
            if (!wait(&S.q_full, units & 1u)) break;
            ++units;
            tc_fence_after();
            scores(0);
            if (n > 1) scores(1);
            for (int i = 0; ok && i < n; ++i) {
                const uint32_t t = (uint32_t)(i & 1);
                const uint32_t vs = (uint32_t)(P.k_slots + v_at.s);
                if (!wait(&S.p_full[t], (t ? items[1] : items[0]) & 1u) || !wait(&S.full[vs], v_at.ph)) break;
                if (t) ++items[1]; else ++items[0];
                tc_fence_after();
                const uint32_t b = v0 + vs * tile_step;
                const bool last = !pair || t;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kAttnTile / 16; ++k)
                        mma_ts(tmem + 256 + t * 128, tmem + t * 128 + (k >> 2) * 64 + (k & 3) * 8, b + k * 128, idesc_o, i > 1 || k > 0);
                    if (last) umma_commit(&S.empty[vs]);
                    if (pair) { if (i + 2 >= n) umma_commit(&S.o_full[t]); }
                    else if (i + 1 == n) { umma_commit(&S.o_full[0]); umma_commit(&S.o_full[1]); }   // the groups share Q
                }
                __syncwarp();
                if (last) v_at.next(P.v_slots);
                if (i + 2 < n) scores(t);
            }
        }
        if (!ok && lane == 0) give_up();
        if (issued) {
            if (elect_one()) umma_commit(&S.mma_done);
            __syncwarp();
            mbar_wait_bounded(&S.mma_done, 0u);
        }
        __syncwarp();
    } else if (warp < kRowWarps) {
        // ---------------- softmax ---------------------------------------------------------------------------
        // A row belongs to a thread in each of two warps, which have 64 of a tile's positions each and later half of the row's
        // components.  They share the row's reference; the two warps vote on it.  A wait that runs out makes `ok` false in its
        // warp; the two leave together, at the next vote.
        const int t = warp >> 3, half = warp >> 2 & 1, row = tid & 127;     // group; half; row of the tile
        const int pair_id = t * 4 + (warp & 3);
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_base + t * 128 + half * 64, tO = tmem + lane_base + 256 + t * 128;
        const int o_begin = half ? (d + 31) / 32 * 16 : 0, o_end = half ? d : (d + 31) / 32 * 16;          // components
        uint32_t units = 0, items = 0, merges = 0;
        uint32_t seq = 0;                        // cache tiles of earlier units
        bool ok = true, merged = false;
        auto wait = [&](uint64_t* bar, uint32_t ph) { ok = ok && mbar_wait_bounded(bar, ph, P.polls); };      // each lane for itself
        auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
        auto vote = [&](bool x) { return barrier_any<64>(pair_id + 1, x); };
        // Row tile `tile` of a unit into shared memory by the eight warps of a group, 16 rows a warp, 16 lanes a row: a row a thread
        // would ask for 32 lines with every load.  In 8-bit mode as fp16, scaled by a power of two so that no value passes the range
        // and what is lost is below 2^-37 of the row's largest (2^-150 at least).
        auto load_q = [&](const AttnUnit& w, int tile) {
            const int sub = lane & 15;
            const bool in = sub < d / 8;
            unsigned char* dst = sQ + tile * tile_bytes + (sub >> 3) * kChunkBytes;
#pragma unroll 1
            for (int i0 = 0; i0 < 8; i0 += 4) {
                const int r0 = (warp & 7) * 16 + i0 * 2 + (lane >> 4);      // and the second, fourth and sixth behind it
                uint4 x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + 2 * i, of = r / P.group, node = w.node0 + tile * tile_nodes + of;
                    x[i] = make_uint4(0, 0, 0, 0);
                    if (in && of < tile_nodes && node < w.n)
                        x[i] = reinterpret_cast<const uint4*>(P.q + (long long)(w.row0 + node) * P.q_row + (long long)(w.head * P.group + r - of * P.group) * P.q_head)[sub];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + 2 * i;
                    if constexpr (kNarrow) {
                        const uint32_t w4[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                        float top = 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) top = max3(top, fabsf(bf16lo(w4[k])), fabsf(bf16hi(w4[k])));
#pragma unroll
                        for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        // 2^e with the largest value below 2^14: exponent field of top to that of 2^13; at most 2^126, whose
                        // inverse is no subnormal
                        const int e = min(127 + 126, max(1, 254 + 13 - (int)(__float_as_uint(top) >> 23)));
                        const float up = __uint_as_float((uint32_t)e << 23);
                        if (sub == 0) scales.q[tile][r] = __uint_as_float((uint32_t)(254 - e) << 23);       // the inverse power
                        x[i].x = pack16<true>(bf16lo(x[i].x) * up, bf16hi(x[i].x) * up);
                        x[i].y = pack16<true>(bf16lo(x[i].y) * up, bf16hi(x[i].y) * up);
                        x[i].z = pack16<true>(bf16lo(x[i].z) * up, bf16hi(x[i].z) * up);
                        x[i].w = pack16<true>(bf16lo(x[i].w) * up, bf16hi(x[i].w) * up);
                    }
                    x[i].x ^= P.q_sign; x[i].y ^= P.q_sign; x[i].z ^= P.q_sign; x[i].w ^= P.q_sign;
                    if (in) *reinterpret_cast<uint4*>(dst + r * 128 + (((sub & 7) ^ (r & 7)) << 4)) = x[i];
                }
            }
            fence_async_smem();
        };
        // Where this row's part of O is put by: the place of the unit's partial result (of a whole unit: that of the CTA's last unit,
        // which comes later), the second group's behind the first one's.
        auto keep_row = [&](const AttnUnit& w) { return P.parts + ((long long)(2 * blockIdx.x + (w.j0 > 0 ? 0 : 1)) * P.part_rows + t * kAttnTile + row) * d; };
        bool have = it.next(P, u);
        // Q of the first unit; afterwards each unit's is loaded at the end of the one before
        auto prepare_q = [&](const AttnUnit& w) {
            if (w.pair || t == 0) load_q(w, t);
            arrive(&S.q_full);
        };
        if (have) prepare_q(u);
        while (have) {
            if (vote(!ok || *abort_flag)) { ok = false; break; }
            const int tile = u.pair ? t : 0;
            const int node = u.node0 + tile * tile_nodes + row / P.group;
            const bool live = row < tile_nodes * P.group && node < u.n;
            const bool warp_live = __any_sync(0xffffffffu, live);           // the same in both warps
            attn_look_at_tree(P, u, S.straight[warp]);
            float factor = P.score_factor;       // 8-bit caches: what the row of Q was scaled by (K's scales hold score_factor)
            if (tid == 0) S.bad_value[(units + kAttnUnitFlags / 2) % kAttnUnitFlags] = 0;
            float ref = kAttnUnset, sum = 0.f;   // O and the sum are relative to 2^ref
            bool any = false, left = false;      // any: O holds something
            const int step = u.pair ? 1 : 2;
            const int count = u.j1 - u.j0;
            for (int jj = u.pair ? 0 : t; jj < count && !left;) {
            const int stretch = jj, end = min(count, jj + kAttnKeep * step);
            for (; jj < end; jj += step) {
                int start, len;
                attn_tile_at(P, u.j0 + jj, start, len);
                const int valid = min(len, u.length - start);               // positions of this tile that exist
                const bool masked = start > u.first - kAttnTile || valid < kAttnTile;
                // which positions this row sees, a bit each
                uint32_t seen[4] = {~0u, ~0u, ~0u, ~0u};
                bool chain = true;               // every node of the unit sees all before it
                if (masked && warp_live) {
                    // positions from this tile's start on that are before the step, or up to a node: a range; other nodes one by one
                    const int straight = attn_straight_of(P, u, S.straight[warp]), before = min(u.first - start, kAttnTile);
                    auto see_to = [&](int upto) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const int c = min(min(upto, valid) - 32 * w, 32);
                            seen[w] = c <= 0 ? 0u : c == 32 ? ~0u : (1u << c) - 1u;
                        }
                    };
                    chain = min(u.n, u.node0 + P.unit_nodes) <= straight;
                    see_to(before + (node < straight ? node + 1 : 0));
                    if (node >= straight && live && start + valid > u.first) {
                        int a = node, steps = 0;
                        uint32_t one[4] = {0u, 0u, 0u, 0u};
                        for (;;) {
                            if (a < straight) { see_to(before + a + 1); break; }
                            const int at = u.first + a - start;
                            if (at < 0) break;
                            if (at < valid) {
#pragma unroll
                                for (int w = 0; w < 4; ++w) if ((at >> 5) == w) one[w] |= 1u << (at & 31);
                            }
                            if (a == 0) break;
                            a = attn_parent(P, u.row0, a, steps);
                            if (a < 0) break;
                        }
#pragma unroll
                        for (int w = 0; w < 4; ++w) seen[w] |= one[w];
                    }
                }
                wait(&S.s_full[t], items & 1u);
                __syncwarp();
                ++items;
                tc_fence_after();
                const float* fk = nullptr;
                const float* fv = nullptr;
                float above = 0.f;               // what a weight may be above its reference is less by this
                if constexpr (kNarrow) {
                    if (warp_live) {
                    // the scales of this tile have been stored before its K tile was announced
                    const int at = (int)((seq + jj) % kAttnScaleTiles);
                    const float* all = scales.v[at];
                    fk = scales.k[at] + half * 64;
                    fv = scales.v[at] + half * 64;
                    if (!any) factor = scales.q[tile][row];                 // stored before Q was announced
                    if (!masked) above = attn_exponent(warp_max_f32(attn_finite_max(reinterpret_cast<const float4*>(all)[lane])));
                    else {                       // of the positions that this row sees
                        // every lane has four positions' scales: the largest up to each (a chain), or of those before the step (a tree)
                        __syncwarp();
                        const float4 mine = reinterpret_cast<const float4*>(all)[lane];
                        const int before = chain ? 4 : u.first - start - lane * 4;         // that many of the four
                        float upto[4], top = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = fabsf(i == 0 ? mine.x : i == 1 ? mine.y : i == 2 ? mine.z : mine.w);
                            upto[i] = top = i < before && x < INFINITY ? fmaxf(top, x) : top;
                        }
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const float x = __shfl_up_sync(0xffffffffu, top, o);
                            if (lane >= o) top = fmaxf(top, x);
                        }
                        if (!chain) {
                            top = __shfl_sync(0xffffffffu, top, 31);
                            const int tree = max(u.first - start, 0);       // the first node's place
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                uint32_t of = tree >= 32 * w + 32 ? 0u : tree > 32 * w ? seen[w] >> (tree - 32 * w) << (tree - 32 * w) : seen[w];
                                for (; of; of &= of - 1) {
                                    const float x = fabsf(all[w * 32 + __ffs(of) - 1]);
                                    if (x < INFINITY) top = fmaxf(top, x);
                                }
                            }
                            __syncwarp();
                        } else {
                            const int last = min(min(u.first - start, kAttnTile) + node, valid - 1);       // the last that this row sees
                            const float earlier = __shfl_up_sync(0xffffffffu, top, 1);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float x = __shfl_sync(0xffffffffu, lane ? fmaxf(earlier, upto[i]) : upto[i], max(last, 0) >> 2);
                                if ((last & 3) == i) top = x;
                            }
                            if (last < 0) top = 0.f;
                        }
                        above = attn_exponent(top);
                    }
                    above -= kAttnNarrowOffset;
                    if (masked) {
                        // scores of positions that the row does not see: -infinity, in place
                        __syncwarp();
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t on = half ? seen[2 + w] : seen[w], odd = on & scales.odd[at][half * 2 + w];
                            attn_hide<true>(tS + w * 32, on, odd, scales.odd_k[at] + half * 64 + w * 32);
                        }
                    }
                    }
                } else if (masked && warp_live) {
                    __syncwarp();
#pragma unroll
                    for (int w = 0; w < 2; ++w) attn_hide<false>(tS + w * 32, half ? seen[2 + w] : seen[w], 0u, nullptr);
                }
                if (warp_live) {
                    // scores from tensor memory, with an 8-bit cache times K's scales; the next ones are asked for meanwhile
                    constexpr int kCols = kAttnCols<kKind>;
                    float ahead[2][kCols];
                    auto scores = [&](int c, float (&x)[kCols], float (&next)[kCols]) {
                        attn_wait<kCols>(x);
                        if (c + kCols < 64) attn_issue<kCols>(tS + c + kCols, next);
                        if constexpr (kNarrow) {
#pragma unroll
                            for (int i = 0; i < kCols; i += 4) {
                                const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(fk + c + i);
                                unpack2(mul2(pack2(x[i], x[i + 1]), k.x), x[i], x[i + 1]);
                                unpack2(mul2(pack2(x[i + 2], x[i + 3]), k.y), x[i + 2], x[i + 3]);
                            }
                        }
                    };
                    float top = -INFINITY;
                    attn_issue<kCols>(tS, ahead[0]);
#pragma unroll
                    for (int c = 0; c < 64; c += kCols) {
                        float (&x)[kCols] = ahead[c / kCols & 1];
                        scores(c, x, ahead[c / kCols + 1 & 1]);
                        float a = -INFINITY, b = -INFINITY;
#pragma unroll
                        for (int i = 0; i < kCols; i += 4) { a = max3(a, x[i], x[i + 1]); b = max3(b, x[i + 2], x[i + 3]); }
                        top = max3(top, a, b);
                    }
                    top = fmaf(top, factor, above);
                    if (vote(!ok || top > ref + kAttnLazy)) {
                        // a new reference for the rows that need one: the larger of the two halves' largest scores
                        S.of_half[t][half][row] = top;
                        if (vote(!ok)) { left = true; break; }
                        const float both = fmaxf(top, S.of_half[t][half ^ 1][row]);
                        const bool raise = both > ref + kAttnLazy;
                        const float by = raise ? ex2_approx(ref - both) : 1.f;
                        if (raise) ref = both;
                        sum *= by;
                        if (any) {
#pragma unroll 1
                            for (int c = o_begin; c < o_end; c += 16) {
                                float o[16];
                                uint32_t w[16];
                                tmem_load16(tO + c, o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * by);
                                tmem_store16(tO + c, w);
                            }
                            tmem_store_wait();
                        }
                        __syncwarp();
                    }
                    any = true;
                    const uint64_t f2 = pack2(factor, factor), b2 = pack2(-ref, -ref);
                    uint64_t s2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    attn_issue<kCols>(tS, ahead[0]);
#pragma unroll
                    for (int c = 0; c < 64; c += kCols) {
                        float (&x)[kCols] = ahead[c / kCols & 1];
                        uint32_t w[kCols / 2];
                        scores(c, x, ahead[c / kCols + 1 & 1]);
#pragma unroll
                        for (int i = 0; i < kCols; i += 4) {
                            float e[4];
                            unpack2(fma2(pack2(x[i], x[i + 1]), f2, b2), e[0], e[1]);
                            unpack2(fma2(pack2(x[i + 2], x[i + 3]), f2, b2), e[2], e[3]);
#pragma unroll
                            for (int k = 0; k < 4; ++k) e[k] = ex2_approx(e[k]);
                            const uint64_t e0 = pack2(e[0], e[1]), e1 = pack2(e[2], e[3]);
                            s2[0] = add2(s2[0], e0);
                            s2[1] = add2(s2[1], e1);
                            if constexpr (kNarrow) {
                                const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(fv + c + i);
                                unpack2(mul2(e0, v.x), e[0], e[1]);
                                unpack2(mul2(e1, v.y), e[2], e[3]);
                            }
                            w[i >> 1] = pack16<kNarrow>(e[0], e[1]);
                            w[(i >> 1) + 1] = pack16<kNarrow>(e[2], e[3]);
                        }
                        attn_write<kCols / 2>(tS + c / 2, w);
                    }
                    float s0, s1;
                    unpack2(add2(s2[0], s2[1]), s0, s1);
                    sum += s0 + s1;
                    tmem_store_wait();
                }
                if (!kNarrow && masked && (!u.pair || t == 0)) {
                    // V of positions that no row sees, or that hold NaN or infinities that only some see, must not meet a
                    // weight of zero in the product: zeros here, the latter added to the rows that see them at the end
                    const uint32_t i = seq + jj, s = P.k_slots + i % P.v_slots;
                    wait(&S.full[s], i / P.v_slots & 1u);
                    if ((row & 1) == half && (row >= u.first - start || row >= valid)) {
                        if (attn_clean_values(ring + (size_t)s * tile_bytes + row * 128, row, P.chunks, row < valid))
                            atomicOr(&S.bad_value[units % kAttnUnitFlags], attn_tile_bit(u.j0 + jj));
                    }
                    fence_async_smem();
                }
                if (merged) {                    // the second group's O of the unit before has been read
                    wait(&S.merge_done, (merges - 1) & 1u);
                    merged = false;
                }
                tc_fence_before();
                arrive(&S.p_full[t]);
            }
            if (!left && jj < count && warp_live) {
                wait(&S.s_full[t], items & 1u);  // O is at rest: these scores were issued behind its last products
                __syncwarp();
                tc_fence_after();
                attn_keep(tO, o_begin, o_end, live ? keep_row(u) : nullptr, stretch < step ? 0.f : ex2_approx(S.kept[t][half][row] - ref), false);
                S.kept[t][half][row] = ref;
                __syncwarp();
            }
            }
            if (left) { ok = false; break; }                                // both warps
            const AttnUnit done = u;
            have = it.next(P, u);
            wait(&S.o_full[t], units & 1u);
            __syncwarp();
            tc_fence_after();
            if (warp_live && (done.pair ? count : (count - t + 1) >> 1) > kAttnKeep) {
                attn_keep(tO, o_begin, o_end, live ? keep_row(done) : nullptr, ex2_approx(S.kept[t][half][row] - ref), true);
                __syncwarp();
            }
            const bool join = !done.pair && count > 1;
            if (merged) { wait(&S.merge_done, (merges - 1) & 1u); merged = false; }
            S.of_half[t][half][row] = sum;
            if (vote(!ok)) { ok = false; break; }
            sum += S.of_half[t][half ^ 1][row];
            if (join && t == 1) {
                if (!half) S.second[row] = make_float2(ref, sum);
                tc_fence_before();
                arrive(&S.merge_ready);
                ++merges;
                merged = true;
            } else if (done.pair || t == 0) {
                float f0 = 1.f, f1 = 0.f;
                if (join) {
                    wait(&S.merge_ready, merges & 1u);
                    ++merges;
                    if (vote(!ok)) { ok = false; break; }
                    tc_fence_after();
                    const float2 o = S.second[row];
                    const float top = fmaxf(ref, o.x);
                    f0 = ex2_approx(ref - top);
                    f1 = ex2_approx(o.x - top);
                    sum = sum * f0 + o.y * f1;
                    ref = top;
                }
                const bool whole = done.j0 == 0 && done.j1 == done.tiles;
                const uint32_t bad_tiles = kKind != kAttnI8 ? *(volatile uint32_t*)&S.bad_value[units % kAttnUnitFlags] : 0u;
                const long long part = (long long)(2 * blockIdx.x + (done.j0 > 0 ? 0 : 1)) * P.part_rows + tile * kAttnTile + row;
                const int head = done.head * P.group + row % P.group;
                const long long out_row = done.row0 + node;
                const float inverse = whole ? 1.f / sum : 1.f;
                if (warp_live) {
                    // 16 components of the warp's rows at a time through this unit's Q, which nobody needs any more: neighbouring
                    // lanes write neighbouring pieces of a row
                    unsigned char* stage = sQ + tile * tile_bytes + (warp & 7) * 2048;
                    unsigned char* to = !live ? nullptr : whole ? P.out + out_row * P.out_row + head * P.out_head : reinterpret_cast<unsigned char*>(P.parts + part * d);
                    auto staged = [&](int r, int piece) { return reinterpret_cast<float4*>(stage + r * 64 + ((piece ^ (r >> 1 & 3)) << 4)); };
                    auto target = [&](int r) { return reinterpret_cast<unsigned char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), r)); };
#pragma unroll 1
                    for (int c = o_begin; c < o_end; c += 16) {
                        float o[16];
                        __syncwarp();
                        tmem_load16(tO + c, o);
                        if (join) {
                            float o1[16];
                            tmem_load16(tO + 128 + c, o1);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = o[i] * f0 + o1[i] * f1;
                        }
                        if (bad_tiles && live) { // values that were left out of the product, where this row sees them
                            float bad[16];
                            attn_bad_row<kNarrow>(P, AttnPart(done), node, attn_straight_of(P, done, S.straight[warp]), bad_tiles, c, bad);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] += bad[i];
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *staged(lane, i) = make_float4(o[4 * i] * inverse, o[4 * i + 1] * inverse, o[4 * i + 2] * inverse, o[4 * i + 3] * inverse);
                        __syncwarp();
                        if (whole) {
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int r = k * 16 + (lane >> 1);
                                unsigned char* at = target(r);
                                const float4 x = *staged(r, (lane & 1) * 2), y = *staged(r, (lane & 1) * 2 + 1);
                                if (at) *reinterpret_cast<uint4*>(at + c * 2 + (lane & 1) * 16) = make_uint4(pack16<false>(x.x, x.y), pack16<false>(x.z, x.w), pack16<false>(y.x, y.y), pack16<false>(y.z, y.w));
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int r = k * 8 + (lane >> 2);
                                unsigned char* at = target(r);
                                const float4 x = *staged(r, lane & 3);
                                if (at) *reinterpret_cast<float4*>(at + c * 4 + (lane & 3) * 16) = x;
                            }
                        }
                    }
                    if (live && !half) {
                        if (!whole) P.part_stats[part] = make_float2(ref, sum);
                        else if (P.out_lse) P.out_lse[out_row * P.q_heads + head] = (ref + log2f(sum)) * 0.6931471805599453f;
                    }
                }
                __syncwarp();
                if (join) { tc_fence_before(); arrive(&S.merge_done); }
            }
            // Q of the next unit: everything of this one has been multiplied, and this group has written what it had to
            if (have) prepare_q(u);
            seq += count;
            ++units;
        }
        if (!ok) give_up();
    } else {
        // ---------------- 8-bit tiles to 16 bits --------------------------------------------------------------
        if constexpr (kNarrow) {
            const int ct = tid - (kRowWarps + 2) * 32;
            // scales of position ct of a tile
            float k_now = 0.f, v_now = 0.f;
            bool node = false, exists = false;
            auto load_scales = [&](const AttnUnit& w, int j) {
                int start, len;
                attn_tile_at(P, j, start, len);
                k_now = v_now = 0.f;
                node = ct >= w.first - start;
                exists = ct < min(kAttnTile, min(len, w.length - start));
                if (!exists) return;
                const int position = start + ct, page_of = attn_page_of(P, position), token = position - page_of * P.c.page_size;
                const int page = P.c.block_table[w.r * P.c.table_stride + page_of];
                if (page < 0 || page >= P.c.n_pages) return;
                const long long at = ((long long)page * P.c.kv_heads + w.head) * P.c.page_size + token;
                k_now = P.c.k_scale[at];
                v_now = P.c.v_scale[at];
            };
            auto store_scales = [&](int number) {
                // free: the scores of tile number - 2 are not computed before the weights of tile number - 4 are there
                if (ct >= kAttnTile) return;
                const int at = number % kAttnScaleTiles;
                const bool bad = node && !(fabsf(k_now) < INFINITY && fabsf(v_now) < INFINITY);     // NaN for the rows that see it
                const float k = k_now * P.score_factor;
                const bool odd = exists && node && (bad || !(k > 0.f));
                scales.k[at][ct] = odd || !exists ? 1.f : k;
                scales.odd_k[at][ct] = bad ? NAN : k;
                scales.v[at][ct] = bad ? 0.f : v_now;
                const uint32_t bits = __ballot_sync(0xffffffffu, odd);
                if (lane == 0) scales.odd[at][ct >> 5] = bits;
            };
            if (!attn_widen<kKind, kAttnConverters * 32, false>(P, it, ct, 0, 1, raw, ring, tile_bytes, S.raw_full, S.raw_empty, S.full, S.empty, 0u, S.bad_value, abort_flag, load_scales,
                                        store_scales) && lane == 0)
                give_up();
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
// A row's references and sums first, then the weighted sum of its parts' accumulators, in the order of the CTAs.  Where there are
// many units each has few parts: a warp a row, and blockIdx.x is the CTA whose end divided the unit.  Where there are few, a unit can
// have a part of every SM: all warps of a CTA for a row, and blockIdx.x counts the divided units.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <int kWarps>                            // of a row
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams P, int ctas)
{
    __shared__ int s_count[kJoinWarps], s_cta;
    __shared__ __align__(16) float s_o[kWarps][kAttnMaxDim];
    __shared__ float s_sum[kWarps];
    static_assert(kAttnSms <= kJoinThreads, "a cut a thread");
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int b = blockIdx.x;
    if constexpr (kWarps > 1) {
        const bool some = tid < ctas && P.cuts[tid].x != 0;
        const uint32_t all = __ballot_sync(0xffffffffu, some);
        if (lane == 0) s_count[warp] = __popc(all);
        if (tid == 0) s_cta = -1;
        __syncthreads();
        int before = 0;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) before += w < warp ? s_count[w] : 0;
        if (some && before + __popc(all & ((1u << lane) - 1u)) == (int)blockIdx.x) s_cta = tid;
        __syncthreads();
        b = s_cta;
        if (b < 0) return;
    }
    const int4 cut = P.cuts[b];
    const int d = P.c.head_dim, tile_rows = P.tile_nodes * P.group, i = kWarps > 1 ? blockIdx.y : blockIdx.y * kJoinWarps + warp;
    if (cut.x == 0 || i >= cut.w * P.group) return;
    const int node = i / P.group, parts = cut.y - b + 2, at = lane * 4;
    const int row = i < tile_rows ? i : kAttnTile + i - tile_rows;           // its place in a partial result
    auto place = [&](int k) { return (long long)(k == 0 ? 2 * (b - 1) + 1 : 2 * (b - 1 + k)) * P.part_rows + row; };
    const int k_first = kWarps > 1 ? warp : 0;
    constexpr int kBatch = 4;
    float4 x[kBatch];
    float2 s[kBatch];
    auto ask = [&](int k0) {
#pragma unroll
        for (int m = 0; m < kBatch; ++m) {
            const int k = k0 + m * kWarps;
            x[m] = make_float4(0.f, 0.f, 0.f, 0.f);
            s[m] = make_float2(-INFINITY, 0.f);
            if (k >= parts) continue;
            s[m] = P.part_stats[place(k)];
            if (at < d) x[m] = *reinterpret_cast<const float4*>(P.parts + place(k) * d + at);
        }
    };
    ask(k_first);
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 32) top = fmaxf(top, P.part_stats[place(k)].x);
    top = warp_max_f32(top);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = k_first; k0 < parts; k0 += kBatch * kWarps) {
        if (k0 != k_first) ask(k0);
#pragma unroll
        for (int m = 0; m < kBatch; ++m) {
            if (k0 + m * kWarps >= parts) continue;
            const float g = ex2_approx(s[m].x - base);
            sum = fmaf(s[m].y, g, sum);
            o[0] = fmaf(x[m].x, g, o[0]); o[1] = fmaf(x[m].y, g, o[1]);
            o[2] = fmaf(x[m].z, g, o[2]); o[3] = fmaf(x[m].w, g, o[3]);
        }
    }
    if constexpr (kWarps > 1) {
        if (at < d) *reinterpret_cast<float4*>(&s_o[warp][at]) = make_float4(o[0], o[1], o[2], o[3]);
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        if (warp != 0) return;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            sum += s_sum[w];
            if (at < d)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[c] += s_o[w][at + c];
        }
    }
    const float inverse = 1.f / sum;
    const int head = (cut.x - 1) * P.group + i % P.group;
    const long long out_row = cut.z + node;
    if (at < d)
        *reinterpret_cast<uint2*>(P.out + out_row * P.out_row + head * P.out_head + lane * 8) =
            make_uint2(pack16<false>(o[0] * inverse, o[1] * inverse), pack16<false>(o[2] * inverse, o[3] * inverse));
    if (P.out_lse && lane == 0) P.out_lse[out_row * P.q_heads + head] = (top + log2f(sum)) * 0.6931471805599453f;
}

// ---- host side -------------------------------------------------------------------------------------------
// One K/V array of a layer as [page][head][token][d]; a box is `tokens` positions of one head of a page.
// `turned`: 8-bit lines of 64 and 128 bytes are swizzled too (widen_line).
static bool cache_map(CUtensorMap* map, const unsigned char* base, const KvView& c, int tokens, bool turned)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const bool wide = c.dtype == DSPARK_BF16;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.kv_heads, (cuuint64_t)c.n_pages};
    auto step = [](long long s) { return (cuuint64_t)(s > 16 ? s : 16); };  // of a single entry: any
    const cuuint64_t strides[3] = {step(c.token_stride), step(c.head_stride), step(c.page_stride)};
    const cuuint32_t box[4] = {(cuuint32_t)(wide ? 64 : c.head_dim), (cuuint32_t)tokens, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    // What the copies bring into the L2 beside their own lines is another head's, and gone before that head's turn, unless a head's
    // positions lie together: 64 tokens over 8192 positions of int8, 128 bytes a line, read 1.66 GB instead of 1.11 when 256 bytes
    // were brought at a time.
    const long long line = c.token_stride == (long long)c.head_dim * (wide ? 2 : 1) ? 256 : c.head_dim * (wide ? 2 : 1);
    const CUtensorMapL2promotion promotion = line >= 256 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : line >= 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B
                                             : line >= 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_64B : CU_TENSOR_MAP_L2_PROMOTION_NONE;
    return fn(map, wide ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<unsigned char*>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, wide || (turned && c.head_dim == 128) ? CU_TENSOR_MAP_SWIZZLE_128B : turned && c.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
              promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static int attn_sms() { const int sms = current_sms(); return sms < kAttnSms ? sms : kAttnSms; }
struct AttnWs { size_t stats, parts, total; int rows; };
static AttnWs attn_ws(long long n_rows, int group, int d)
{
    AttnWs w;
    const long long rows = n_rows * group;
    w.rows = rows <= 64 ? (int)rows : 2 * kAttnTile;         // more: the kernel for many rows has two accumulators to put by
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
    if (!attn_allow_smem(attn_kernel<kKind>, kSmem, ready)) return launch_status();
    const int tile = P.chunks * kChunkBytes;
    // 8-bit: four 16-bit tiles beside one of Q, three beside two; the rest for 8-bit ones
    int slots = kNarrow ? (P.q_tiles == 1 ? 4 : 3) : kAttnRingBytes / tile - P.q_tiles;
    if (slots > kAttnMaxSlots) slots = kAttnMaxSlots;
    P.k_slots = slots / 2;
    P.v_slots = slots - P.k_slots;
    const int raw = (kAttnNarrowBytes - (P.q_tiles + slots) * tile) / (kAttnTile * P.c.head_dim), most = raw < kAttnMaxRaw ? raw : kAttnMaxRaw;
    P.raw_k = kNarrow ? most / 2 : 0;
    P.raw_v = kNarrow ? most - P.raw_k : 0;
    KernelTimerScope timer(DSPARK_K_TREE_ATTENTION, s);
    launch_pdl(attn_kernel<kKind>, dim3((unsigned)sms), dim3(kAttnThreads<kKind>), kSmem, s, P, k, v);
    return launch_status();
}

}  // namespace dspark

// Polls of a wait by device, 0 standing for kWaitPollLimit (dspark_set_wait_poll_limit).  The waits for copies and products under
// way before a CTA leaves keep their own.
static std::atomic<uint32_t> g_attn_poll_limit[64];
namespace dspark {
void attn_set_poll_limit(uint32_t polls)
{
    int dev = 0;
    cudaGetDevice(&dev);
    g_attn_poll_limit[dev & 63].store(polls ^ kWaitPollLimit, std::memory_order_relaxed);
}
static uint32_t attn_poll_limit()
{
    int dev = 0;
    cudaGetDevice(&dev);
    const uint32_t polls = g_attn_poll_limit[dev & 63].load(std::memory_order_relaxed) ^ kWaitPollLimit;
    return polls < kAttnPolls ? polls : kAttnPolls;
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
    if (!q || !out || q_heads < 1 || !(fabsf(scale) <= 0x1p127f)) return DSPARK_ERR_INVALID_ARG;
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
    if (cache->dtype == DSPARK_BF16 && P.score_factor == 0.f) P.score_factor = kAttnLeastFactor;
    P.q_sign = scale < 0.f ? 0x80008000u : 0u;
    P.dev_status = dev_status;
    // rows of a request with one K/V head on average
    const long long rows = (long long)((n_rows + R - 1) / R) * P.group;
    const bool few = rows <= 64;
    // two row tiles a unit where one does not hold a request's rows: their cache tiles are then read once
    P.q_tiles = rows > kAttnTile ? 2 : 1;
    P.tile_nodes = (few ? (rows <= 16 ? 16 : rows <= 32 ? 32 : 64) : kAttnTile) / P.group;
    P.unit_nodes = P.tile_nodes * P.q_tiles;
    P.chunks = d > 64 ? 2 : 1;
    P.tile_tokens = cache->page_size < kAttnTile ? cache->page_size : kAttnTile;
    P.page_boxes = kAttnTile / P.tile_tokens;
    P.page_tiles = (cache->page_size + kAttnTile - 1) / kAttnTile;
    P.page_shift = -1;
    for (int i = 3; i <= 7; ++i) if (cache->page_size == 1 << i) P.page_shift = i;
    P.part_rows = w.rows;
    P.polls = attn_poll_limit();
    unsigned char* ws = (unsigned char*)workspace;
    P.cuts = (int4*)ws;
    P.part_stats = (float2*)(ws + w.stats);
    P.parts = (float*)(ws + w.parts);
    CUtensorMap map_k, map_v;
    if (!cache_map(&map_k, P.c.k, P.c, P.tile_tokens, few) || !cache_map(&map_v, P.c.v, P.c, P.tile_tokens, false)) return DSPARK_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int sms = attn_sms();
    int rc;
    if (few) rc = attn_few_launch(P, (int)rows, map_k, map_v, sms, s);
    else if (cache->dtype == DSPARK_BF16) rc = attn_launch<kAttnWide>(P, map_k, map_v, sms, s);
    else if (cache->dtype == DSPARK_I8) rc = attn_launch<kAttnI8>(P, map_k, map_v, sms, s);
    else rc = attn_launch<kAttnE4M3>(P, map_k, map_v, sms, s);
    if (rc) return rc;
    KernelTimerScope timer(DSPARK_K_TREE_COMBINE, s);
    // at most this many units, one of n_rows / unit_nodes whole ones or the last of a request for each K/V head
    const long long units = ((long long)n_rows / P.unit_nodes + R) * cache->kv_heads;
    const int join_rows = (n_rows < P.unit_nodes ? n_rows : P.unit_nodes) * P.group;
    // (one unit of 16 rows over 20000 positions: 18.7 us with a CTA a row for both kernels, 34 with a warp; 8 units of 256 rows: a CTA a
    // row would be 2048 of them, 257.6 us instead of 253.5)
    if (units * 8 <= sms && units * join_rows <= 8 * sms) launch_pdl(attn_join_kernel<kJoinWarps>, dim3((unsigned)units, (unsigned)join_rows), dim3(kJoinThreads), 0, s, P, sms);
    else launch_pdl(attn_join_kernel<1>, dim3((unsigned)sms, (unsigned)((join_rows + kJoinWarps - 1) / kJoinWarps)), dim3(kJoinThreads), 0, s, P, sms);
    return launch_status();
}

}  // extern "C"
