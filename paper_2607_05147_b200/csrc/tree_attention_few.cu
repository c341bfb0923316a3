// dspark_tree_attention for requests whose nodes make few rows with a K/V head (up to 64): single tokens, short drafts, trees.
//
// The products are turned round: S^T = K Q^T and O^T = V^T P^T, so that the 128 positions of a cache tile are the 128 rows of the
// tensor cores' tile and the rows of Q are its columns.  With rows as lanes, 8 rows of one decoding token would leave 120 of 128
// threads idle in a softmax of 128 exponentials a thread; here every thread has one position and 16 to 64 exponentials, and what
// belongs to a position (its scales in an 8-bit cache, whether it exists) belongs to a thread.
//
//   * S^T = K Q^T: K as it lies (k-major), Q in shared memory, N = rows rounded up to 16, 32 or 64;
//   * a thread reads its position's N scores, weighs them against one reference a row and writes N 16-bit weights, one line of the
//     mn-major operand P^T, to shared memory;
//   * O^T += V^T P^T: V as it lies (mn-major), O^T has a row per component and a column per row of Q.
// The maximum of a row would need a reduction over the threads for every row and tile.  It is not needed: any reference serves
// that keeps the exponentials in range, so the threads only vote whether one of their scores is above its reference by more than
// 2^8; then, seldom, the maxima are found, and O^T and the sums scaled.  The sums of the weights stay in the threads until the
// end of a unit.
//
// Two groups of four warps take the even and the odd tiles of a unit, as in the kernel for many rows, and join at its end.
// Bound by the cache's bytes.
#include <math.h>

#include "tree_attention.cuh"

namespace dspark {

constexpr int kFewSmem = 217 * 1024;             // Q, two of P, the ring; tables beside it
constexpr int kFewPBytes = kAttnTile * 128;      // P^T of one group: a line of 128 bytes a position
constexpr float kFewUnset = 1e38f;               // less a reference that every score is above

struct FewShared {
    uint64_t full[kAttnMaxSlots], empty[kAttnMaxSlots], raw_full[kAttnMaxRaw], raw_empty[kAttnMaxRaw];
    uint64_t q_full, q_empty, s_full[2], p_full[2], o_done[2], merge_ready, merge_done, mma_done[2];
    uint32_t tmem_base;
    int abort, bad_value[kAttnUnitFlags];
    AttnList list;
};
template <int kN>
struct FewTables {
    float less[2][kN];                           // less the references, in units of log2, of each group
    float last[kN];                              // those of the second group at the end of a unit
    float scale[2][kN];                          // what O^T and the sums are multiplied by when they change; joining: weights
    float q[2][kN];                              // 8-bit caches: what a row of Q was divided by, of this unit and the next
    float top[2][4][kN], sum[2][4][kN];          // a warp's maxima; its sums at the end
    unsigned long long seen[2][kAttnTile];       // rows that see a position (tiles with nodes)
};

__device__ __forceinline__ bool group_any(int group, bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "r"(group + 1) : "memory");
    return r != 0;
}
__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(group + 1) : "memory"); }
template <int kCols> __device__ __forceinline__ void tmem_read(uint32_t addr, float (&v)[kCols])
{
    if constexpr (kCols == 16) tmem_load16(addr, v);
    else { tmem_load32_issue(addr, v); tmem_load_wait(v); }
}

template <int kKind> constexpr int kFewConverters = kKind == kAttnWide ? 0 : 4;
template <int kKind> constexpr int kFewThreads = (kSoftmaxWarps + 3 + kFewConverters<kKind>) * 32;

template <int kKind, int kN>
__global__ void __launch_bounds__(kFewThreads<kKind>, 1)
attn_few_kernel(const __grid_constant__ AttnParams P, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    constexpr bool kNarrow = kKind != kAttnWide;
    constexpr int kThreads = kFewThreads<kKind>, kProducer = kSoftmaxWarps, kIssuer = kSoftmaxWarps + 1, kIssuerO = kSoftmaxWarps + 2;
    constexpr int kWarps = kFewConverters<kKind>, kCols = kN < 32 || (kNarrow && kN == 64) ? 16 : 32;
    constexpr bool kKeep = kN <= 32; // a tile's scores stay in registers between the vote and the exponentials
    constexpr int kParts = kKeep ? kN / kCols : 1;
    constexpr uint32_t kO = 128;                 // columns of tensor memory: S^T at 0 and 64, O^T at 128 and 192
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzle atoms: 1 KB
    __shared__ FewShared S;
    __shared__ __align__(16) FewTables<kN> T;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;    // warp: uniform, and known to be
    const int d = P.c.head_dim, tile_bytes = P.chunks * kChunkBytes;
    unsigned char* sP = smem;
    unsigned char* sQ = sP + 2 * kFewPBytes;     // per 64 components: kN lines of 128 bytes
    unsigned char* ring = sQ + P.chunks * kN * 128;
    unsigned char* raw = ring + P.slots * tile_bytes;

    if (tid == 0) {
        for (int s = 0; s < P.slots; ++s) { mbar_init(&S.full[s], kNarrow ? kWarps : 1); mbar_init(&S.empty[s], 1); }
        for (int s = 0; s < P.raw_slots; ++s) { mbar_init(&S.raw_full[s], 1); mbar_init(&S.raw_empty[s], kNarrow ? kWarps : 1); }
        mbar_init(&S.q_full, 4); mbar_init(&S.q_empty, 1);
        for (int t = 0; t < 2; ++t) { mbar_init(&S.s_full[t], 1); mbar_init(&S.p_full[t], 4); mbar_init(&S.o_done[t], 1); mbar_init(&S.mma_done[t], 1); }
        for (int i = 0; i < kAttnUnitFlags; ++i) S.bad_value[i] = 0;
        mbar_init(&S.merge_ready, 4); mbar_init(&S.merge_done, 4);
        S.abort = 0;
        mbar_fence_init();
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(256) : "memory");
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
                              kNarrow ? P.raw_slots : P.slots, abort_flag);
    } else if (warp == kIssuer || warp == kIssuerO) {
        // ---------------- products --------------------------------------------------------------------------
        // One warp issues S^T = K Q^T, another O^T += V^T P^T: what a single one has to wait for and to issue for a tile takes it
        // longer than the tile's bytes take to arrive.  K and V tiles alternate in the ring.
        const bool second = warp == kIssuerO;
        const uint32_t type = kNarrow ? 0u : 1u;                            // fp16 or bf16 operands, fp32 sums
        const uint32_t idesc_s = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(kAttnTile >> 4) << 24);
        const uint32_t idesc_o = idesc_s | (1u << 15) | (1u << 16);
        const uint32_t tile_step = (uint32_t)tile_bytes >> 4;
        uint32_t units = 0, items[2] = {0, 0}, s = second ? 1 : 0, ph = 0;
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t p) { ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, p)); return ok; };
        while (ok && !__any_sync(0xffffffffu, *abort_flag) && it.next(P, u)) {
            const int n = u.j1 - u.j0;
            const uint32_t turn = units & 1u;                               // the group that has the even tiles
            if (!second && !wait(&S.q_full, units & 1u)) break;
            ++units;
            for (int i = 0; i < n; ++i) {
                const uint32_t t = turn ^ (uint32_t)(i & 1), item = t ? items[1]++ : items[0]++;
                if (second) {
                    if (!wait(&S.full[s], ph) || !wait(&S.p_full[t], item & 1u)) break;
                    tc_fence_after();
                    const uint32_t a = desc_mn_major(smem_u32(ring)) + s * tile_step, b = desc_mn_major(smem_u32(sP)) + t * (kFewPBytes >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kAttnTile / 16; ++k) mma_ss(tmem + kO + t * 64, a + k * 128, b + k * 128, idesc_o, i > 1 || k > 0);
                        umma_commit(&S.empty[s]);
                        umma_commit(&S.o_done[t]);
                    }
                } else {
                    // the scores that were here before have been read
                    if ((item && !wait(&S.p_full[t], (item - 1) & 1u)) || !wait(&S.full[s], ph)) break;
                    tc_fence_after();
                    const uint32_t a = desc_k_major(smem_u32(ring)) + s * tile_step, b = desc_k_major(smem_u32(sQ));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kAttnMaxDim / 16; ++k)
                            if (k < d / 16)
                                mma_ss(tmem + t * 64, a + (k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2, b + (k >> 2) * (kN * 8) + (k & 3) * 2, idesc_s, k > 0);
                        umma_commit(&S.s_full[t]);
                        umma_commit(&S.empty[s]);
                        if (i + 1 == n) umma_commit(&S.q_empty);
                    }
                }
                __syncwarp();
                s += 2;
                if (s >= (uint32_t)P.slots) { s -= P.slots; ph ^= 1u; }
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
        // The group that has a unit's odd tiles brings the next unit's Q and has that one's even tiles, so that it begins with it
        // while the other group writes the results.  A wait that runs out makes `ok` false in its warp; the threads of a group leave
        // together, at the next vote.
        const int t = warp >> 2, pos = tid & 127;                           // group; position in a tile, later component
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_base + t * 64, tO = tmem + lane_base + kO + t * 64, tOther = tmem + lane_base + kO + (t ^ 1) * 64;
        unsigned char* p_line = sP + t * kFewPBytes + pos * 128;
        uint32_t units = 0, items = 0, merges = 0, seq = 0;                 // seq: tiles of the ring used by earlier units
        bool ok = true, merged = false;
        auto wait = [&](uint64_t* bar, uint32_t ph) { ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, ph)); };
        auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
        // Q of a unit: 128 / kN threads a row, asked for and later stored.
        constexpr int kPer = 128 / kN, kMost = (kAttnMaxDim / 8 + kPer - 1) / kPer;
        uint4 x[kMost];
        auto fetch_q = [&](const AttnUnit& w) {
            const int row = pos / kPer, sub = pos % kPer, node = w.node0 + row / P.group, pieces = d / 8;
            const bool live = row < P.tile_nodes * P.group && node < w.n;
            const uint4* src = reinterpret_cast<const uint4*>(P.q + (long long)(w.row0 + node) * P.q_row +
                                                              (long long)(w.head * P.group + row % P.group) * P.q_head);
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                x[i] = make_uint4(0, 0, 0, 0);
                if (live && i * kPer + sub < pieces) x[i] = src[i * kPer + sub];
            }
        };
        // With an 8-bit cache as fp16, scaled by a power of two so that no value passes the range and what is lost is below 2^-37
        // of the row's largest.
        auto store_q = [&](uint32_t unit) {
            const int row = pos / kPer, sub = pos % kPer, pieces = d / 8;
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
                // 2^e with the largest value below 2^14: exponent field of top to that of 2^13; at most 2^60
                const int e = min(127 + 60, max(1, 254 + 13 - (int)(__float_as_uint(top) >> 23)));
                const float up = __uint_as_float((uint32_t)e << 23);
                if (sub == 0) T.q[unit & 1u][row] = __uint_as_float((uint32_t)(254 - e) << 23);
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
                const int c = i * kPer + sub;
                x[i].x ^= P.q_sign; x[i].y ^= P.q_sign; x[i].z ^= P.q_sign; x[i].w ^= P.q_sign;
                if (c < pieces) *reinterpret_cast<uint4*>(sQ + (c >> 3) * (kN * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = x[i];
            }
            fence_async_smem();
            arrive(&S.q_full);
        };
        // An 8-bit cache's scales of this thread's position, asked for one tile of the group ahead, their page two ahead.
        struct Ahead { int page, token; };
        auto page_of = [&](const AttnUnit& w, int jj) {
            Ahead a = {-1, 0};
            if (kNarrow && w.j0 + jj < w.j1) {
                int start, len;
                attn_tile_at(P, w.j0 + jj, start, len);
                if (pos < min(len, w.length - start)) {
                    const int position = start + pos, page = position / P.c.page_size;
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
        bool have = it.next(P, u);
        Ahead ahead = {-1, 0};
        float2 scale_next = make_float2(0.f, 0.f);
        auto first_scales = [&](int at) {
            scale_next = scales_of(u, page_of(u, at));
            ahead = page_of(u, at + 2);
        };
        if (have) {
            if (t == 1) { fetch_q(u); store_q(0); }
            first_scales(t);
        }
        while (have) {
            const int turn = t ^ (int)(units & 1u);                         // 0: this group has the even tiles
            if (pos < kN) T.less[t][pos] = kFewUnset;
            if (tid == 0) S.bad_value[(units + kAttnUnitFlags / 2) % kAttnUnitFlags] = 0;
            if (group_any(t, !ok || *abort_flag)) { ok = false; break; }
            uint64_t sums[kN / 2];                                          // of this position's weights, two rows each
#pragma unroll
            for (int c = 0; c < kN / 2; ++c) sums[c] = pack2(0.f, 0.f);
            const int count = u.j1 - u.j0;
            bool any = false, left = false;
            for (int jj = turn; jj < count; jj += 2) {
                int start, len;
                attn_tile_at(P, u.j0 + jj, start, len);
                const int valid = min(len, u.length - start);               // positions of this tile that exist
                const bool masked = start + kAttnTile > u.first || valid < kAttnTile;
                // rows that see this thread's position, a bit each
                unsigned long long seen = ~0ull;
                if (masked) {
                    const int node = start + pos - u.first;                 // the node at this position
                    if (pos >= valid) seen = 0;
                    else if (node >= 0 && !P.parents) {
                        const int shift = (node - u.node0) * P.group;
                        seen = shift <= 0 ? ~0ull : shift >= 64 ? 0 : ~0ull << shift;
                    }
                    if (P.parents && start + valid > u.first) {
                        T.seen[t][pos] = 0;
                        group_sync(t);
                        const int self = u.node0 + pos;
                        if (pos < P.tile_nodes && self < u.n) {
                            const unsigned long long rows = (P.group == 64 ? ~0ull : (1ull << P.group) - 1) << (pos * P.group);
                            int a = self;
                            for (;;) {
                                const int at = u.first + a - start;
                                if (at < 0) break;
                                if (at < valid) atomicOr(&T.seen[t][at], rows);
                                if (a == 0) break;
                                const int p = P.parents[u.row0 + a];
                                if (p < 0 || p >= a) { atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE); break; }
                                a = p;
                            }
                        }
                        group_sync(t);
                        if (node >= 0 && pos < valid) seen = T.seen[t][pos];
                    }
                }
                const float2 scale = scale_next;
                scale_next = scales_of(u, ahead);
                ahead = page_of(u, jj + 4);
                float k_scale = P.score_factor, v_scale = scale.y;
                // an 8-bit V: 2^exponent > its scale; what a weight may be above its reference depends on it
                float above = 0.f;
                if constexpr (kNarrow) {
                    k_scale *= scale.x;
                    if (k_scale < kAttnLeastFactor) k_scale = kAttnLeastFactor;
                    above = attn_exponent(scale.y < INFINITY ? fmaxf(scale.y, 0.f) : 0.f) - kAttnNarrowOffset;
                }
                if (items) wait(&S.o_done[t], (items - 1) & 1u);            // P and O^T of the tile before
                wait(&S.s_full[t], items & 1u);
                ++items;
                tc_fence_after();
                if (masked) {
                    // scores of rows that do not see the position: -infinity, in place.  Where a scale is no number the position
                    // is NaN for the rows that see it, and the scales are not used.
                    const bool bad = kNarrow && !(fabsf(scale.x) < INFINITY && fabsf(scale.y) < INFINITY);
#pragma unroll 1
                    for (int c0 = 0; c0 < kN; c0 += 16) {
                        float s[16];
                        uint32_t w[16];
                        tmem_load16(tS + c0, s);
#pragma unroll
                        for (int c = 0; c < 16; ++c) w[c] = __float_as_uint(!(seen >> (c0 + c) & 1) ? -INFINITY : bad ? NAN : s[c]);
                        tmem_store16(tS + c0, w);
                    }
                    tmem_store_wait();
                    if (bad) { k_scale = 1.f; v_scale = 0.f; above = -kAttnNarrowOffset; }
                }
                const uint64_t k2 = pack2(k_scale, k_scale);
                // y = score * factor - reference for the columns from c0 on, in place
                auto relative = [&](float (&s)[kCols], int c0) {
#pragma unroll
                    for (int c = 0; c < kCols; c += 2) {
                        uint64_t k = k2;
                        if constexpr (kNarrow) k = mul2(k, *reinterpret_cast<const uint64_t*>(&T.q[units & 1u][c0 + c]));
                        unpack2(fma2(pack2(s[c], s[c + 1]), k, *reinterpret_cast<const uint64_t*>(&T.less[t][c0 + c])), s[c], s[c + 1]);
                    }
                };
                float y[kParts][kCols];
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int h = 0; h < kN / kCols; ++h) {
                    float (&s)[kCols] = y[kKeep ? h : 0];
                    tmem_read(tS + h * kCols, s);
                    relative(s, h * kCols);
#pragma unroll
                    for (int c = 0; c < kCols; c += 2) tops[c / 2 % 4] = fmaxf(tops[c / 2 % 4], fmaxf(s[c], s[c + 1]));
                }
                const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                if (group_any(t, !ok || top + above > kAttnLazy)) {
                    // references: the largest score of each row in this tile, where it is that much above
                    if (group_any(t, !ok)) { left = true; break; }
#pragma unroll 1
                    for (int c0 = 0; c0 < kN; c0 += 16) {
                        float s[16], mine = -INFINITY;
                        tmem_load16(tS + c0, s);
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            float z = s[c] * (kNarrow ? k_scale * T.q[units & 1u][c0 + c] : k_scale) + above;
                            z = warp_max_f32(z);
                            if (lane == c) mine = z;
                        }
                        if (lane < 16) T.top[t][warp & 3][c0 + lane] = mine;
                    }
                    group_sync(t);
                    if (pos < kN) {
                        const float old = -T.less[t][pos];
                        const float now = fmaxf(fmaxf(T.top[t][0][pos], T.top[t][1][pos]), fmaxf(T.top[t][2][pos], T.top[t][3][pos]));
                        const bool raise = now > old + kAttnLazy;
                        T.scale[t][pos] = raise ? ex2_approx(old - now) : 1.f;
                        if (raise) T.less[t][pos] = -now;
                    }
                    group_sync(t);
#pragma unroll
                    for (int c = 0; c < kN / 2; ++c) sums[c] = mul2(sums[c], *reinterpret_cast<const uint64_t*>(&T.scale[t][2 * c]));
                    if (any) {
#pragma unroll 1
                        for (int c0 = 0; c0 < kN; c0 += 16) {
                            float o[16];
                            uint32_t w[16];
                            tmem_load16(tO + c0, o);
#pragma unroll
                            for (int c = 0; c < 16; ++c) w[c] = __float_as_uint(o[c] * T.scale[t][c0 + c]);
                            tmem_store16(tO + c0, w);
                        }
                        tmem_store_wait();
                    }
                    if (kKeep)
#pragma unroll
                        for (int h = 0; h < kN / kCols; ++h) {
                            tmem_read(tS + h * kCols, y[kKeep ? h : 0]);
                            relative(y[kKeep ? h : 0], h * kCols);
                        }
                }
                any = true;
#pragma unroll
                for (int h = 0; h < kN / kCols; ++h) {
                    float (&s)[kCols] = y[kKeep ? h : 0];
                    if (!kKeep) {
                        tmem_read(tS + h * kCols, s);
                        relative(s, h * kCols);
                    }
                    uint32_t w[kCols / 2];
#pragma unroll
                    for (int c = 0; c < kCols; c += 2) {
                        float e0 = ex2_approx(s[c]), e1 = ex2_approx(s[c + 1]);
                        const uint64_t e = pack2(e0, e1);
                        sums[(h * kCols + c) / 2] = add2(sums[(h * kCols + c) / 2], e);
                        if constexpr (kNarrow) {
                            unpack2(mul2(e, pack2(v_scale, v_scale)), e0, e1);
                        }
                        w[c / 2] = pack16<kNarrow>(e0, e1);
                    }
#pragma unroll
                    for (int c = 0; c < kCols / 8; ++c)
                        *reinterpret_cast<uint4*>(p_line + (((h * kCols / 8 + c) ^ (pos & 7)) << 4)) =
                            make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                }
                if (!kNarrow && masked) {
                    // V of positions that no row sees, or that hold NaN or infinities that only some see, must not meet a
                    // weight of zero in the product: zeros here, the latter added to the rows that see them at the end
                    const uint32_t i = seq + 2 * jj + 1, s = i % P.slots;
                    wait(&S.full[s], i / P.slots & 1u);
                    if (start + pos >= u.first || pos >= valid)
                        if (attn_clean_values(ring + (size_t)s * tile_bytes + pos * 128, pos, P.chunks, pos < valid))
                            S.bad_value[units % kAttnUnitFlags] = 1;
                }
                fence_async_smem();
                if (merged) {                    // this group's O^T of the unit before has been read
                    wait(&S.merge_done, (merges - 1) & 1u);
                    merged = false;
                }
                tc_fence_before();
                arrive(&S.p_full[t]);
            }
            if (left) { ok = false; break; }                                // all of the group
            // The next unit's Q and scales, asked for while the products of this one are finished.
            const AttnUnit done = u;
            have = it.next(P, u);
            if (have) {
                if (turn == 1) fetch_q(u);
                first_scales(turn ^ 1);
            }
            const bool join = count > 1;
            if (turn == 0 || join) {
                // sums over the positions of this warp: half of the rows pass to the other half of the lanes, five times
                float v[kN];
#pragma unroll
                for (int c = 0; c < kN / 2; ++c) unpack2(sums[c], v[2 * c], v[2 * c + 1]);
                int rows = kN;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    if (rows > 1) {
                        rows >>= 1;
#pragma unroll
                        for (int c = 0; c < kN / 2; ++c)
                            if (c < rows) {
                                const float give = (lane & o) ? v[c] : v[c + rows], keep = (lane & o) ? v[c + rows] : v[c];
                                v[c] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                            }
                    } else
                        v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                }
                // lane bits 4, 3, .. chose the upper half of what was left
                constexpr int kLeft = kN >= 32 ? kN / 32 : 1, kSteps = kN >= 32 ? 5 : 4;
                int row = 0;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) row += (lane >> (4 - i) & 1) * (kN >> (i + 1));
                if (kN >= 32 || (lane & 1) == 0)
#pragma unroll
                    for (int c = 0; c < kLeft; ++c) T.sum[t][warp & 3][row + c] = v[c];
            }
            if (turn == 0 || join) wait(&S.o_done[t], (items - 1) & 1u);
            tc_fence_after();
            if (turn == 1) {
                if (have) {                      // Q takes the place of this unit's, which has been multiplied
                    wait(&S.q_empty, units & 1u);
                    store_q(units + 1);
                }
                if (join) {
                    if (pos < kN) T.last[pos] = -T.less[t][pos];
                    tc_fence_before();
                    arrive(&S.merge_ready);
                    ++merges;
                    merged = true;
                }
            } else {
                if (join) { wait(&S.merge_ready, merges & 1u); ++merges; tc_fence_after(); }
                if (group_any(t, !ok)) { ok = false; break; }
                const bool whole = done.j0 == 0 && done.j1 == done.tiles;
                const long long part = (long long)(2 * blockIdx.x + (done.j0 > 0 ? 0 : 1)) * P.part_rows;
                const int rows = min(P.tile_nodes, done.n - done.node0) * P.group;
                if (pos < rows) {
                    float base = -T.less[t][pos], f0 = 1.f, f1 = 0.f;
                    float sum = (T.sum[t][0][pos] + T.sum[t][1][pos]) + (T.sum[t][2][pos] + T.sum[t][3][pos]);
                    if (join) {
                        const float base1 = T.last[pos], both = fmaxf(base, base1);
                        f0 = ex2_approx(base - both);
                        f1 = ex2_approx(base1 - both);
                        const float (&other)[4][kN] = T.sum[t ^ 1];
                        sum = sum * f0 + ((other[0][pos] + other[1][pos]) + (other[2][pos] + other[3][pos])) * f1;
                        base = both;
                    }
                    if (whole) {
                        const float inverse = 1.f / sum;
                        f0 *= inverse;
                        f1 *= inverse;
                        if (P.out_lse)
                            P.out_lse[(long long)(done.row0 + done.node0 + pos / P.group) * P.q_heads + done.head * P.group + pos % P.group] =
                                (base + log2f(sum)) * 0.6931471805599453f;
                    } else
                        P.part_stats[part + pos] = make_float2(base, sum);
                    T.scale[t][pos] = f0;
                    T.top[t][0][pos] = f1;
                }
                group_sync(t);
                unsigned char* to = P.out + (long long)(done.row0 + done.node0) * P.out_row + (long long)(done.head * P.group) * P.out_head + pos * 2;
                const long long next_node = P.out_row - (P.group - 1) * P.out_head;
                float* to_part = P.parts + part * d + pos;
                int in_group = 0;
#pragma unroll 1
                for (int h = 0; h < rows; h += 16) {
                    float o[16];
                    tmem_load16(tO + h, o);
#pragma unroll
                    for (int c = 0; c < 16; ++c) o[c] *= T.scale[t][h + c];
                    if (join) {
                        float a[16];
                        tmem_load16(tOther + h, a);
#pragma unroll
                        for (int c = 0; c < 16; ++c) o[c] = fmaf(a[c], T.top[t][0][h + c], o[c]);
                    }
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        if (h + c < rows && pos < d) {
                            if (whole) *reinterpret_cast<uint16_t*>(to) = (uint16_t)pack16<false>(o[c], 0.f);
                            else to_part[(h + c) * d] = o[c];
                        }
                        to += P.out_head;
                        if (++in_group == P.group) { in_group = 0; to += next_node - P.out_head; }
                    }
                    __syncwarp();
                }
                if (join) { tc_fence_before(); arrive(&S.merge_done); }
                if (kKind != kAttnI8 && pos < d && *(volatile int*)&S.bad_value[units % kAttnUnitFlags] != 0)
                    for (int c = 0; c < rows; ++c) {     // values that were left out, where the row sees them
                        const int node = done.node0 + c / P.group;
                        const float bad = attn_bad_values<kNarrow>(P, done, node, pos);
                        if (bad == 0.f) continue;
                        if (!whole) P.parts[(part + c) * d + pos] += bad;
                        else {
                            uint16_t* at = reinterpret_cast<uint16_t*>(P.out + (long long)(done.row0 + node) * P.out_row +
                                                                       (long long)(done.head * P.group + c % P.group) * P.out_head) + pos;
                            *at = (uint16_t)pack16<false>(__uint_as_float((uint32_t)*at << 16) + bad, 0.f);
                        }
                    }
            }
            seq += 2 * count;
            ++units;
        }
        if (!ok && lane == 0) give_up();
    } else {
        if constexpr (kNarrow)
            if (!attn_widen<kKind, kWarps * 32>(P, it, tid - (kSoftmaxWarps + 3) * 32, raw, ring, tile_bytes, S.raw_full, S.raw_empty, S.full, S.empty,
                                                S.bad_value, abort_flag, [](const AttnUnit&, int) {}, [](int) {}) &&
                lane == 0)
                give_up();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256) : "memory");
    }
}

template <int kKind, int kN>
static int few_launch(AttnParams& P, const CUtensorMap& k, const CUtensorMap& v, int sms, cudaStream_t s)
{
    static std::atomic<unsigned long long> ready{0};
    constexpr int kSmem = kFewSmem + 1024;
    if (!attn_allow_smem(attn_few_kernel<kKind, kN>, kSmem, ready)) return launch_status();
    const int tile = P.chunks * kChunkBytes;
    // a chunk is left behind the ring: with up to 64 components the products read one past a tile (and nobody its results)
    int room = kFewSmem - 2 * kFewPBytes - P.chunks * kN * 128 - (P.chunks == 1 ? kChunkBytes : 0);
    if (kKind != kAttnWide) {
        P.slots = 4;
        room -= P.slots * tile;
        P.raw_slots = room / (kAttnTile * P.c.head_dim);
        if (P.raw_slots > kAttnMaxRaw) P.raw_slots = kAttnMaxRaw;
    } else {
        P.slots = room / tile;
        if (P.slots > kAttnMaxSlots) P.slots = kAttnMaxSlots;
        P.raw_slots = 0;
    }
    KernelTimerScope timer(DSPARK_K_TREE_ATTENTION, s);
    launch_pdl(attn_few_kernel<kKind, kN>, dim3((unsigned)sms), dim3(kFewThreads<kKind>), kSmem, s, P, k, v);
    return launch_status();
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
