// The vocabulary projection: int8 logits for serving (dspark_lm_head_int8) and the cross entropy of a hidden state
// against the vocabulary with its gradients (dspark_lm_head_loss, dspark_lm_head_loss_backward), logits never kept.
//
// All of it are tcgen05 contractions  D[m, n] = sum_k A[m, k] B[n, k]  with five epilogues:
//
//   unit        A                    B                    D (tensor memory)      epilogue
//   Int8Logits  w_q   [V, K]         x_q   [rows, K]      vocabulary x rows      sx * sw * D -> bf16 / fp32 logits
//   LossStats   H     [rows, d]      W     [V, d]         rows x vocabulary      softmax statistics, label's logit
//   LossGrad    H                    W (a piece)          rows x piece           G = g (softmax - onehot) -> bf16
//   GradHidden  G     [rows, piece]  W^T (a piece)        rows x d               fp32 partial sums of G W
//   GradWeight  G^T   [piece, rows]  H^T   [d, rows]      piece x d              dW = G^T H -> bf16
//
// A tile is 128 x (up to) 256: the accumulator is 256 of the 512 tensor-memory columns, so one is filled while the
// other is read.  A producer thread brings 128-byte wide tiles of both operands into a ring of stages by tensor-map
// copies (128-byte swizzle), one thread issues tcgen05.mma, eight warps read accumulators back, each owning a lane
// quarter and every other group of 32 columns.  Where the contraction runs over an operand's rows (the gradients), the
// tile is loaded as it lies in memory, [64 k][64 mn] boxes, and the MMA descriptor says so (mn-major): nothing is
// transposed in memory.
//
// Tile order: the index of the row tiles runs fastest, so that all row tiles of one stretch of the vocabulary run side
// by side and the weight is fetched from HBM once.
#include <cuda_bf16.h>
#include <cstring>
#include <math.h>

#include "common.cuh"
#include "tcgen05.cuh"

namespace dspark {

enum HeadMode { kInt8Logits = 0, kLossStats = 1 };
enum BackUnit { kLossGrad = 0, kGradHidden = 1, kGradWeight = 2, kEnd = 3 };

constexpr int kHeadM = 128;
constexpr int kHeadN = 256;                       // columns of one accumulator at most
constexpr int kRowBytes = 128;                    // bytes of k in one stage: 64 bf16 or 128 int8
constexpr int kTileABytes = kHeadM * kRowBytes;   // 16 KB
constexpr int kBoxMnBytes = 64 * kRowBytes;       // [64 k][64 mn] of bf16: 8 KB
constexpr int kHeadMaxStages = 10;
constexpr int kHeadRingBytes = 4 * (kTileABytes + kHeadN * kRowBytes);   // 192 KB
constexpr int kHeadEpiWarps = 8;                   // 16 take issue slots and polls from the issuer: backward 5 % slower, statistics 2 x
constexpr int kUnitSlots = 4;
constexpr int kHeadThreads = (2 + kHeadEpiWarps) * 32;
constexpr int kTurnPitch = 17;                   // words of 2 bf16: rows fall into different banks
constexpr int kTurnBytes = 32 * kTurnPitch * 4;   // one warp's block
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kHeadParts = kHeadEpiWarps / 4;     // warps per lane quarter
constexpr int kHeadGroups = kHeadN / 32 / kHeadParts;     // groups of 32 columns of one warp
// k blocks (of 64) of one accumulator of logits: see add_accumulator()
template <int kCtas> __host__ __device__ constexpr int logit_blocks() { return kCtas == 2 ? 8 : 4; }

struct HeadParams {
    int m, n, k;                    // extents; the one that counts rows is bounded by *live
    int n_tile, stages;
    int box_n;                      // rows of a B box: n_tile, or less where the operand has less
    const int32_t* live;            // number of rows that count, NULL: all
    int32_t* dev_status;
    void* out; long long out_stride; int out_bf16;                  // Int8Logits; out_bf16 2: pairs of entries may be stored
    const float* row_scale; const float* col_scale;
    float2* stats; long long stats_stride;                          // LossStats: [2 n_tiles][rows] (largest logit, sum of e^(z - it))
    const int32_t* labels; float* z_label;
    const __nv_bfloat16* rows; long long rows_stride;               // LossStats: the operands, for the labels' logits
    const __nv_bfloat16* w; long long w_stride;
};

// ---- descriptors ------------------------------------------------------------------------------------
// 128-byte swizzle (layout type 2), descriptor version 1.  k-major: rows of 128 B, groups of 8 rows 1 024 B apart
// (stride offset); the leading offset is not used.  mn-major: 64 mn elements per 128 B, one k per row; groups of 8 k
// 1 024 B apart (stride offset), the next 64 mn elements 8 KB further (leading offset).
__device__ __forceinline__ uint64_t head_desc(uint32_t addr, bool mn_major)
{
    const uint64_t lead = mn_major ? (uint64_t)(kBoxMnBytes >> 4) : 1ull;
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (lead << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <bool kInt8, int kCtas>
__device__ __forceinline__ void head_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
#define DSPARK_HEAD_MMA(GROUP, KIND)                                                       \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"                       \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n\t}" \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory")
    if (kInt8 && kCtas == 1) DSPARK_HEAD_MMA("1", "i8");
    if (kInt8 && kCtas == 2) DSPARK_HEAD_MMA("2", "i8");
    if (!kInt8 && kCtas == 1) DSPARK_HEAD_MMA("1", "f16");
    if (!kInt8 && kCtas == 2) DSPARK_HEAD_MMA("2", "f16");
#undef DSPARK_HEAD_MMA
}

// ---- pairs of CTAs -------------------------------------------------------------------------------------
// kCtas = 2: the two CTAs of a cluster share a tile of 256 rows.  Each holds 128 rows of A and half of B's columns in its
// shared memory and 128 rows of D in its tensor memory; the first one (the leader) issues the products for both.  B passes
// from the L2 once per pair instead of once per CTA: at 128 x 256 tiles the copies (48 KB a k block) kept the tensor cores
// waiting for a third of the time.  Barriers: `full` is the leader's (both CTAs' copies count on it), `empty` and
// `acc_full` each CTA's own (the products' completion is announced to both), `acc_empty` and `unit_empty` the leader's.
template <int kCtas>
__device__ __forceinline__ uint32_t pair_rank()
{
    uint32_t r = 0;
    if (kCtas == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// address of the same variable in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t pair_address(const void* p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
template <int kCtas>
__device__ __forceinline__ void pair_arrive(uint64_t* bar, uint32_t rank)
{
    if (kCtas == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(pair_address(bar, rank)) : "memory");
}
// The same where only the end of reads is announced (an accumulator or a unit's slot may be written again): without the
// release at cluster scope, which waits for the thread's stores to global memory, 3 us after the logits of a tile (int8,
// 1024 rows K 1024 142 -> 129 us).  What has been read is in registers by then: tcgen05.wait::ld, or a use of it.
template <int kCtas>
__device__ __forceinline__ void pair_arrive_read(uint64_t* bar, uint32_t rank)
{
    if (kCtas == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(pair_address(bar, rank)) : "memory");
}
// bounded wait on a barrier of this CTA that the other CTA may arrive on
template <int kCtas>
__device__ __forceinline__ bool pair_wait(uint64_t* bar, uint32_t parity)
{
    if constexpr (kCtas == 1) return mbar_wait_bounded(bar, parity);
    else for (uint32_t i = 0; i < kWaitPollLimit; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
template <int kCtas>
__device__ __forceinline__ void pair_sync()
{
    if (kCtas == 2) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
}
// completion of the products issued so far, announced on `bar` of both CTAs
template <int kCtas>
__device__ __forceinline__ void pair_commit(uint64_t* bar)
{
    if (kCtas == 1) umma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// tensor-map loads into this CTA's shared memory, counted on the leader's barrier (bit 24 of a shared address is the rank)
template <int kCtas>
__device__ __forceinline__ void pair_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar, uint64_t policy)
{
    if (kCtas == 1) tma_load_2d(dst, map, x, y, bar, policy);
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
                     "[%0], [%1, {%2, %3}], [%4], %5;"
                     ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar) & 0xFEFFFFFFu), "l"(policy)
                     : "memory");
}
template <int kCtas>
__device__ __forceinline__ void pair_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar, uint64_t policy)
{
    if (kCtas == 1) tma_load_3d(dst, map, x, y, z, bar, policy);
    else
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
                     "[%0], [%1, {%2, %3, %4}], [%5], %6;"
                     ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar) & 0xFEFFFFFFu),
                     "l"(policy)
                     : "memory");
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 consecutive bf16 of this lane's row (p 32-byte aligned): two whole sectors.  kOnce: nobody reads them soon
template <bool kOnce>
__device__ __forceinline__ void store_row32(__nv_bfloat16* p, const float (&v)[32])
{
#define DSPARK_STORE8(HINT)                                                                                                            \
    asm volatile("st.global" HINT ".v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"                                                         \
                 ::"l"(p + i), "r"(bf16_pair(v[i], v[i + 1])), "r"(bf16_pair(v[i + 2], v[i + 3])), "r"(bf16_pair(v[i + 4], v[i + 5])), \
                   "r"(bf16_pair(v[i + 6], v[i + 7])), "r"(bf16_pair(v[i + 8], v[i + 9])), "r"(bf16_pair(v[i + 10], v[i + 11])),       \
                   "r"(bf16_pair(v[i + 12], v[i + 13])), "r"(bf16_pair(v[i + 14], v[i + 15]))                                          \
                 : "memory")
#pragma unroll
    for (int i = 0; i < 32; i += 16) {
        if (kOnce) DSPARK_STORE8(".L2::evict_first");
        else DSPARK_STORE8("");
    }
#undef DSPARK_STORE8
}
// The same for rows that are not aligned or end inside: the 32 x 32 block of the warp is turned in shared memory (a pitch of
// 17 words), so that neighbouring lanes store neighbours of one row: pairs of two rows at a time where pairs are aligned
// (`pairs`), single elements otherwise.  `rows` and `n`: rows and columns that exist.
__device__ __forceinline__ void store_block32(__nv_bfloat16* p, long long stride, const float (&v)[32], int rows, int n, bool pairs,
                                              uint32_t* block, int lane)
{
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) block[lane * kTurnPitch + i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    __syncwarp();
    if (pairs) {
        const int c = lane & 15, r0 = lane >> 4;
        uint32_t* q = reinterpret_cast<uint32_t*>(p + r0 * stride) + c;
        if (2 * c + 1 < n)
#pragma unroll 8
            for (int r = r0; r < rows; r += 2) {
                *q = block[r * kTurnPitch + c];
                q += stride;                                // two rows of bf16: `stride` words
            }
        else if (2 * c < n)
            for (int r = r0; r < rows; r += 2) p[r * stride + 2 * c] = reinterpret_cast<const __nv_bfloat16*>(block + r * kTurnPitch)[2 * c];
    } else if (lane < n) {
#pragma unroll 8
        for (int r = 0; r < rows; ++r) p[r * stride + lane] = reinterpret_cast<const __nv_bfloat16*>(block + r * kTurnPitch)[lane];
    }
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// One element to each of 16 rows from `row` on, the first `n` of which exist.
template <typename T>
__device__ __forceinline__ void store_column16(T* p, long long stride, int row, int n, const float* v)
{
    p += row * stride;
    if (n >= 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) { put(p, v[i]); p += stride; }
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) { if (i < n) put(p, v[i]); p += stride; }
    }
}
// The same for bf16 in pairs: even lanes store the even rows' entries (their own and the next lane's), odd lanes the odd
// rows'.  p: the pair's first entry in row 0.
__device__ __forceinline__ void store_pairs16(__nv_bfloat16* p, long long stride, int row, int n, const float* v, int lane)
{
    const int odd = lane & 1;
    p += (row + odd) * stride;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float other = __shfl_xor_sync(0xffffffffu, odd ? v[i] : v[i + 1], 1);
        const uint32_t w = odd ? bf16_pair(other, v[i + 1]) : bf16_pair(v[i], other);
        if (i + odd < n) *reinterpret_cast<uint32_t*>(p) = w;
        p += 2 * stride;
    }
}

// Logits of a 128 x 256 tile, one row a lane: z (+)= this warp's groups of columns of an accumulator.
// The tensor cores cut an accumulator off after every product instead of rounding it, so its error grows with the length of
// the sum (d = 2 048: -1.3e-5 on a logit of 6, 9.7e-7 of the loss).  Sums are therefore cut into accumulators of 512 terms
// for many rows (3.0e-7 of the loss, with fp32 products 3.2e-7; 4096 rows 1.35 -> 1.42 ms) or 256 for few (64 rows 57 ->
// 60 us) that are added up here, rounded.  The gradients need no such care: a probability is only relatively off.
// `groups`: how many of the groups the tile has.
__device__ __forceinline__ void add_accumulator(float (&z)[kHeadGroups][32], uint32_t address, bool first, int groups)
{
    __syncwarp();
    if (first) {
#pragma unroll
        for (int j = 0; j < kHeadGroups; ++j) tmem_load32_issue(address + (uint32_t)(j * kHeadParts * 32), z[j]);
#pragma unroll
        for (int j = 0; j < kHeadGroups; ++j) tmem_load_wait(z[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kHeadGroups; ++j) {
            if (j >= groups) break;
            float v[32];
            tmem_load32_issue(address + (uint32_t)(j * kHeadParts * 32), v);
            tmem_load_wait(v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                const uint64_t sum = add2(pack2(z[j][i], z[j][i + 1]), pack2(v[i], v[i + 1]));
                unpack2(sum, z[j][i], z[j][i + 1]);
            }
        }
    }
}

// The logit of a row's label, a product of two rows summed by a warp in fp32, rounded.  Where a row is sure of its label,
// softmax - 1 there and the loss are small differences of this logit and lse, in which the tensor cores' cut-off sums showed
// (a loss of 5e-3: gradients 2.5 % off).  So the loss is written with this logit and the sum over the other entries, and the
// gradient takes the same logit, bit for bit.  16 MB more of W for 4096 rows: at most 1 % of a call.
// kAligned: h in vectors of 8; the sums are the same either way.
template <bool kAligned>
__device__ __forceinline__ float label_logit(const __nv_bfloat16* h, const __nv_bfloat16* w, int d, int lane)
{
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = lane; i < d / 8; i += 32) {
        const uint4 b = reinterpret_cast<const uint4*>(w)[i];
        const uint32_t y[4] = {b.x, b.y, b.z, b.w};
        uint4 a;
        if (kAligned) a = reinterpret_cast<const uint4*>(h)[i];
        else {
            const unsigned short* e = reinterpret_cast<const unsigned short*>(h) + 8 * i;
            a = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
        }
        const uint32_t x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum[2 * j] = fmaf(bf16lo(x[j]), bf16lo(y[j]), sum[2 * j]);
            sum[2 * j + 1] = fmaf(bf16hi(x[j]), bf16hi(y[j]), sum[2 * j + 1]);
        }
    }
    float z = ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
    const int i = d / 8 * 8 + lane;
    if (i < d) z = fmaf(__bfloat162float(h[i]), __bfloat162float(w[i]), z);
#pragma unroll
    for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    return z;
}

// What both kernels set up and take down: barriers, tensor memory.
struct HeadShared {
    uint64_t full[kHeadMaxStages], empty[kHeadMaxStages], acc_full[2], acc_empty[2], mma_done;
    uint64_t unit_full[kUnitSlots], unit_empty[kUnitSlots];         // backward: the units on their way
    int4 unit[kUnitSlots][2];
    uint32_t tmem_base;
    int abort;
};

template <int kCtas>
__device__ __forceinline__ uint32_t head_setup(HeadShared& S, int stages, int warp)
{
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(&S.full[s], 1); mbar_init(&S.empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&S.acc_full[s], 1); mbar_init(&S.acc_empty[s], kCtas * kHeadEpiWarps); }
        // read by: the issuer, the epilogue warps, the other CTA's producer
        for (int s = 0; s < kUnitSlots; ++s) { mbar_init(&S.unit_full[s], 1); mbar_init(&S.unit_empty[s], kCtas * (1 + kHeadEpiWarps)); }
        mbar_init(&S.mma_done, 1);
        S.abort = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        if (kCtas == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(2 * kHeadN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&S.tmem_base)), "r"(2 * kHeadN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    pair_sync<kCtas>();
    tc_fence_after();
    pdl_wait();
    return S.tmem_base;
}
// Both CTAs of a pair meet before either leaves: each may still be written to by the other until then.
template <int kCtas>
__device__ __forceinline__ void head_takedown(uint32_t tmem, int warp)
{
    tc_fence_before();
    __syncthreads();
    pair_sync<kCtas>();
    if (warp == 1) {
        tc_fence_after();
        if (kCtas == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kHeadN) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kHeadN) : "memory");
    }
}
// Somebody gave up: the leader's producer leaves only after the copies of the stages it has announced have landed (bounded);
// those of the other CTA count on the same barriers, so it just gives its last ones the time.
__device__ __forceinline__ void head_drain(HeadShared& S, int stages, int issued, bool leader)
{
    if (leader)
        for (int i = issued > stages ? issued - stages : 0; i < issued; ++i) mbar_wait_bounded(&S.full[i % stages], (uint32_t)(i / stages) & 1u);
    else
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}
// tensor memory is returned only after the last product
__device__ __forceinline__ void head_finish_products(HeadShared& S, bool issued, int ctas)
{
    if (issued) {
        if (ctas == 1) umma_commit(&S.mma_done);
        else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&S.mma_done)) : "memory");
        mbar_wait_bounded(&S.mma_done, 0u);
    }
}
template <int kCtas>
__device__ __forceinline__ uint32_t head_idesc(bool int8, bool a_mn, bool b_mn, int n)
{
    return ((int8 ? 2u : 1u) << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kCtas * kHeadM >> 4) << 24);
}

// ---- logits and softmax statistics ----------------------------------------------------------------------
template <int kMode, int kCtas>
__global__ void __launch_bounds__(kHeadThreads, 1)
lm_head_kernel(const __grid_constant__ HeadParams P, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    constexpr bool kInt8 = kMode == kInt8Logits;
    constexpr int kBlockK = kInt8 ? 128 : 64, kM = kCtas * kHeadM;
    constexpr int kPerAcc = kInt8 ? 1 << 20 : logit_blocks<kCtas>();       // integers are exact

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzle atoms: 1 KB
    __shared__ HeadShared S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = head_setup<kCtas>(S, P.stages, warp), rank = pair_rank<kCtas>();
    volatile int* abort_flag = &S.abort;
    auto give_up = [&]() { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; };

    // extents of this call: the row count may live on the device
    int m = P.m, n = P.n;
    if (P.live) {
        int live = *P.live;
        live = live < 0 ? 0 : live;
        int& rows = kInt8 ? n : m;
        rows = live < rows ? live : rows;
    }
    const int m_tiles = (m + kM - 1) / kM, n_tiles = (n + P.n_tile - 1) / P.n_tile;
    const int k_blocks = (P.k + kBlockK - 1) / kBlockK;
    const int n_units = m_tiles * n_tiles;
    // unit -> tile; the index over rows runs fastest
    auto tile = [&](int u, int& m0, int& nt) {
        if (kInt8) { nt = u % n_tiles; m0 = u / n_tiles * kM; }
        else { m0 = u % m_tiles * kM; nt = u / m_tiles; }
    };
    const int share = P.n_tile / kCtas;                     // B rows of one CTA
    // First B row of a CTA.  Int8Logits: a box that would reach past the last row is moved back -- the copy engine takes
    // some 24 clocks for each row outside, more than the products leave it -- and a few rows are computed twice.
    auto b_start = [&](int nt, int r) {
        const int at = nt * P.n_tile + r * share;
        return kInt8 ? (at < P.n - P.box_n ? at : P.n - P.box_n) : at;
    };
    const int stage_bytes = kTileABytes + share * kRowBytes;
    const uint32_t load_bytes = (uint32_t)(kCtas * (kTileABytes + P.box_n * kRowBytes));
    const int first = (int)blockIdx.x / kCtas, step = (int)gridDim.x / kCtas;

    if (warp == 0) {
        // ---------------- producer: operand tiles ---------------------------------------------------------
        if (lane == 0) {
            const uint64_t pol = l2_policy_evict_normal();
            int issued = 0, s = 0;
            uint32_t ph = 0;
            for (int u = first; u < n_units && !*abort_flag; u += step) {
                int m0, nt;
                tile(u, m0, nt);
                for (int kb = 0; kb < k_blocks; ++kb) {
                    if (!mbar_wait_bounded(&S.empty[s], ph ^ 1u)) { give_up(); break; }
                    unsigned char* a = smem + (size_t)s * stage_bytes;
                    if (rank == 0) mbar_arrive_expect_tx(&S.full[s], load_bytes);
                    pair_load_2d<kCtas>(a, &map_a, kb * kBlockK, m0 + (int)rank * kHeadM, &S.full[s], pol);
                    pair_load_2d<kCtas>(a + kTileABytes, &map_b, kb * kBlockK, b_start(nt, (int)rank), &S.full[s], pol);
                    ++issued;
                    if (++s == P.stages) { s = 0; ph ^= 1u; }
                }
            }
            for (int i = 0; i < P.stages && !*abort_flag; ++i) {   // the last announcements of free stages have arrived
                if (!mbar_wait_bounded(&S.empty[s], ph ^ 1u)) break;
                if (++s == P.stages) { s = 0; ph ^= 1u; }
            }
            if (*abort_flag) head_drain(S, P.stages, issued, rank == 0);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (of a pair: the leader's) -------------------------------------------
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = head_idesc<kCtas>(kInt8, false, false, P.n_tile);
            int s = 0, t = 0;
            uint32_t ph = 0;
            bool issued = false;
            bool ok = true;
            for (int u = first; ok && u < n_units && !*abort_flag; u += step)
                for (int k0 = 0; ok && k0 < k_blocks; k0 += kPerAcc, ++t) {
                    const uint32_t acc = (uint32_t)(t & 1), aph = (uint32_t)(t >> 1) & 1u;
                    ok = pair_wait<kCtas>(&S.acc_empty[acc], aph ^ 1u);
                    tc_fence_after();
                    for (int kb = k0; ok && kb < k_blocks && kb - k0 < kPerAcc; ++kb) {
                        ok = mbar_wait_bounded(&S.full[s], ph);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t a0 = smem_u32(smem + (size_t)s * stage_bytes), b0 = a0 + kTileABytes;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            head_mma<kInt8, kCtas>(tmem + acc * kHeadN, head_desc(a0 + ks * 32, false), head_desc(b0 + ks * 32, false), idesc,
                                                   (kb > k0 || ks > 0) ? 1u : 0u);
                        pair_commit<kCtas>(&S.empty[s]);
                        issued = true;
                        if (++s == P.stages) { s = 0; ph ^= 1u; }
                    }
                    if (ok) pair_commit<kCtas>(&S.acc_full[acc]);
                }
            if (!ok) give_up();
            head_finish_products(S, issued, kCtas);
        }
    } else {
        // ---------------- epilogue -----------------------------------------------------------------------
        const int q = warp & 3, part = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        const int chunks = (P.n_tile + 31) / 32;
        float* scales = (float*)(smem + kHeadRingBytes) + (warp - 2) * kHeadGroups * 32;
        int t = 0;
        bool ok = true;
        // the next accumulator, and its release
        auto take = [&](uint32_t& address) {
            const uint32_t acc = (uint32_t)(t & 1), aph = (uint32_t)(t >> 1) & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&S.acc_full[acc], aph));
            if (!ok && lane == 0) give_up();
            tc_fence_after();
            address = tmem + lane_base + acc * kHeadN;
        };
        auto release = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) pair_arrive_read<kCtas>(&S.acc_empty[t & 1], 0);
            ++t;
        };
        // the labels' logits, while the first tile is being computed: in the gather launch they cost 2 us of 59
        if (!kInt8)
            for (int r = (int)blockIdx.x * kHeadEpiWarps + warp - 2; r < m; r += (int)gridDim.x * kHeadEpiWarps) {
                const float z = label_logit<true>(P.rows + r * P.rows_stride, P.w + P.labels[r] * P.w_stride, P.k, lane);
                if (lane == 0) P.z_label[r] = z;
            }
        for (int u = first; ok && u < n_units && !*abort_flag; u += step) {
            int m0, nt;
            tile(u, m0, nt);
            const int row0 = m0 + (int)rank * kHeadM + q * 32, row = row0 + lane, n0 = nt * P.n_tile;
            const bool in = row < m;
            // Int8Logits: the row of the batch that a column of the accumulator is (past the last one: none)
            const int start0 = b_start(nt, 0), start1 = kCtas == 2 ? b_start(nt, 1) : 0;
            auto row_of = [&](int col) {
                if (col >= P.n_tile) return 1 << 30;
                return kCtas == 2 && col >= share ? start1 + col - share : start0 + col;
            };
            // what the tile needs besides the accumulator, asked for while it is being computed
            float sw = 0.f;
            int label = -1;
            if (kInt8) {
                if (in) sw = P.col_scale[row];
                __syncwarp();                               // the scales of the tile before have been read
#pragma unroll
                for (int j = 0; j < kHeadGroups; ++j) {
                    const int r = row_of((part + j * kHeadParts) * 32 + lane);
                    scales[j * 32 + lane] = r < n ? P.row_scale[r] : 0.f;
                }
                __syncwarp();
            } else if (in) {
                label = P.labels[row];
            }
            uint32_t acc_addr;
            if constexpr (kInt8) {
                take(acc_addr);
                if (!ok) break;
                if (row0 < m) {
                    for (int c = part; c < chunks; c += kHeadParts) {
                        // a CTA's share is a multiple of 16 rows: the 32 columns are two runs of 16 neighbouring rows
                        const int r0 = row_of(c * 32), r1 = row_of(c * 32 + 16);
                        if (r0 >= n && r1 >= n) continue;
                        const float* chunk_scales = scales + (c - part) / kHeadParts * 32;
                        float v[32];
                        __syncwarp();
                        tmem_load32(acc_addr + (uint32_t)(c * 32), v);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            const float4 sx = *reinterpret_cast<const float4*>(chunk_scales + i);
                            v[i] = (float)__float_as_int(v[i]) * sx.x * sw;
                            v[i + 1] = (float)__float_as_int(v[i + 1]) * sx.y * sw;
                            v[i + 2] = (float)__float_as_int(v[i + 2]) * sx.z * sw;
                            v[i + 3] = (float)__float_as_int(v[i + 3]) * sx.w * sw;
                        }
                        // lanes are neighbouring vocabulary entries: a warp stores 32 neighbours of one row at a time, or,
                        // bf16 rows that pairs of entries may be stored to, 32 neighbours of two rows
                        if (P.out_bf16 == 2 && row0 + 32 <= m) {
                            store_pairs16((__nv_bfloat16*)P.out + (row & ~1), P.out_stride, r0, n - r0, v, lane);
                            store_pairs16((__nv_bfloat16*)P.out + (row & ~1), P.out_stride, r1, n - r1, v + 16, lane);
                        } else if (P.out_bf16) {
                            store_column16((__nv_bfloat16*)P.out + row, P.out_stride, r0, in ? n - r0 : 0, v);
                            store_column16((__nv_bfloat16*)P.out + row, P.out_stride, r1, in ? n - r1 : 0, v + 16);
                        } else {
                            store_column16((float*)P.out + row, P.out_stride, r0, in ? n - r0 : 0, v);
                            store_column16((float*)P.out + row, P.out_stride, r1, in ? n - r1 : 0, v + 16);
                        }
                    }
                }
                release();
            } else {
                float z[kHeadGroups][32];
                const int groups = (chunks - part + kHeadParts - 1) / kHeadParts, end = n < n0 + P.n_tile ? n : n0 + P.n_tile;
                for (int k0 = 0; k0 < k_blocks; k0 += kPerAcc) {
                    take(acc_addr);
                    if (!ok) break;
                    if (row0 < m) add_accumulator(z, acc_addr + (uint32_t)(part * 32), k0 == 0, groups);
                    release();
                }
                if (!ok) break;
                // The sum of e^(z - top) without the label's term, top the largest of the lane's (up to) 128 logits: what
                // the loss of a row that is sure of its label consists of is not added to a one.
                float top = -INFINITY, sum = 0.f;
                if (row0 < m) {
#pragma unroll
                    for (int j = 0; j < kHeadGroups; ++j) {
                        const int col0 = n0 + (part + j * kHeadParts) * 32;
                        if (label >= col0 && label < col0 + 32) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (label == col0 + i) z[j][i] = -INFINITY;
                        }
                        if (end - col0 < 32) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i >= end - col0) z[j][i] = -INFINITY;
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) top = fmaxf(top, z[j][i]);
                    }
                    const float base = top == -INFINITY ? 0.f : top;
                    const uint64_t sc = pack2(kLog2e, kLog2e), no = pack2(-base, -base);
                    uint64_t a = pack2(0.f, 0.f), b = pack2(0.f, 0.f);
#pragma unroll
                    for (int j = 0; j < kHeadGroups; ++j) {
                        if (j >= groups) break;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float t0, t1, t2, t3;
                            unpack2(mul2(add2(pack2(z[j][i], z[j][i + 1]), no), sc), t0, t1);
                            unpack2(mul2(add2(pack2(z[j][i + 2], z[j][i + 3]), no), sc), t2, t3);
                            a = add2(a, pack2(ex2_approx(t0), ex2_approx(t1)));
                            b = add2(b, pack2(ex2_approx(t2), ex2_approx(t3)));
                        }
                    }
                    float s0, s1;
                    unpack2(add2(a, b), s0, s1);
                    sum = s0 + s1;
                }
                if (in) P.stats[(size_t)(nt * kHeadParts + part) * P.stats_stride + row] = make_float2(top, sum);
            }
        }
    }
    head_takedown<kCtas>(tmem, warp);
}

// ---- gradients -------------------------------------------------------------------------------------------
// One launch for all pieces of the vocabulary.  Units are handed out in order from a counter (the producer asks, the
// other roles read the unit from shared memory), long ones first within a phase:
//     C(0)  C(1) AB(0)  C(2) AB(1)  ...  C(P-1) AB(P-2)  AB(P-1)
// C(p): the tiles of G of piece p; AB(p): the tiles of dH's partial sums over piece p, then those of dW's rows of it.  G of
// three pieces is kept.  A unit waits (bounded) until what it needs is done: AB(p) for C(p) and, dH adding to what the
// piece before left, for the dH tiles of piece p-1; C(p) for AB(p-3), whose piece of G it overwrites.  All of that was
// handed out earlier, by at least a phase, to CTAs that are running: the waits end, and are short.  One launch per product
// and piece left SMs idle at the end of each of three launches a piece: 4096 rows, d 2048 6.9 ms, 6.0 ms this way (single
// CTAs), 5.1 ms with pairs.
struct BackParams {
    int n_pad, V, d;
    int piece, pieces;              // entries of a piece (a multiple of 256), number of pieces
    int n_tile_d, d_tiles;
    int slices, kb_slice;           // k blocks of a piece, cut for GradHidden
    int want_h, want_w;
    int box_v;                      // rows of a box of w_k
    int w_blocks;                   // 1: w_mn is the three-dimensional view (d a multiple of 64), 0: two-dimensional
    const int32_t* live;
    int32_t* dev_status;
    int32_t* sync;                  // [0] next unit, [1 + 3 p + kind] warps done with the units of that kind of piece p; zeros at the start
    __nv_bfloat16* G;               // three buffers [n_pad][piece]
    const int32_t* labels; const float* lse2; const float* grad; const float* at_label; const float* label_err;  // rows in the order of their labels
    const int32_t* first;           // first row of a vocabulary entry that has rows
    const __nv_bfloat16* rows; long long rows_stride;
    float* part; long long part_stride;
    __nv_bfloat16* dw; long long dw_stride;
};
struct BackMaps { CUtensorMap rows_k, w_k, g_k, w_mn, g_mn, rows_mn; };

__device__ __forceinline__ bool wait_for_count(const int32_t* cell, int want)
{
    for (uint32_t i = 0; i < kWaitPollLimit; ++i) {
        int v;
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(cell) : "memory");
        if (v >= want) return true;
    }
    return false;
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// v += a * 32 bf16
__device__ __forceinline__ void add_scaled32(float (&v)[32], float a, const uint4 (&h)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {h[i].x, h[i].y, h[i].z, h[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[8 * i + 2 * j] = fmaf(a, bf16lo(w[j]), v[8 * i + 2 * j]);
            v[8 * i + 2 * j + 1] = fmaf(a, bf16hi(w[j]), v[8 * i + 2 * j + 1]);
        }
    }
}
// The same for a vocabulary entry that is the label of many rows, by the whole warp: eight rows at a time, four lanes a row;
// lane `owner`, whose entry it is, gets the sum.  A lane alone waits for a load a row: 200 rows of one label, V = 10 007,
// d = 500 226 us a call, 47.5 this way; 4096 rows, V = 129 280, d = 2 048 9.3 ms, 5.2.  But lanes with short runs work side by
// side: label frequencies falling as 1 / rank, runs of up to 11, 48 us alone and 54 this way.
constexpr int kLongRun = 16;
__device__ __forceinline__ void add_long_run32(float (&v)[32], const __nv_bfloat16* rows, long long stride, const float* err, int run,
                                               int owner, int lane)
{
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int r = lane >> 2; r < run; r += 8) {
        const uint4 h = reinterpret_cast<const uint4*>(rows + r * stride)[lane & 3];
        const float e = err[r];
        const uint32_t w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum[2 * j] = fmaf(e, bf16lo(w[j]), sum[2 * j]);
            sum[2 * j + 1] = fmaf(e, bf16hi(w[j]), sum[2 * j + 1]);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = 4; o < 32; o *= 2) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const float t = __shfl_sync(0xffffffffu, sum[i & 7], i >> 3);
        if (lane == owner) v[i] += t;
    }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    asm volatile("ld.relaxed.gpu.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store8(float* p, const float* v)
{
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}

template <int kCtas>
__global__ void __launch_bounds__(kHeadThreads, 1)
lm_head_backward_kernel(const __grid_constant__ BackParams P, const __grid_constant__ BackMaps M)
{
    constexpr int kM = kCtas * kHeadM;
    constexpr int kStageBytes = kTileABytes + kHeadN / kCtas * kRowBytes;
    constexpr int kStages = kHeadRingBytes / kStageBytes;
    constexpr int kDone = kCtas * kHeadEpiWarps;            // arrivals of a unit
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ HeadShared S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = head_setup<kCtas>(S, kStages, warp), rank = pair_rank<kCtas>();
    volatile int* abort_flag = &S.abort;
    auto give_up = [&]() { atomicOr(P.dev_status, DSPARK_DEV_TIMEOUT); *abort_flag = 1; };

    if (P.want_h) pdl_trigger();                            // the sum of the slices is the next launch, and ours
    const int live = *P.live;
    const int m_tiles = (live + kM - 1) / kM;

    if (warp == 0) {
        // ---------------- producer: units, then operand tiles ----------------------------------------------
        if (lane == 0) {
            // W is read for G and, a phase later, for dH, and then no more: kept until then (dW is stored past it); 128 rows,
            // d 1024 205 -> 199 us
            const uint64_t pol = l2_policy_evict_normal(), pol_keep = l2_policy_evict_last(), pol_done = l2_policy_evict_first();
            const int last = P.V - (P.pieces - 1) * P.piece;               // entries of the last piece
            const int row_blocks = (live + 63) / 64;
            auto here = [&](int p) { return p == P.pieces - 1 ? last : P.piece; };
            auto count_c = [&](int p) { return m_tiles * ((here(p) + kHeadN - 1) / kHeadN); };
            const int count_a = P.want_h ? m_tiles * P.d_tiles * P.slices : 0;
            auto count_b = [&](int p) { return P.want_w ? (here(p) + kM - 1) / kM * P.d_tiles : 0; };
            int issued = 0, s = 0, slot = 0;
            uint32_t ph = 0, sph = 0;
            // The walk over the phases: units arrive in rising order, so the phase only moves forward.
            int phase = 0, phase_first = 0, phase_count = count_c(0), phase_piece = 0;
            bool phase_c = true;
            const int n_phases = 2 * P.pieces;
            auto next_phase = [&]() {
                phase_first += phase_count;
                ++phase;
                // 0: C(0); odd i: C((i + 1) / 2) while there is one; even i: AB(i / 2 - 1); the last: AB(P - 1)
                if (phase >= n_phases) return;
                if (phase == n_phases - 1) { phase_c = false; phase_piece = P.pieces - 1; }
                else if (phase & 1) { phase_c = true; phase_piece = (phase + 1) / 2; }
                else { phase_c = false; phase_piece = phase / 2 - 1; }
                phase_count = phase_c ? count_c(phase_piece) : count_a + count_b(phase_piece);
            };
            // A unit is asked for while the one before it is being loaded, and a phase that was seen done is not looked at
            // again: either costs a round trip to the L2, which is most of what the ring holds.
            int next = rank == 0 ? atomicAdd(P.sync, 1) : 0, seen[3] = {-1, -1, -1};
            auto wait_for = [&](int kind, int p) {
                if (p <= seen[kind]) return true;
                seen[kind] = p;
                const int count = kind == kLossGrad ? count_c(p) : kind == kGradHidden ? count_a : count_b(p);
                return wait_for_count(P.sync + 1 + 3 * p + kind, count * kDone);
            };
            for (;;) {
                int kind = kEnd, m0 = 0, n0 = 0, kb0 = 0, kb1 = 0, p = 0;
                if (rank == 0) {
                    // ---- the next unit: its tile, and what it has to wait for ----
                    if (!pair_wait<kCtas>(&S.unit_empty[slot], sph ^ 1u)) { give_up(); break; }
                    if (*abort_flag) break;
                    const int u = next;
                    int slice = 0;
                    bool ok = true;
                    while (phase < n_phases && u - phase_first >= phase_count) next_phase();
                    p = phase_piece;
                    if (phase < n_phases) {
                        int i = u - phase_first;
                        const int piece_blocks = (here(p) + 63) / 64;
                        if (phase_c) {
                            kind = kLossGrad;
                            m0 = i % m_tiles * kM; n0 = i / m_tiles * kHeadN;
                            kb1 = (P.d + 63) / 64;
                            if (p >= 3) ok = wait_for(kGradHidden, p - 3) && wait_for(kGradWeight, p - 3);
                        } else {
                            ok = wait_for(kLossGrad, p);
                            if (i < count_a) {
                                kind = kGradHidden;
                                m0 = i % m_tiles * kM; i /= m_tiles;
                                n0 = i % P.d_tiles * P.n_tile_d; slice = i / P.d_tiles;
                                kb0 = slice * P.kb_slice;
                                kb0 = kb0 < piece_blocks ? kb0 : piece_blocks;
                                kb1 = kb0 + P.kb_slice < piece_blocks ? kb0 + P.kb_slice : piece_blocks;
                                if (p >= 1) ok = ok && wait_for(kGradHidden, p - 1);
                            } else {
                                kind = kGradWeight;
                                i -= count_a;
                                n0 = i % P.d_tiles * P.n_tile_d; m0 = i / P.d_tiles * kM;
                                kb1 = row_blocks;
                            }
                        }
                        if (!ok) { give_up(); break; }
                    }
                    const int4 u0 = make_int4(kind, m0, n0, kb0), u1 = make_int4(kb1, p, slice, 0);
                    S.unit[slot][0] = u0;
                    S.unit[slot][1] = u1;
                    mbar_arrive(&S.unit_full[slot]);
                    if (kCtas == 2) {
                        const uint32_t to = pair_address(&S.unit[slot][0], 1);
                        asm volatile("st.shared::cluster.v4.s32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(u0.x), "r"(u0.y), "r"(u0.z), "r"(u0.w) : "memory");
                        asm volatile("st.shared::cluster.v4.s32 [%0], {%1,%2,%3,%4};" ::"r"(to + 16), "r"(u1.x), "r"(u1.y), "r"(u1.z), "r"(u1.w) : "memory");
                        pair_arrive<kCtas>(&S.unit_full[slot], 1);
                    }
                } else {
                    // ---- the unit that the leader has taken ----
                    if (!pair_wait<kCtas>(&S.unit_full[slot], sph)) { give_up(); break; }
                    const int4 u0 = S.unit[slot][0], u1 = S.unit[slot][1];
                    pair_arrive<kCtas>(&S.unit_empty[slot], 0);
                    kind = u0.x; m0 = u0.y; n0 = u0.z; kb0 = u0.w; kb1 = u1.x; p = u1.y;
                }
                if (++slot == kUnitSlots) { slot = 0; sph ^= 1u; }
                if (kind == kEnd) break;
                if (kind != kLossGrad) fence_proxy_async_all();            // G was written by ordinary stores and is read by copies
                if (rank == 0) next = atomicAdd(P.sync, 1);
                const int v0 = p * P.piece, g0 = p % 3 * P.n_pad;          // first entry of the piece, first row of its G
                const int half_d = P.n_tile_d / kCtas;                     // columns of B in this CTA
                const uint32_t load_bytes = (uint32_t)(kCtas * (kTileABytes + (kind == kLossGrad ? P.box_v : half_d) * kRowBytes));
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait_bounded(&S.empty[s], ph ^ 1u)) { give_up(); break; }
                    unsigned char* a = smem + (size_t)s * kStageBytes;
                    unsigned char* b = a + kTileABytes;
                    uint64_t* bar = &S.full[s];
                    if (rank == 0) mbar_arrive_expect_tx(bar, load_bytes);
                    const int kx = kb * 64, mr = m0 + (int)rank * kHeadM;
                    if (kind == kLossGrad) {
                        pair_load_2d<kCtas>(a, &M.rows_k, kx, mr, bar, pol);
                        pair_load_2d<kCtas>(b, &M.w_k, kx, v0 + n0 + (int)rank * (kHeadN / kCtas), bar, pol_keep);
                    } else {
                        const int nr = n0 + (int)rank * half_d;
                        if (kind == kGradHidden) {
                            pair_load_2d<kCtas>(a, &M.g_k, kx, g0 + mr, bar, pol);
                            if (P.w_blocks) pair_load_3d<kCtas>(b, &M.w_mn, 0, v0 + kx, nr / 64, bar, pol_done);
                            else for (int j = 0; j < half_d; j += 64) pair_load_2d<kCtas>(b + j * kRowBytes, &M.w_mn, nr + j, v0 + kx, bar, pol_done);
                        } else {
                            pair_load_3d<kCtas>(a, &M.g_mn, 0, g0 + kx, mr / 64, bar, pol);
                            pair_load_3d<kCtas>(b, &M.rows_mn, 0, kx, nr / 64, bar, pol);
                        }
                    }
                    ++issued;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (*abort_flag) break;
            }
            for (int i = 0; i < kStages && !*abort_flag; ++i) {   // the last announcements of free stages have arrived
                if (!mbar_wait_bounded(&S.empty[s], ph ^ 1u)) break;
                if (++s == kStages) { s = 0; ph ^= 1u; }
            }
            if (*abort_flag) head_drain(S, kStages, issued, rank == 0);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (of a pair: the leader's) -------------------------------------------
        if (lane == 0 && rank == 0) {
            int s = 0, t = 0, slot = 0;
            uint32_t ph = 0, sph = 0;
            bool issued = false, ok = true;
            while (!*abort_flag) {
                ok = mbar_wait_bounded(&S.unit_full[slot], sph);
                if (!ok) break;
                const int4 u0 = S.unit[slot][0], u1 = S.unit[slot][1];
                mbar_arrive(&S.unit_empty[slot]);
                if (++slot == kUnitSlots) { slot = 0; sph ^= 1u; }
                const int kind = u0.x, kb0 = u0.w, kb1 = u1.x;
                if (kind == kEnd) break;
                if (kb0 == kb1) continue;                   // nothing to add up: the epilogue knows
                const bool a_mn = kind == kGradWeight, b_mn = kind != kLossGrad;
                const uint32_t idesc = head_idesc<kCtas>(false, a_mn, b_mn, kind == kLossGrad ? kHeadN : P.n_tile_d);
                const uint32_t step_a = a_mn ? 2048 : 32, step_b = b_mn ? 2048 : 32;
                const uint32_t acc = (uint32_t)(t & 1), aph = (uint32_t)(t >> 1) & 1u;
                ok = pair_wait<kCtas>(&S.acc_empty[acc], aph ^ 1u);
                tc_fence_after();
                for (int kb = kb0; ok && kb < kb1; ++kb) {
                    ok = mbar_wait_bounded(&S.full[s], ph);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a0 = smem_u32(smem + (size_t)s * kStageBytes), b0 = a0 + kTileABytes;
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        head_mma<false, kCtas>(tmem + acc * kHeadN, head_desc(a0 + ks * step_a, a_mn), head_desc(b0 + ks * step_b, b_mn), idesc,
                                        (kb > kb0 || ks > 0) ? 1u : 0u);
                    pair_commit<kCtas>(&S.empty[s]);
                    issued = true;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                pair_commit<kCtas>(&S.acc_full[acc]);
                ++t;
            }
            if (!ok) give_up();
            head_finish_products(S, issued, kCtas);
        }
    } else {
        // ---------------- epilogue -----------------------------------------------------------------------
        const int q = warp & 3, part = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(q * 32) << 16;
        uint32_t* turn = (uint32_t*)(smem + kHeadRingBytes + (warp - 2) * kTurnBytes);
        const bool dw_pairs = ((uintptr_t)P.dw & 3u) == 0 && (P.dw_stride & 1) == 0;
        const bool dw_vec = ((uintptr_t)P.dw & 31u) == 0 && (P.dw_stride & 15) == 0;
        int t = 0, slot = 0;
        uint32_t sph = 0;
        while (!*abort_flag) {
            if (!__all_sync(0xffffffffu, pair_wait<kCtas>(&S.unit_full[slot], sph))) {
                if (lane == 0) give_up();
                break;
            }
            const int4 u0 = S.unit[slot][0], u1 = S.unit[slot][1];
            __syncwarp();
            if (lane == 0 && u0.x >= 0 && u1.x >= 0) pair_arrive_read<kCtas>(&S.unit_empty[slot], 0);      // always: both have been read
            if (++slot == kUnitSlots) { slot = 0; sph ^= 1u; }
            const int kind = u0.x, row0 = u0.y + (int)rank * kHeadM + q * 32, n0 = u0.z, p = u1.y;
            const bool any = u0.w < u1.x;
            if (kind == kEnd) break;
            const uint32_t acc = (uint32_t)(t & 1), aph = (uint32_t)(t >> 1) & 1u;
            const int row = row0 + lane;
            int label = -1;
            float lse2 = 0.f, g = 0.f, at_label = 0.f;
            if (kind == kLossGrad && row < live) { label = P.labels[row]; lse2 = P.lse2[row]; g = P.grad[row]; at_label = P.at_label[row]; }
            // GradWeight: the rows whose label is this lane's vocabulary entry, and what the first of them lost
            int run = 0, run_first = 0;
            float run_err = 0.f;
            if (kind == kGradWeight && p * P.piece + row < P.V) {
                const int v = p * P.piece + row;
                run_first = P.first[v];
                if ((unsigned)run_first < (unsigned)live && P.labels[run_first] == v) {
                    run_err = P.label_err[run_first];
                    // rows are in the order of their labels: the end of the run, by doubling and then halving
                    auto inside = [&](int r) { return run_first + r < live && P.labels[run_first + r] == v; };
                    int in = 0;
                    for (run = 1; inside(run); run *= 2) in = run;
                    while (run - in > 1) {
                        const int at = (run + in) / 2;
                        if (inside(at)) in = at; else run = at;
                    }
                }
            }
            const unsigned long_runs = __ballot_sync(0xffffffffu, run > kLongRun);
            if (any) {
                if (!__all_sync(0xffffffffu, mbar_wait_bounded(&S.acc_full[acc], aph))) {
                    if (lane == 0) give_up();
                    break;
                }
                tc_fence_after();
                ++t;
            }
            const uint32_t acc_addr = tmem + lane_base + acc * kHeadN;
            auto load = [&](int c, float (&v)[32]) {
                __syncwarp();
                if (any) tmem_load32(acc_addr + (uint32_t)(c * 32), v);
                else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0.f;
                }
            };
            if (kind == kLossGrad) {
                // rows past the last one that counts are written as zeros: the product over rows reads them
                const bool in = row < live;
                const int v0 = p * P.piece;
                label -= v0;
                __nv_bfloat16* out = P.G + ((long long)(p % 3) * P.n_pad + row) * P.piece;
                for (int c = part; c < kHeadN / 32; c += kHeadParts) {
                    const int col0 = n0 + c * 32;
                    float z[32];
                    load(c, z);
                    const int valid = in ? P.V - v0 - col0 : 0;            // vocabulary entries from here on
#pragma unroll
                    for (int i = 0; i < 32; ++i) z[i] = ex2_approx(fmaf(z[i], kLog2e, -lse2)) * g;
                    if (label >= col0 && label < col0 + 32) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (label == col0 + i) z[i] = at_label;
                    }
                    if (valid < 32) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= valid) z[i] = 0.f;
                    }
                    store_row32<false>(out + col0, z);
                }
            } else if (kind == kGradHidden) {
                float* out = P.part + ((long long)u1.z * P.n_pad + row) * P.part_stride;
                if (row0 < live)
                    for (int c = part; c < P.n_tile_d / 32; c += kHeadParts) {
                        const int col0 = n0 + c * 32;
                        if (col0 >= P.d) break;
                        float v[32];
                        load(c, v);
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            if (row >= live || col0 + i >= P.d) break;     // the pitch is a multiple of 8
                            if (p) {
                                float before[8];
                                load8(out + col0 + i, before);
#pragma unroll
                                for (int j = 0; j < 8; ++j) v[i + j] += before[j];
                            }
                            store8(out + col0 + i, v + i);
                        }
                    }
            } else {
                const int first = p * P.piece + row0;               // vocabulary entry of lane 0
                const int rows = P.V - first < 32 ? P.V - first : 32;
                __nv_bfloat16* out = P.dw + (long long)first * P.dw_stride;
                if (rows > 0)
                    for (int c = part; c < P.n_tile_d / 32; c += kHeadParts) {
                        const int col0 = n0 + c * 32;
                        if (col0 >= P.d) break;
                        // What the rounding of G lost of the labels' entries, most of a row of G and, with equal weights,
                        // the same part of each (without this dW was 2.4e-3 off instead of 1.7e-3, its own rounding).
                        const __nv_bfloat16* h = P.rows + (long long)run_first * P.rows_stride + col0;
                        uint4 h0[4];
                        const int alone = run > kLongRun ? 0 : run;
                        if (alone)
#pragma unroll
                            for (int i = 0; i < 4; ++i) h0[i] = reinterpret_cast<const uint4*>(h)[i];
                        float v[32];
                        load(c, v);
                        if (alone) add_scaled32(v, run_err, h0);
                        for (int r = 1; r < alone; ++r) {
                            h += P.rows_stride;
#pragma unroll
                            for (int i = 0; i < 4; ++i) h0[i] = reinterpret_cast<const uint4*>(h)[i];
                            add_scaled32(v, P.label_err[run_first + r], h0);
                        }
                        for (unsigned left = long_runs; left; left &= left - 1) {
                            const int owner = __ffs(left) - 1, at = __shfl_sync(0xffffffffu, run_first, owner);
                            add_long_run32(v, P.rows + (long long)at * P.rows_stride + col0, P.rows_stride, P.label_err + at,
                                           __shfl_sync(0xffffffffu, run, owner), owner, lane);
                        }
                        if (dw_vec && P.d - col0 >= 32) {
                            if (lane < rows) store_row32<true>(out + lane * P.dw_stride + col0, v);
                        } else {
                            store_block32(out + col0, P.dw_stride, v, rows, P.d - col0, dw_pairs, turn, lane);
                        }
                    }
            }
            tc_fence_before();
            if (kind != kGradWeight) fence_proxy_async_all();
            __syncwarp();
            if (lane == 0) {
                if (any) pair_arrive_read<kCtas>(&S.acc_empty[acc], 0);
                // Nobody in this launch reads dW: what is counted for it is that G has been read.  (The fence waits for the
                // stores: a microsecond or two, as long as a short unit's products take.)
                if (kind != kGradWeight) __threadfence();
                atomicAdd(P.sync + 1 + 3 * p + kind, 1);
            }
        }
    }
    head_takedown<kCtas>(tmem, warp);
}

// ---- rows that count ------------------------------------------------------------------------
// A row whose label is negative is ignored: it is left out of the products altogether, so it costs nothing and nothing
// it holds (padding, NaN) can reach a gradient.  The rows that count are copied next to each other; each CTA finds the
// places of its own rows by looking at all labels.  The last CTA fills up the last block of 64 rows with zeros (the product
// over rows reads it) and leaves the count.
struct GatherParams {
    const __nv_bfloat16* h; long long h_stride;
    const int32_t* labels;
    int N, V, d;
    __nv_bfloat16* rows; long long rows_stride;     // compact copy
    int32_t* live; int32_t* idx; int32_t* label;
    int32_t* first;                                 // backward: [V]
    float* loss; float* lse;                        // forward: zeros of the ignored rows
    const float* lse_in; const float* grad_in; float* grad;    // backward (lse: the compact rows', times log2(e))
    const float* loss_in;                           // backward: the rows' losses, or NULL
    const __nv_bfloat16* w; long long w_stride;     // backward
    float* at_label; float* label_err;              // backward: the label's entry of G, and what is lost when it is rounded to bf16
    __nv_bfloat16* dh; long long dh_stride;         // backward: zeros of the ignored rows
    int32_t* sync; int n_sync;                      // backward: the counters of the units, zeroed
    int32_t* dev_status;
};
constexpr int kGatherThreads = 256;

// One row by a warp, kFlight elements of each lane in flight.
template <int kFlight, typename T>
__device__ __forceinline__ void copy_row(T* dst, const T* src, int n, int lane)
{
    for (int i = lane; i < n; i += 32 * kFlight) {
        T v[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (i + 32 * u < n) v[u] = src[i + 32 * u];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (i + 32 * u < n) dst[i + 32 * u] = v[u];
    }
}

// kGatherRows: 8, a row per warp, while looking at all labels costs nothing; 32 for long inputs.
// kSort (gradients): in the order of (label, row) instead of the rows' own, so that the rows of one vocabulary entry lie next
// to each other from first[entry] on (entries without rows: whatever was there, which the reader checks).
template <int kGatherRows, bool kSort>
__global__ void __launch_bounds__(kGatherThreads) lm_head_gather_kernel(const __grid_constant__ GatherParams P)
{
    __shared__ int s_slot[kGatherRows], s_label[kGatherRows], s_later[kGatherRows], s_total;
    pdl_wait();
    pdl_trigger();                                          // the contraction may set up its barriers and tensor memory
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r0 = blockIdx.x * kGatherRows;
    for (int i = blockIdx.x * kGatherThreads + tid; i < P.n_sync; i += gridDim.x * kGatherThreads) P.sync[i] = 0;
    const unsigned V = (unsigned)P.V;                       // a label counts when it is below V as an unsigned number
    const bool last = blockIdx.x == gridDim.x - 1;
    const int end_scan = kSort || last ? P.N : r0;
    int other = tid < end_scan ? P.labels[tid] : -1;        // of the scan below, asked for together with the CTA's own
    if (tid < kGatherRows) {
        s_label[tid] = r0 + tid < P.N ? P.labels[r0 + tid] : -1;
        s_slot[tid] = s_later[tid] = 0;
    }
    if (tid == 0) s_total = 0;
    __syncthreads();
    const int vectors = ((uintptr_t)P.h & 15u) == 0 && P.h_stride % 8 == 0 ? P.d / 8 : 0;
    float at_label[kGatherRows / (kGatherThreads / 32)];    // g (softmax - 1) of the warp's rows
    if (kSort)
#pragma unroll
        for (int j = 0; j < kGatherRows / (kGatherThreads / 32); ++j) {
            const int r = warp + j * (kGatherThreads / 32), label = s_label[r];
            if ((unsigned)label >= V) continue;
            const float g = P.grad_in[r0 + r];
            float x;                                        // the logarithm of the label's probability
            if (P.loss_in) {
                x = -P.loss_in[r0 + r];
            } else {
                // lse holds it to half a unit of its own last place and no better (losses of 1e-5 at a logit of 13: 4.6 % off)
                const __nv_bfloat16* h = P.h + (long long)(r0 + r) * P.h_stride;
                const __nv_bfloat16* w = P.w + (long long)label * P.w_stride;
                x = (vectors ? label_logit<true>(h, w, P.d, lane) : label_logit<false>(h, w, P.d, lane)) - P.lse_in[r0 + r];
            }
            at_label[j] = expm1f(x > 0.f ? 0.f : x) * g;
        }
    // every row's place: the rows that come before it
    int count[kSort ? kGatherRows : 1], total = 0;
#pragma unroll
    for (int j = 0; j < (kSort ? kGatherRows : 1); ++j) count[j] = 0;
    for (int m = tid; m < end_scan; m += kGatherThreads) {
        if (m != tid) other = P.labels[m];
        if ((unsigned)other >= V) continue;
        ++total;
        if (kSort) {
#pragma unroll
            for (int j = 0; j < kGatherRows; ++j) {
                const int mine = s_label[j];
                count[j] += other < mine || (other == mine && m < r0 + j);
                if (other == mine && m < r0 + j) s_later[j] = 1;           // not the first of its entry (every writer writes 1)
            }
        } else {
            count[0] += m < r0;
        }
    }
#pragma unroll
    for (int j = 0; j < (kSort ? kGatherRows : 1); ++j) {
        const int sum = __reduce_add_sync(0xffffffffu, count[j]);
        if (lane == 0 && sum) atomicAdd(&s_slot[j], sum);
    }
    total = __reduce_add_sync(0xffffffffu, total);
    if (lane == 0 && total) atomicAdd(&s_total, total);
    __syncthreads();
    if (warp == 0) {
        const int row = r0 + lane, label = lane < kGatherRows ? s_label[lane] : -1;
        const bool in = (unsigned)label < V;
        const unsigned mask = __ballot_sync(0xffffffffu, in);
        const int slot = kSort ? s_slot[lane < kGatherRows ? lane : 0] : s_slot[0] + __popc(mask & ((1u << lane) - 1u));
        const bool head = lane < kGatherRows && !s_later[lane < kGatherRows ? lane : 0];
        __syncwarp();
        if (lane < kGatherRows) s_slot[lane] = in ? slot : -1;
        if (in) {
            P.idx[slot] = row;
            P.label[slot] = label;
            if (kSort) {
                P.lse[slot] = P.lse_in[row] * kLog2e;
                P.grad[slot] = P.grad_in[row];
                if (head) P.first[label] = slot;
            }
        } else if (lane < kGatherRows && row < P.N) {
            if (P.loss) { P.loss[row] = 0.f; P.lse[row] = 0.f; }
            if (label >= 0) atomicOr(P.dev_status, DSPARK_DEV_BAD_TOKEN);
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kGatherRows / (kGatherThreads / 32); ++j) {
        const int r = warp + j * (kGatherThreads / 32);
        if (r0 + r >= P.N) break;
        const int to = s_slot[r];
        const __nv_bfloat16* src = P.h + (long long)(r0 + r) * P.h_stride;
        if (to >= 0) {
            __nv_bfloat16* dst = P.rows + (long long)to * P.rows_stride;
            copy_row<4>(reinterpret_cast<uint4*>(dst), reinterpret_cast<const uint4*>(src), vectors, lane);
            copy_row<16>(dst + vectors * 8, src + vectors * 8, P.d - vectors * 8, lane);
            if (kSort && lane == 0) {
                P.at_label[to] = at_label[j];               // the products read the bf16 of it
                P.label_err[to] = at_label[j] - __bfloat162float(__float2bfloat16_rn(at_label[j]));
            }
        } else if (P.dh) {
            __nv_bfloat16* dst = P.dh + (long long)(r0 + r) * P.dh_stride;
            for (int i = lane; i < P.d; i += 32) dst[i] = __float2bfloat16_rn(0.f);
        }
    }
    if (last) {
        const int live = s_total;
        if (tid == 0) *P.live = live;
        const int end = (live + 63) & ~63;
        for (int r = live + warp; r < end; r += kGatherThreads / 32)
            for (int i = lane; i < P.d; i += 32) P.rows[(long long)r * P.rows_stride + i] = __float2bfloat16_rn(0.f);
    }
}

template <bool kSort>
static void gather_launch(const GatherParams& g, cudaStream_t s)
{
    if (g.N <= 16384) launch_pdl(lm_head_gather_kernel<8, kSort>, dim3((g.N + 7) / 8), dim3(kGatherThreads), 0, s, g);
    else launch_pdl(lm_head_gather_kernel<32, kSort>, dim3((g.N + 31) / 32), dim3(kGatherThreads), 0, s, g);
}

// ---- loss of every row from the statistics of the vocabulary tiles --------------------------------------
// Eight rows per CTA, 128 threads per row, each taking every 128th entry (eight loads in flight; ten: no faster): at
// V = 129 280 a row has 1 010 to 1 156 entries.  loss = log(1 + T e^(R - z)), lse = z + loss, with z the label's logit and T = sum s_i e^(r_i - R) over the
// other entries, R the largest r_i; the sum over threads and the rest in 64 bits.
struct LossParams {
    const float2* stats; long long stats_stride; int entries;
    const float* z_label; const int32_t* idx; const int32_t* live;
    float* loss; float* lse; int32_t* dev_status;
};
constexpr int kLossRows = 8, kLossThreads = 1024, kLossPer = 8;

__global__ void __launch_bounds__(kLossThreads) lm_head_loss_kernel(const __grid_constant__ LossParams P)
{
    __shared__ float s_ref[kLossThreads / 32][kLossRows];
    __shared__ double s_sum[kLossThreads / 32][kLossRows];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x * kLossRows + (lane & 7), live = *P.live;
    if (blockIdx.x * kLossRows >= live) return;
    const int first = (int)threadIdx.x >> 3;
    const int at = row < live ? P.idx[row] : 0;
    const double z = row < live ? P.z_label[row] : 0.f;
    float ref = -INFINITY, sum = 0.f;
    for (int e0 = first; e0 < P.entries; e0 += 128 * kLossPer) {
        float2 v[kLossPer];
        float now = ref;
#pragma unroll
        for (int i = 0; i < kLossPer; ++i) {
            const int e = e0 + 128 * i;
            v[i] = e < P.entries && row < live ? P.stats[(size_t)e * P.stats_stride + row] : make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int i = 0; i < kLossPer; ++i) now = fmaxf(now, v[i].x);
        const float base = now == -INFINITY ? 0.f : now;
        sum *= ex2_approx((ref - base) * kLog2e);
#pragma unroll
        for (int i = 0; i < kLossPer; ++i) sum = fmaf(v[i].y, ex2_approx((v[i].x - base) * kLog2e), sum);
        ref = now;
    }
    float top = ref;
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    double part = (double)(sum * ex2_approx((ref - (top == -INFINITY ? 0.f : top)) * kLog2e));
    part += __shfl_xor_sync(0xffffffffu, part, 8);
    part += __shfl_xor_sync(0xffffffffu, part, 16);
    if (lane < kLossRows) { s_ref[warp][lane] = top; s_sum[warp][lane] = part; }
    __syncthreads();
    if (warp || lane >= kLossRows || row >= live) return;
    top = -INFINITY;
    for (int w = 0; w < kLossThreads / 32; ++w) top = fmaxf(top, s_ref[w][lane]);
    const float base = top == -INFINITY ? 0.f : top;
    double total = 0.0;
    for (int w = 0; w < kLossThreads / 32; ++w) total += s_sum[w][lane] * (double)ex2_approx((s_ref[w][lane] - base) * kLog2e);
    // `total` e^base is the sum over the other entries (none of them: 0); z - z is not a number when z is none or not finite
    const double shift = total == 0.0 ? 0.0 : base - z;
    const double loss = (z - z) + (shift > 0.0 ? shift + log(total + exp(-shift)) : log1p(total * exp(shift)));
    P.loss[at] = (float)loss;
    P.lse[at] = (float)(z + loss);
    if (!(fabsf((float)loss) < INFINITY)) atomicOr(P.dev_status, DSPARK_DEV_BAD_ROW);      // as it is stored
}

// ---- gradient of the hidden states from the slices' partial sums ---------------------------------------
// The label's entry of G is most of the row: what its rounding to bf16 lost is added back here, times the label's row of
// W.  The sum runs over the slices in order: the same bits every time.
struct HiddenParams {
    const float* part; long long part_stride; int slices, m;
    const float* label_err; const int32_t* label; const int32_t* idx; const int32_t* live;
    const __nv_bfloat16* w; long long w_stride;
    int d;
    __nv_bfloat16* dh; long long dh_stride;
};
constexpr int kHiddenThreads = 128;               // four columns each
__global__ void __launch_bounds__(kHiddenThreads) lm_head_grad_hidden_kernel(const __grid_constant__ HiddenParams P)
{
    pdl_wait();
    const int row = blockIdx.x;
    if (row >= *P.live) return;
    const int c = (int)(blockIdx.y * kHiddenThreads + threadIdx.x) * 4;
    if (c >= P.d) return;
    const float* part = P.part + (long long)row * P.part_stride + c;       // the pitch is a multiple of 8
    const long long step = (long long)P.m * P.part_stride;
    const float err = P.label_err[row];
    const __nv_bfloat16* w = P.w + (long long)P.label[row] * P.w_stride + c;
    __nv_bfloat16* out = P.dh + (long long)P.idx[row] * P.dh_stride + c;
    float at_label[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) at_label[i] = c + i < P.d ? __bfloat162float(w[i]) : 0.f;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 16
    for (int s = 0; s < P.slices; ++s) {
        const float4 v = *reinterpret_cast<const float4*>(part + s * step);
        sum[0] += v.x; sum[1] += v.y; sum[2] += v.z; sum[3] += v.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < P.d) out[i] = __float2bfloat16_rn(fmaf(err, at_label[i], sum[i]));
}

// ---- int8 weights ------------------------------------------------------------------------------------------
// One row (a vocabulary entry) per CTA: q = rint(127 w / max|w|), scale = max|w| / 127.
__global__ void __launch_bounds__(256) lm_head_quantize_kernel(const __nv_bfloat16* __restrict__ W, long long w_stride, int K,
                                                               int8_t* __restrict__ q, long long q_stride, float* __restrict__ scale)
{
    __shared__ float s_top[8];
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const __nv_bfloat16* w = W + (long long)blockIdx.x * w_stride;
    int8_t* out = q + (long long)blockIdx.x * q_stride;
    float top = 0.f;
    for (int i = tid; i < K; i += 256) {
        const float a = fabsf(__bfloat162float(w[i]));
        top = (a > top || a != a) ? a : top;
    }
    const bool bad = __syncthreads_or(!(top < INFINITY)) != 0;
    top = warp_max_f32(top);
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, s_top[i]);
    // above, 127 w passes the range: 127 and the maximum 2^16 smaller there
    const float up = top > 1e36f ? 127.f * 0x1p-16f : 127.f, by = top > 1e36f ? top * 0x1p-16f : top;
    for (int i = tid; i < K; i += 256) {
        // 127 w has 15 significant bits: the correctly rounded quotient keeps a half a half
        const float v = (bad || top == 0.f) ? 0.f : rintf(__fdiv_rn(up * __bfloat162float(w[i]), by));
        out[i] = (int8_t)v;
    }
    if (tid == 0) scale[blockIdx.x] = bad ? NAN : top / 127.f;
}

// ---- host side ---------------------------------------------------------------------------------------------
static size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }

// 2-D operand [rows, cols] of `es`-byte elements; boxes of box_cols x box_rows, 128-byte swizzle, zeros outside
static bool operand_map(CUtensorMap* map, const void* base, int es, long long rows, long long cols, long long pitch_bytes, int box_cols, int box_rows)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, es == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
              strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same matrix by blocks of 64 columns, [block][row][64]: one copy brings `blocks` mn-major boxes of `box_rows` rows that
// lie behind one another in shared memory.  The columns of the last block past `cols` are read: the matrix has them.
static bool block_map(CUtensorMap* map, const void* base, long long rows, long long cols, long long pitch_bytes, int box_rows, int blocks)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)((cols + 63) / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch_bytes, 128};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, (cuuint32_t)blocks};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int device_sms()
{
    static std::atomic<int> sms[64];
    int dev = 0;
    cudaGetDevice(&dev);
    int v = sms[dev & 63].load(std::memory_order_relaxed);
    if (!v) {
        cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
        sms[dev & 63].store(v, std::memory_order_relaxed);
    }
    return v;
}

// the dynamic shared memory of a kernel, once per device
template <typename Kernel>
static bool allow_smem(Kernel kernel, int bytes, std::atomic<unsigned long long>& ready)
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

// launch_pdl with clusters of kCtas CTAs
template <int kCtas, typename... KArgs, typename... Args>
static void launch_pairs(void (*kernel)(KArgs...), int ctas, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kHeadThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCtas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kCtas > 1 ? 2 : 1;
    cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int kMode, int kCtas>
static int head_launch(HeadParams P, const CUtensorMap& a, const CUtensorMap& b, cudaStream_t s, int timer_id)
{
    constexpr int kSmem = kHeadRingBytes + 1024 + (kMode == kInt8Logits ? kHeadN * 16 : 0);   // four lane quarters x 256 scales
    static std::atomic<unsigned long long> ready{0};
    if (!allow_smem(lm_head_kernel<kMode, kCtas>, kSmem, ready)) return launch_status();
    P.stages = kHeadRingBytes / (kTileABytes + P.n_tile / kCtas * kRowBytes);
    if (P.stages > kHeadMaxStages) P.stages = kHeadMaxStages;
    const long long units = (long long)((P.m + kCtas * kHeadM - 1) / (kCtas * kHeadM)) * ((P.n + P.n_tile - 1) / P.n_tile);
    const int groups = device_sms() / kCtas;
    KernelTimerScope timer(timer_id, s);
    launch_pairs<kCtas>(lm_head_kernel<kMode, kCtas>, kCtas * (int)(units < groups ? units : groups), kSmem, s, P, a, b);
    return launch_status();
}

template <int kCtas>
static int back_launch(const BackParams& P, const BackMaps& M, cudaStream_t s)
{
    constexpr int kSmem = kHeadRingBytes + 1024 + kHeadEpiWarps * kTurnBytes;
    static std::atomic<unsigned long long> ready{0};
    if (!allow_smem(lm_head_backward_kernel<kCtas>, kSmem, ready)) return launch_status();
    KernelTimerScope timer(DSPARK_K_HEAD_GRAD, s);
    launch_pairs<kCtas>(lm_head_backward_kernel<kCtas>, device_sms() / kCtas * kCtas, kSmem, s, P, M);
    return launch_status();
}

// A B200's.  Not asked of the device: the size of the workspace is known without one, and the same everywhere.
constexpr int kSms = 148;
constexpr int kMaxRows = 1 << 20, kMaxVocab = 1 << 24, kMaxWidth = 1 << 16;
constexpr long long kPieceBytes = 32ll << 20;

struct LossWs {
    size_t live, sync, first, idx, label, at_label, lse, grad, label_err, rows, stats, G, part, total;
    long long n_pad, d_pitch, part_pitch;
    int ctas, n_tile, piece, pieces, n_sync, slices, kb_slice, n_tile_d, d_tiles;
};
static LossWs loss_layout(int N, int V, int d)
{
    LossWs w;
    w.ctas = N > kHeadM ? 2 : 1;                            // one row tile of 128 rows: the second CTA of a pair would hold none
    w.n_pad = (long long)up((size_t)N, w.ctas * kHeadM);
    // Vocabulary entries of a tile of the statistics: for up to 128 rows narrower than 256 where few rounds of tiles over the
    // SMs leave many of them idle in the last one, by at least 1/16.  256 / this rule, us: 64 rows V 129 280 d 1024 57.8 /
    // 55.7, V 151 936 68.8 / 65.7, V 50 257 d 768 27.2 / 25.7, V 10 007 d 500 14.3 / 13.0.  (Pairs read B once for both rows
    // of tiles and lose by it: 600 rows V 40 000 d 300 32.8 / 43.6.)
    auto rounds = [&](int tile) { return ((V + tile - 1) / tile + kSms - 1) / kSms * tile; };
    w.n_tile = kHeadN;
    for (int tile = kHeadN - 32; w.ctas == 1 && tile >= 128; tile -= 32)
        if (rounds(tile) * 16ll <= rounds(w.n_tile) * 15ll) w.n_tile = tile;
    w.d_pitch = (long long)up((size_t)d, 64);               // whole blocks of columns (block_map)
    w.part_pitch = (long long)up((size_t)d, 8);
    w.n_tile_d = d >= kHeadN ? kHeadN : (int)up((size_t)d, 64 * w.ctas);
    w.d_tiles = (d + w.n_tile_d - 1) / w.n_tile_d;
    // A piece of the vocabulary: at most 32 MB of G and 128 MB of W, so that the three pieces of G stay in or near the L2
    // and few rows (G small) do not make pieces whose phases are shorter than the waits between them; not narrower than
    // 2 048 entries, below which adding the partial sums of dH would cost more than the products.  Measured with 16 / 32 /
    // 64 MB: 128 rows, d 1024 221 / 206 / 205 us; 1000 rows, d 1024 727 / 681 / 662; 2867 rows, d 2048 3465 / 3436 / 3304
    // (twice the workspace); 600 rows, V 40 000, d 300 174 / 154 / 166.
    const long long all = (long long)up((size_t)V, kHeadN);
    long long piece = kPieceBytes / (2 * w.n_pad) / kHeadN * kHeadN;
    const long long by_w = 4 * kPieceBytes / (2 * d) / kHeadN * kHeadN;
    if (piece > by_w) piece = by_w;
    if (piece < 2048) piece = 2048;
    if (piece > all) piece = all;
    w.piece = (int)piece;
    w.pieces = (int)((V + piece - 1) / piece);
    w.n_sync = 1 + 3 * w.pieces;
    // k blocks of the units of one piece, over the SMs: a slice of dH's sum over the piece is at most half of an SM's share
    const long long m_tiles = w.n_pad / (w.ctas * kHeadM), blocks = piece / 64;
    const long long work = 2 * m_tiles * w.d_tiles * blocks + m_tiles * (piece / kHeadN) * ((d + 63) / 64);
    long long most = work / (2 * kSms / w.ctas);
    if (most < 8) most = 8;
    long long slices = (blocks + most - 1) / most;
    if (slices > 64) slices = 64;
    w.kb_slice = (int)((blocks + slices - 1) / slices);
    w.slices = (int)((blocks + w.kb_slice - 1) / w.kb_slice);

    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += up(bytes, 256); return at; };
    w.live = take(4);
    w.sync = take(4 * (size_t)w.n_sync);
    w.first = take(4 * (size_t)V);
    w.idx = take(4 * (size_t)w.n_pad); w.label = take(4 * (size_t)w.n_pad); w.at_label = take(4 * (size_t)w.n_pad);
    w.lse = take(4 * (size_t)w.n_pad); w.grad = take(4 * (size_t)w.n_pad); w.label_err = take(4 * (size_t)w.n_pad);
    w.rows = take(2 * (size_t)w.n_pad * (size_t)w.d_pitch);
    const size_t common = o;
    // forward: two entries per vocabulary tile and row
    w.stats = take((size_t)kHeadParts * up((size_t)V, w.n_tile) / w.n_tile * (size_t)w.n_pad * sizeof(float2));
    const size_t forward = o;
    // backward: three pieces of G, the slices' sums
    o = common;
    w.G = take(3 * 2 * (size_t)w.n_pad * (size_t)piece);
    w.part = take(4 * (size_t)w.slices * (size_t)w.n_pad * (size_t)w.part_pitch);
    w.total = o > forward ? o : forward;
    return w;
}

static int loss_check(const void* hidden, int64_t h_stride, const void* weight, int64_t w_stride, const void* labels, int N, int V, int d,
                      const void* dev_status, const void* workspace, size_t workspace_bytes, const LossWs& w)
{
    if (!hidden || !weight || !labels || !dev_status || h_stride < d || w_stride < d) return DSPARK_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < w.total) return DSPARK_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) || ((uintptr_t)hidden & 1u) || ((uintptr_t)weight & 15u) || (w_stride & 7) || ((uintptr_t)labels & 3u))
        return DSPARK_ERR_ALIGNMENT;
    return DSPARK_OK;
}

// Both backward calls; loss NULL: the label's entry of G from lse.
static int loss_backward(const void* hidden, int64_t hidden_row_stride, const void* weight, int64_t weight_row_stride,
                         const int32_t* labels, const float* lse, const float* loss, const float* grad_loss, int N, int V, int d,
                         void* out_grad_hidden, int64_t grad_hidden_row_stride, void* out_grad_weight,
                         int64_t grad_weight_row_stride, int32_t* dev_status, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!lse || !grad_loss || (!out_grad_hidden && !out_grad_weight) || N < 1 || V < 1 || d < 1) return DSPARK_ERR_INVALID_ARG;
    if ((out_grad_hidden && grad_hidden_row_stride < d) || (out_grad_weight && grad_weight_row_stride < d)) return DSPARK_ERR_INVALID_ARG;
    if (N > kMaxRows || V > kMaxVocab || d > kMaxWidth) return DSPARK_ERR_SHAPE;
    const LossWs w = loss_layout(N, V, d);
    const int rc0 = loss_check(hidden, hidden_row_stride, weight, weight_row_stride, labels, N, V, d, dev_status, workspace, workspace_bytes, w);
    if (rc0 != DSPARK_OK) return rc0;
    if ((((uintptr_t)lse | (uintptr_t)loss | (uintptr_t)grad_loss) & 3u) || (((uintptr_t)out_grad_hidden | (uintptr_t)out_grad_weight) & 1u))
        return DSPARK_ERR_ALIGNMENT;
    unsigned char* ws = (unsigned char*)workspace;
    cudaStream_t s = (cudaStream_t)stream;
    GatherParams g;
    memset(&g, 0, sizeof g);
    g.h = (const __nv_bfloat16*)hidden; g.h_stride = hidden_row_stride; g.labels = labels; g.N = N; g.V = V; g.d = d;
    g.rows = (__nv_bfloat16*)(ws + w.rows); g.rows_stride = w.d_pitch;
    g.live = (int32_t*)(ws + w.live); g.idx = (int32_t*)(ws + w.idx); g.label = (int32_t*)(ws + w.label);
    g.lse_in = lse; g.loss_in = loss; g.grad_in = grad_loss; g.lse = (float*)(ws + w.lse); g.grad = (float*)(ws + w.grad);
    g.w = (const __nv_bfloat16*)weight; g.w_stride = weight_row_stride;
    g.at_label = (float*)(ws + w.at_label); g.label_err = (float*)(ws + w.label_err);
    g.sync = (int32_t*)(ws + w.sync); g.n_sync = w.n_sync; g.first = (int32_t*)(ws + w.first);
    g.dh = (__nv_bfloat16*)out_grad_hidden; g.dh_stride = grad_hidden_row_stride; g.dev_status = dev_status;
    {
        KernelTimerScope timer(DSPARK_K_HEAD_ROWS, s);
        gather_launch<true>(g, s);
    }
    BackMaps M;
    const int box_v = V < kHeadN / w.ctas ? V : kHeadN / w.ctas;
    const long long g_pitch = (long long)w.piece * 2;
    if (!operand_map(&M.rows_k, g.rows, 2, w.n_pad, d, w.d_pitch * 2, 64, kHeadM) ||
        !operand_map(&M.w_k, weight, 2, V, d, weight_row_stride * 2, 64, box_v) ||
        !operand_map(&M.g_k, ws + w.G, 2, 3 * w.n_pad, w.piece, g_pitch, 64, kHeadM) ||
        !(d % 64 == 0 ? block_map(&M.w_mn, weight, V, d, weight_row_stride * 2, 64, w.n_tile_d / w.ctas / 64)
                      : operand_map(&M.w_mn, weight, 2, V, d, weight_row_stride * 2, 64, 64)) ||
        !block_map(&M.g_mn, ws + w.G, 3 * w.n_pad, w.piece, g_pitch, 64, kHeadM / 64) ||
        !block_map(&M.rows_mn, g.rows, w.n_pad, d, w.d_pitch * 2, 64, w.n_tile_d / w.ctas / 64))
        return DSPARK_ERR_CUDA;
    BackParams P;
    memset(&P, 0, sizeof P);
    P.n_pad = (int)w.n_pad; P.V = V; P.d = d;
    P.piece = w.piece; P.pieces = w.pieces; P.n_tile_d = w.n_tile_d; P.d_tiles = w.d_tiles;
    P.slices = w.slices; P.kb_slice = w.kb_slice;
    P.box_v = box_v; P.w_blocks = d % 64 == 0;
    P.want_h = out_grad_hidden != nullptr; P.want_w = out_grad_weight != nullptr;
    P.live = g.live; P.dev_status = dev_status; P.sync = g.sync;
    P.G = (__nv_bfloat16*)(ws + w.G);
    P.labels = g.label; P.lse2 = g.lse; P.grad = g.grad; P.at_label = g.at_label; P.label_err = g.label_err;
    P.first = g.first; P.rows = g.rows; P.rows_stride = w.d_pitch;
    P.part = (float*)(ws + w.part); P.part_stride = w.part_pitch;
    P.dw = (__nv_bfloat16*)out_grad_weight; P.dw_stride = grad_weight_row_stride;
    const int rc = w.ctas == 2 ? back_launch<2>(P, M, s) : back_launch<1>(P, M, s);
    if (rc != DSPARK_OK) return rc;
    if (out_grad_hidden) {
        HiddenParams Hp;
        Hp.part = (const float*)(ws + w.part); Hp.part_stride = w.part_pitch; Hp.slices = w.slices; Hp.m = (int)w.n_pad;
        Hp.label_err = g.label_err; Hp.label = g.label; Hp.idx = g.idx; Hp.live = g.live;
        Hp.w = (const __nv_bfloat16*)weight; Hp.w_stride = weight_row_stride; Hp.d = d;
        Hp.dh = g.dh; Hp.dh_stride = grad_hidden_row_stride;
        KernelTimerScope timer(DSPARK_K_HEAD_ROWS, s);
        launch_pdl(lm_head_grad_hidden_kernel, dim3(N, (d + 4 * kHiddenThreads - 1) / (4 * kHiddenThreads)), dim3(kHiddenThreads), 0, s, Hp);
    }
    return launch_status();
}

}  // namespace dspark

using namespace dspark;

extern "C" {

int dspark_lm_head_quantize(const void* W, int64_t w_row_stride, int V, int K, int8_t* out_q, int64_t out_q_row_stride,
                            float* out_scale, void* stream)
{
    if (!W || !out_q || !out_scale || V < 1 || K < 1 || w_row_stride < K || out_q_row_stride < K) return DSPARK_ERR_INVALID_ARG;
    if (((uintptr_t)W & 1u) || ((uintptr_t)out_scale & 3u)) return DSPARK_ERR_ALIGNMENT;
    launch_pdl(lm_head_quantize_kernel, dim3(V), dim3(256), 0, (cudaStream_t)stream, (const __nv_bfloat16*)W, (long long)w_row_stride, K,
               out_q, (long long)out_q_row_stride, out_scale);
    return launch_status();
}

int dspark_lm_head_int8(const int8_t* x_q, int64_t x_row_stride, const float* x_scale, const int8_t* w_q, int64_t w_row_stride,
                        const float* w_scale, int rows, int V, int K, const int32_t* n_live, void* out_logits, int out_dtype,
                        int64_t out_row_stride, int32_t* dev_status, void* stream)
{
    if (!x_q || !x_scale || !w_q || !w_scale || !out_logits || !dev_status || rows < 1 || V < 1 || K < 1) return DSPARK_ERR_INVALID_ARG;
    if (out_dtype != DSPARK_F32 && out_dtype != DSPARK_BF16) return DSPARK_ERR_INVALID_ARG;
    if (x_row_stride < K || w_row_stride < K || out_row_stride < V) return DSPARK_ERR_INVALID_ARG;
    if (rows > kMaxRows || V > kMaxVocab || K > kMaxWidth) return DSPARK_ERR_SHAPE;
    if (((uintptr_t)x_q & 15u) || ((uintptr_t)w_q & 15u) || (x_row_stride & 15) || (w_row_stride & 15) || ((uintptr_t)x_scale & 3u) ||
        ((uintptr_t)w_scale & 3u) || ((uintptr_t)out_logits & (out_dtype == DSPARK_BF16 ? 1u : 3u)) || ((uintptr_t)n_live & 3u))
        return DSPARK_ERR_ALIGNMENT;
    HeadParams P;
    memset(&P, 0, sizeof P);
    P.m = V; P.n = rows; P.k = K;
    // Pairs where the copies from the L2 bound the call, single CTAs where the weight's bytes or the stores do, or the call is
    // too short for the 3 us that a launch of pairs takes longer.  Single / pair, us: V = 129 280, K 512 256 rows 33 / 32,
    // 1482 rows 136 / 137; K 768 256 rows 39 / 36, 1482 rows 168 / 164; K 1024 129 rows 35 / 35, 256 rows 46 / 39, 352 rows
    // (pairs' tiles are multiples of 32) 60 / 62, 500 rows 75 / 69, 1482 rows 201 / 185; K 4096 1482 rows 732 / 591.
    // V = 32 000, K 1024 256 rows 18 / 20, 500 rows 26 / 23; K 1040 200 rows 25.5 / 19.8; K 1536 129 rows 18 / 17, 512 rows
    // 28.3 / 26.6; V = 16 000, K 1024 512 rows 16 / 16, K 2048 256 rows 13.5 / 13.1.  V is not asked for beyond K 1024: where
    // there are few tiles an SM, pairs lose up to 2 us -- K 1536 V 1000 200 rows 8.2 / 9.3, K 2048 V 10 007 200 rows
    // 11.4 / 12.3, 512 rows 19.8 / 18.5, K 4096 V 1000 129 rows 13.3 / 15.4, V 10 007 129 rows 14.7 / 16.0.
    // Both choices go by the rows there is room for, since the count is on the device: 576 rows of which 1 counts, K 1024
    // 32.5 us (a call for 1 row 29.2), K 4096 97 (83); 192 of 576 as a call for 192.
    const int ctas = rows > kHeadM && (K > 1024 || (K >= 768 && (double)rows * V * K > 1.2e10)) ? 2 : 1;
    // row tiles of one size, and no taller a box than there are rows (one row of 32 in a box: 170 us instead of 84 at
    // K = 4 096)
    const int row_tiles = (rows + kHeadN - 1) / kHeadN;
    P.n_tile = (int)up((size_t)((rows + row_tiles - 1) / row_tiles), 16 * ctas);
    P.box_n = rows < P.n_tile / ctas ? rows : P.n_tile / ctas;
    P.live = n_live; P.dev_status = dev_status;
    P.out = out_logits; P.out_stride = out_row_stride; P.out_bf16 = out_dtype != DSPARK_BF16 ? 0 : (((uintptr_t)out_logits & 3u) == 0 && (out_row_stride & 1) == 0) ? 2 : 1;
    P.row_scale = x_scale; P.col_scale = w_scale;
    CUtensorMap a, b;
    if (!operand_map(&a, w_q, 1, V, K, w_row_stride, kRowBytes, kHeadM) || !operand_map(&b, x_q, 1, rows, K, x_row_stride, kRowBytes, P.box_n))
        return DSPARK_ERR_CUDA;
    return ctas == 2 ? head_launch<kInt8Logits, 2>(P, a, b, (cudaStream_t)stream, DSPARK_K_HEAD_INT8)
                     : head_launch<kInt8Logits, 1>(P, a, b, (cudaStream_t)stream, DSPARK_K_HEAD_INT8);
}

size_t dspark_lm_head_loss_workspace_bytes(int N, int V, int d)
{
    if (N < 1 || V < 1 || d < 1 || N > kMaxRows || V > kMaxVocab || d > kMaxWidth) return 0;
    // The layout of fewer rows may be larger (longer pieces, more slices of dH's sums), so the answer is the largest over all
    // row counts up to N.  A layout depends on the rows only through n_pad, and through one row tile or pairs of them.
    size_t most = loss_layout(N, V, d).total;
    for (int n = kHeadM; n < N; n += n == kHeadM ? kHeadM : 2 * kHeadM) {
        const size_t bytes = loss_layout(n, V, d).total;
        if (bytes > most) most = bytes;
    }
    return most;
}

int dspark_lm_head_loss(const void* hidden, int64_t hidden_row_stride, const void* weight, int64_t weight_row_stride,
                        const int32_t* labels, int N, int V, int d, float* out_loss, float* out_lse, int32_t* dev_status,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    if (!out_loss || !out_lse || N < 1 || V < 1 || d < 1) return DSPARK_ERR_INVALID_ARG;
    if (N > kMaxRows || V > kMaxVocab || d > kMaxWidth) return DSPARK_ERR_SHAPE;
    const LossWs w = loss_layout(N, V, d);
    const int rc0 = loss_check(hidden, hidden_row_stride, weight, weight_row_stride, labels, N, V, d, dev_status, workspace, workspace_bytes, w);
    if (rc0 != DSPARK_OK) return rc0;
    if (((uintptr_t)out_loss | (uintptr_t)out_lse) & 3u) return DSPARK_ERR_ALIGNMENT;
    unsigned char* ws = (unsigned char*)workspace;
    cudaStream_t s = (cudaStream_t)stream;
    GatherParams g;
    memset(&g, 0, sizeof g);
    g.h = (const __nv_bfloat16*)hidden; g.h_stride = hidden_row_stride; g.labels = labels; g.N = N; g.V = V; g.d = d;
    g.rows = (__nv_bfloat16*)(ws + w.rows); g.rows_stride = w.d_pitch;
    g.live = (int32_t*)(ws + w.live); g.idx = (int32_t*)(ws + w.idx); g.label = (int32_t*)(ws + w.label);
    g.loss = out_loss; g.lse = out_lse; g.dev_status = dev_status;
    {
        KernelTimerScope timer(DSPARK_K_HEAD_ROWS, s);
        gather_launch<false>(g, s);
    }
    HeadParams P;
    memset(&P, 0, sizeof P);
    P.m = N; P.n = V; P.k = d;
    P.n_tile = w.n_tile; P.box_n = V < w.n_tile / w.ctas ? V : w.n_tile / w.ctas;
    P.live = g.live; P.dev_status = dev_status;
    P.stats = (float2*)(ws + w.stats); P.stats_stride = w.n_pad; P.labels = g.label; P.z_label = (float*)(ws + w.at_label);
    P.rows = g.rows; P.rows_stride = w.d_pitch; P.w = (const __nv_bfloat16*)weight; P.w_stride = weight_row_stride;
    CUtensorMap a, b;
    if (!operand_map(&a, g.rows, 2, w.n_pad, d, w.d_pitch * 2, 64, kHeadM) || !operand_map(&b, weight, 2, V, d, weight_row_stride * 2, 64, P.box_n))
        return DSPARK_ERR_CUDA;
    const int rc = w.ctas == 2 ? head_launch<kLossStats, 2>(P, a, b, s, DSPARK_K_HEAD_LOSS) : head_launch<kLossStats, 1>(P, a, b, s, DSPARK_K_HEAD_LOSS);
    if (rc != DSPARK_OK) return rc;
    LossParams L;
    L.stats = P.stats; L.stats_stride = w.n_pad; L.entries = kHeadParts * ((V + w.n_tile - 1) / w.n_tile);
    L.z_label = P.z_label; L.idx = g.idx; L.live = g.live; L.loss = out_loss; L.lse = out_lse; L.dev_status = dev_status;
    {
        KernelTimerScope timer(DSPARK_K_HEAD_ROWS, s);
        launch_pdl(lm_head_loss_kernel, dim3((N + kLossRows - 1) / kLossRows), dim3(kLossThreads), 0, s, L);
    }
    return launch_status();
}

int dspark_lm_head_loss_backward(const void* hidden, int64_t hidden_row_stride, const void* weight, int64_t weight_row_stride,
                                 const int32_t* labels, const float* lse, const float* grad_loss, int N, int V, int d,
                                 void* out_grad_hidden, int64_t grad_hidden_row_stride, void* out_grad_weight,
                                 int64_t grad_weight_row_stride, int32_t* dev_status, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    return loss_backward(hidden, hidden_row_stride, weight, weight_row_stride, labels, lse, nullptr, grad_loss, N, V, d, out_grad_hidden,
                         grad_hidden_row_stride, out_grad_weight, grad_weight_row_stride, dev_status, workspace, workspace_bytes, stream);
}

int dspark_lm_head_loss_backward_from_loss(const void* hidden, int64_t hidden_row_stride, const void* weight, int64_t weight_row_stride,
                                           const int32_t* labels, const float* lse, const float* loss, const float* grad_loss, int N,
                                           int V, int d, void* out_grad_hidden, int64_t grad_hidden_row_stride, void* out_grad_weight,
                                           int64_t grad_weight_row_stride, int32_t* dev_status, void* workspace,
                                           size_t workspace_bytes, void* stream)
{
    if (!loss) return DSPARK_ERR_INVALID_ARG;
    return loss_backward(hidden, hidden_row_stride, weight, weight_row_stride, labels, lse, loss, grad_loss, N, V, d, out_grad_hidden,
                         grad_hidden_row_stride, out_grad_weight, grad_weight_row_stride, dev_status, workspace, workspace_bytes, stream);
}

}  // extern "C"
