// dspark_tree_attention: attention of a step's nodes (trees or chains of drafted tokens) over the paged cache.
//
//     out[i] = sum_t w_t v_t,  w = softmax_t(scale q_i . k_t) over the positions before the step, node i and its ancestors.
//
// One warp per row and head, one pass over the positions with the running maximum and sum of the softmax.
#include <math.h>

#include "kv_cache.cuh"

namespace dspark {

constexpr int kAttnMaxDim = 128;

struct AttnParams {
    KvView c;
    const unsigned char* q; long long q_row, q_head;          // bytes
    unsigned char* out; long long out_row, out_head;
    float* out_lse;
    const int32_t* first; const int32_t* row_offsets; const int32_t* parents;
    int R, n_rows, q_heads, group;
    float scale;
    int32_t* dev_status;
};

__device__ __forceinline__ float kv_element(const KvView& c, const unsigned char* base, const float* scales, int page, int token, int head, int i)
{
    const unsigned char* p = base + page * c.page_stride + token * c.token_stride + head * c.head_stride;
    if (c.dtype == DSPARK_BF16) return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
    const float s = scales[((long long)page * c.kv_heads + head) * c.page_size + token];
    if (c.dtype == DSPARK_I8) return (float)(int8_t)p[i] * s;
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)p[i]));
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)h));
    return f * s;
}

__global__ void __launch_bounds__(256) attn_rows_kernel(const __grid_constant__ AttnParams P)
{
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x == 0) kv_report(P.first, P.row_offsets, P.R, P.n_rows, kv_capacity(P.c), P.dev_status);
    const long long item = (long long)blockIdx.x * 8 + warp;
    const int row = (int)(item / P.q_heads), h = (int)(item % P.q_heads), kvh = h / P.group;
    if (row >= P.n_rows) return;
    int lo = 0, hi = P.R;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (P.row_offsets[mid + 1] <= row) lo = mid + 1; else hi = mid;
    }
    if (lo >= P.R) return;
    const KvRequest rq = kv_request(P.first, P.row_offsets, lo, P.n_rows, kv_capacity(P.c));
    if (rq.n < 0 || row < rq.row0) return;
    const int d = P.c.head_dim, self = row - rq.row0;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    const uint16_t* qr = reinterpret_cast<const uint16_t*>(P.q + row * P.q_row + h * P.q_head);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = i * 32 + lane < d ? __uint_as_float((uint32_t)qr[i * 32 + lane] << 16) : 0.f;
    auto position = [&](int t) {
        const int page = P.c.block_table[lo * P.c.table_stride + t / P.c.page_size], token = t % P.c.page_size;
        const bool there = page >= 0 && page < P.c.n_pages;
        if (!there && lane == 0) atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);
        float s = 0.f, v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = there && i * 32 + lane < d;
            s = fmaf(q[i], in ? kv_element(P.c, P.c.k, P.c.k_scale, page, token, kvh, i * 32 + lane) : 0.f, s);
            v[i] = in ? kv_element(P.c, P.c.v, P.c.v_scale, page, token, kvh, i * 32 + lane) : 0.f;
        }
        s = warp_sum_f32(s) * P.scale;
        const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top, f = expf(m - ref), w = expf(s - ref);
        l = l * f + w;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f + w * v[i];
        m = top;
    };
    for (int t = 0; t < rq.first; ++t) position(t);
    if (!P.parents) {
        for (int i = 0; i <= self; ++i) position(rq.first + i);
    } else {
        int node = self;
        while (true) {
            position(rq.first + node);
            if (node == 0) break;
            const int parent = P.parents[rq.row0 + node];
            if (parent < 0 || parent >= node) {
                if (lane == 0) atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE);
                break;
            }
            node = parent;
        }
    }
    uint16_t* out = reinterpret_cast<uint16_t*>(P.out + row * P.out_row + h * P.out_head);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 32 + lane < d) {
            uint32_t b;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(0.f), "f"(o[i] / l));
            out[i * 32 + lane] = (uint16_t)b;
        }
    if (P.out_lse && lane == 0) P.out_lse[(long long)row * P.q_heads + h] = m + logf(l);
}

}  // namespace dspark

extern "C" {

size_t dspark_tree_attention_workspace_bytes(int n_rows, int q_heads, int kv_heads, int head_dim)
{
    if (n_rows < 1 || q_heads < 1 || kv_heads < 1 || head_dim < 1) return 0;
    return 256;
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
    if (!workspace || workspace_bytes < dspark_tree_attention_workspace_bytes(n_rows, q_heads, cache->kv_heads, d)) return DSPARK_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255) return DSPARK_ERR_ALIGNMENT;
    AttnParams P = {};
    P.c = kv_view(cache, layer);
    P.q = (const unsigned char*)q; P.q_row = q_row_stride * 2; P.q_head = q_head_stride * 2;
    P.out = (unsigned char*)out; P.out_row = out_row_stride * 2; P.out_head = out_head_stride * 2;
    P.out_lse = out_lse;
    P.first = first; P.row_offsets = row_offsets; P.parents = parents;
    P.R = R; P.n_rows = n_rows; P.q_heads = q_heads; P.group = q_heads / cache->kv_heads;
    P.scale = scale; P.dev_status = dev_status;
    KernelTimerScope timer(DSPARK_K_TREE_ATTENTION, (cudaStream_t)stream);
    launch_pdl(attn_rows_kernel, dim3((unsigned)(((long long)n_rows * q_heads + 7) / 8)), dim3(256), 0, (cudaStream_t)stream, P);
    return launch_status();
}

}  // extern "C"
