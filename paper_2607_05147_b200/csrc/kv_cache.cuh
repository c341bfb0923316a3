// The paged cache and the ragged step as the kernels see them, and the host's checks of both.
#pragma once

#include <math.h>

#include "common.cuh"

namespace dspark {

// One layer of the cache.
struct KvView {
    unsigned char* k; unsigned char* v;
    float* k_scale; float* v_scale;             // [n_pages][kv_heads][page_size]
    int dtype, n_pages, page_size, kv_heads, head_dim, max_pages;
    int page_shift;                             // log2 of page_size, or -1
    long long page_stride, token_stride, head_stride;      // bytes
    const int32_t* block_table; long long table_stride;
};

// The rows of a request and the tokens before them.  n < 0: the request is left alone, `status` says why.
struct KvRequest { int row0, n, first, status; };

__device__ __forceinline__ KvRequest kv_request(const int32_t* first, const int32_t* row_offsets, int r, int n_rows, long long capacity)
{
    KvRequest q;
    q.row0 = row_offsets[r];
    const int end = row_offsets[r + 1];
    q.first = first[r];
    q.n = end - q.row0;
    q.status = 0;
    if (q.row0 < 0 || end < q.row0 || end > n_rows) { q.n = -1; q.status = DSPARK_DEV_BAD_OFFSETS; }
    else if (q.first < 0 || (long long)q.first + q.n > capacity) { q.n = -1; q.status = DSPARK_DEV_BAD_PAGE; }
    return q;
}

// Every request of the step looked at once, by one CTA.
__device__ __forceinline__ void kv_report(const int32_t* first, const int32_t* row_offsets, int R, int n_rows, long long capacity, int32_t* dev_status)
{
    int status = 0;
    for (int r = threadIdx.x; r < R; r += blockDim.x) status |= kv_request(first, row_offsets, r, n_rows, capacity).status;
    if (status) atomicOr(dev_status, status);
}

// What a cache allows, on the host: DSPARK_OK or an error.
inline int kv_cache_check(const dspark_kv_cache_t* c, int layer)
{
    if (!c || !c->k || !c->v || !c->block_table) return DSPARK_ERR_INVALID_ARG;
    const bool narrow = c->dtype == DSPARK_I8 || c->dtype == DSPARK_E4M3;
    if (!narrow && c->dtype != DSPARK_BF16) return DSPARK_ERR_INVALID_ARG;
    if (narrow && (!c->k_scale || !c->v_scale)) return DSPARK_ERR_INVALID_ARG;
    if (c->n_layers < 1 || layer < 0 || layer >= c->n_layers || c->n_pages < 1 || c->page_size < 1 || c->kv_heads < 1 ||
        c->head_dim < 1 || c->max_pages < 1 || c->block_table_stride < c->max_pages)
        return DSPARK_ERR_INVALID_ARG;
    if (c->n_layers > 1024 || c->n_pages > (1 << 28) || c->page_size > (1 << 20) || c->kv_heads > 1024 || c->head_dim > 256 ||
        c->head_dim % 16 != 0 || (c->page_size <= 128 && (c->page_size < 8 || (c->page_size & (c->page_size - 1)) != 0)))
        return DSPARK_ERR_SHAPE;
    const long long unit = narrow ? 16 : 8;
    const long long strides[4] = {c->layer_stride, c->page_stride, c->token_stride, c->head_stride};
    for (long long s : strides) {
        if (s < 0) return DSPARK_ERR_INVALID_ARG;
        if (s % unit) return DSPARK_ERR_ALIGNMENT;
    }
    if ((c->n_pages > 1 && c->page_stride < c->head_dim) || (c->page_size > 1 && c->token_stride < c->head_dim) ||
        (c->kv_heads > 1 && c->head_stride < c->head_dim) || (c->n_layers > 1 && c->layer_stride < c->head_dim))
        return DSPARK_ERR_INVALID_ARG;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return DSPARK_ERR_ALIGNMENT;
    if (((uintptr_t)c->block_table | (uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) return DSPARK_ERR_ALIGNMENT;
    return DSPARK_OK;
}
inline int kv_step_check(const void* first, const void* row_offsets, int R, int n_rows, const void* dev_status)
{
    if (!first || !row_offsets || !dev_status || R < 1 || n_rows < 1) return DSPARK_ERR_INVALID_ARG;
    if (R > (1 << 20) || n_rows > (1 << 24)) return DSPARK_ERR_SHAPE;
    if (((uintptr_t)first | (uintptr_t)row_offsets | (uintptr_t)dev_status) & 3) return DSPARK_ERR_ALIGNMENT;
    return DSPARK_OK;
}
inline KvView kv_view(const dspark_kv_cache_t* c, int layer)
{
    const long long es = c->dtype == DSPARK_BF16 ? 2 : 1;
    const long long scales = (long long)c->n_pages * c->kv_heads * c->page_size;
    KvView v;
    v.k = (unsigned char*)c->k + layer * c->layer_stride * es;
    v.v = (unsigned char*)c->v + layer * c->layer_stride * es;
    v.k_scale = c->k_scale ? c->k_scale + layer * scales : nullptr;
    v.v_scale = c->v_scale ? c->v_scale + layer * scales : nullptr;
    v.dtype = c->dtype; v.n_pages = c->n_pages; v.page_size = c->page_size; v.kv_heads = c->kv_heads;
    v.head_dim = c->head_dim; v.max_pages = c->max_pages;
    v.page_shift = -1;
    for (int i = 0; i < 31; ++i) if (c->page_size == 1 << i) v.page_shift = i;
    v.page_stride = c->page_stride * es; v.token_stride = c->token_stride * es; v.head_stride = c->head_stride * es;
    v.block_table = c->block_table; v.table_stride = c->block_table_stride;
    return v;
}
// positions a request can have: those of its row of the block table, below 2^31
__host__ __device__ inline long long kv_capacity(const KvView& c)
{
    const long long all = (long long)c.max_pages * c.page_size;
    return all < 0x7fffffffll ? all : 0x7fffffffll;
}

}  // namespace dspark
