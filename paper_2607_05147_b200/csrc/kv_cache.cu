// dspark_kv_write, dspark_kv_read, dspark_kv_commit: the paged cache of K and V rows in 16 or 8 bits.
//
// A head's row x [d] is stored with one scale,
//     int8:  s = max|x| / 127, q = rint(127 x / max|x|);      e4m3:  s = max|x| / 448, q = e4m3(448 x / max|x|),
// and read as s q.  127 x and 448 x of a bf16 x are exact in fp32 (15 and 11 significant bits), and a quotient of such a number
// by a bf16 one that is not a tie of either target differs from every tie by more than 2^-17 of its size, so that the correctly
// rounded fp32 quotient decides every rounding as the exact one would.
//
// All three are bound by memory, or, for few rows, by a chain of dependent loads: row_offsets -> first -> block_table -> store.
// The rows are therefore read before that chain is begun.  A head's row belongs to 8, 16 or 32 neighbouring lanes, 16 bytes of
// bf16 each, so that the maximum is a few shuffles and neighbouring heads fill whole sectors; a thread has four such rows in
// flight.
#include "kv_cache.cuh"

namespace dspark {

constexpr int kKvThreads = 256;
constexpr int kKvRows = 4;                       // head rows of one thread

struct KvStep {
    KvView c;
    const int32_t* first; const int32_t* row_offsets; int R, n_rows;
    int32_t* dev_status;
    const unsigned char* k; const unsigned char* v;            // kv_write: the rows
    unsigned char* out_k; unsigned char* out_v; int out_f32;   // kv_read
    long long row_stride, head_stride;                         // bytes, of either
};

// Byte offset of a head's row in the cache, and the index of its scale; false: there is no such page.
struct KvSlot { long long at, scale; };
__device__ __forceinline__ bool kv_slot(const KvView& c, int r, int position, int head, KvSlot& s)
{
    const int page_of = position / c.page_size, token = position - page_of * c.page_size;
    const int page = c.block_table[r * c.table_stride + page_of];
    s.at = page * c.page_stride + token * c.token_stride + head * c.head_stride;
    s.scale = ((long long)page * c.kv_heads + head) * c.page_size + token;
    return page >= 0 && page < c.n_pages;
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t v)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
    return r;
}
__device__ __forceinline__ float f16_value(uint32_t bits)
{
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)bits));
    return f;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int kDtype> __device__ constexpr float kv_whole() { return kDtype == DSPARK_I8 ? 127.f : 448.f; }
// 8 of a head row's values, 8 bits each; top: the row's largest magnitude, bad: it holds NaN or an infinity
template <int kLanes, int kDtype>
__device__ __forceinline__ uint2 kv_quantise(uint4 x, float& top, bool& bad)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float e[8];
    top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { e[2 * i] = bf16lo(w[i]); e[2 * i + 1] = bf16hi(w[i]); }
#pragma unroll
    for (int i = 0; i < 8; ++i) { const float a = fabsf(e[i]); top = (a > top || a != a) ? a : top; }   // NaN stays
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) {
        const float a = __shfl_xor_sync(0xffffffffu, top, o);
        top = (a > top || a != a) ? a : top;
    }
    bad = !(top < INFINITY);
    uint32_t q[2] = {0, 0};
    if (!bad && top != 0.f) {
        // above, whole * x passes the range of fp32: both 2^16 smaller there
        const float up = top > 1e35f ? kv_whole<kDtype>() * 0x1p-16f : kv_whole<kDtype>(), by = top > 1e35f ? top * 0x1p-16f : top;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float a = __fdiv_rn(up * e[i], by), b = __fdiv_rn(up * e[i + 1], by);
            const uint32_t two = kDtype == DSPARK_I8 ? ((uint32_t)(int)rintf(a) & 0xffu) | ((uint32_t)(int)rintf(b) & 0xffu) << 8 : e4m3x2(a, b);
            q[i >> 2] |= two << (8 * (i & 3));
        }
    }
    return make_uint2(q[0], q[1]);
}
// 8 values of a head row to `out` (the row's start)
template <int kDtype>
__device__ __forceinline__ void kv_put(unsigned char* out, int sub, uint4 x, float scale, bool f32)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float e[8];
    if constexpr (kDtype == DSPARK_BF16) {
        if (!f32) { *reinterpret_cast<uint4*>(out + sub * 16) = x; return; }
#pragma unroll
        for (int i = 0; i < 4; ++i) { e[2 * i] = bf16lo(w[i]); e[2 * i + 1] = bf16hi(w[i]); }
    } else if constexpr (kDtype == DSPARK_I8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t h = f16x2_of_e4m3x2(w[i >> 2] >> (8 * (i & 3)));
            e[i] = f16_value(h) * scale;
            e[i + 1] = f16_value(h >> 16) * scale;
        }
    }
    if (f32) {
        float4* o = reinterpret_cast<float4*>(out + sub * 32);
        o[0] = make_float4(e[0], e[1], e[2], e[3]);
        o[1] = make_float4(e[4], e[5], e[6], e[7]);
    } else
        *reinterpret_cast<uint4*>(out + sub * 16) = make_uint4(bf16x2(e[0], e[1]), bf16x2(e[2], e[3]), bf16x2(e[4], e[5]), bf16x2(e[6], e[7]));
}

// Which request a row belongs to: the number of requests that end at or before it.  Up to kCountRequests of them the CTA
// counts those of its first row, one load a thread, and each row goes on from there; beyond, every row is searched for.
constexpr int kCountRequests = 1024;
__device__ __forceinline__ int kv_count_requests(const int32_t* row_offsets, int R, int row)     // all threads of the CTA
{
    int r = 0;
    for (int i0 = 1; i0 <= R; i0 += kKvThreads) {
        const int i = i0 + (int)threadIdx.x;
        r += __syncthreads_count(i <= R && row_offsets[i] <= row);
    }
    return r;
}
__device__ __forceinline__ int kv_find_request(const int32_t* row_offsets, int R, int row, int from)
{
    if (R <= kCountRequests) {
        while (from < R && row_offsets[from + 1] <= row) ++from;
        return from;
    }
    int lo = 0, hi = R;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (row_offsets[mid + 1] <= row) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Head rows [blockIdx.x * per, ...): index = (row * 2 + (0: K, 1: V)) * heads + head.
template <int kLanes, int kDtype, bool kWrite>
__global__ void __launch_bounds__(kKvThreads) kv_rows_kernel(const __grid_constant__ KvStep P)
{
    constexpr int kPer = kKvThreads / kLanes;
    pdl_wait();
    const int tid = threadIdx.x, sub = tid & (kLanes - 1), slot = tid / kLanes;
    const int heads = P.c.kv_heads;
    const long long total = (long long)P.n_rows * 2 * heads, base = (long long)blockIdx.x * (kPer * kKvRows);
    const bool in = sub * 8 < P.c.head_dim;
    int row[kKvRows], head[kKvRows];
    bool value[kKvRows], live[kKvRows];
    uint4 x[kKvRows];
#pragma unroll
    for (int j = 0; j < kKvRows; ++j) {
        const long long i = base + j * kPer + slot;
        live[j] = i < total;
        const int at = (int)(i / heads);
        row[j] = at >> 1;
        value[j] = at & 1;
        head[j] = (int)(i - (long long)at * heads);
        if (kWrite) {
            x[j] = make_uint4(0, 0, 0, 0);
            if (live[j] && in)
                x[j] = *reinterpret_cast<const uint4*>((value[j] ? P.v : P.k) + row[j] * P.row_stride + head[j] * P.head_stride + sub * 16);
        }
    }
    const long long capacity = kv_capacity(P.c);
    if (blockIdx.x == 0) kv_report(P.first, P.row_offsets, P.R, P.n_rows, capacity, P.dev_status);
    const int r0 = P.R <= kCountRequests ? kv_count_requests(P.row_offsets, P.R, (int)(base / (2 * heads))) : 0;

    KvSlot s[kKvRows];
    bool page_there[kKvRows];
    bool bad_page = false;
#pragma unroll
    for (int j = 0; j < kKvRows; ++j) {
        const int r = live[j] ? kv_find_request(P.row_offsets, P.R, row[j], r0) : P.R;
        live[j] = r < P.R;
        page_there[j] = false;
        if (live[j]) {
            const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, capacity);
            live[j] = q.n >= 0 && row[j] >= q.row0;
            if (live[j]) page_there[j] = kv_slot(P.c, r, q.first + row[j] - q.row0, head[j], s[j]);
            bad_page = bad_page || (live[j] && !page_there[j]);
        }
    }
    if (bad_page) atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);

    if constexpr (kWrite) {
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            unsigned char* cache = value[j] ? P.c.v : P.c.k;
            const bool store = live[j] && page_there[j];
            if constexpr (kDtype == DSPARK_BF16) {
                if (store && in) *reinterpret_cast<uint4*>(cache + s[j].at + sub * 16) = x[j];
            } else {
                bool bad;
                float top;
                const uint2 q = kv_quantise<kLanes, kDtype>(x[j], top, bad);
                if (store && in) {
                    *reinterpret_cast<uint2*>(cache + s[j].at + sub * 8) = q;
                    if (sub == 0) (value[j] ? P.c.v_scale : P.c.k_scale)[s[j].scale] = bad ? NAN : top / kv_whole<kDtype>();
                }
            }
        }
    } else {
        float scale[kKvRows];                               // all loads first
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            x[j] = make_uint4(0, 0, 0, 0);
            scale[j] = 0.f;
            if (live[j] && page_there[j] && in) {
                const unsigned char* cache = value[j] ? P.c.v : P.c.k;
                if constexpr (kDtype == DSPARK_BF16) x[j] = *reinterpret_cast<const uint4*>(cache + s[j].at + sub * 16);
                else {
                    const uint2 q = *reinterpret_cast<const uint2*>(cache + s[j].at + sub * 8);
                    x[j].x = q.x; x[j].y = q.y;
                    scale[j] = (value[j] ? P.c.v_scale : P.c.k_scale)[s[j].scale];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            unsigned char* out = value[j] ? P.out_v : P.out_k;
            if (live[j] && in && out) kv_put<kDtype>(out + row[j] * P.row_stride + head[j] * P.head_stride, sub, x[j], scale[j], P.out_f32);
        }
    }
}

template <int kLanes, bool kWrite>
static void kv_rows_launch(const KvStep& P, cudaStream_t s)
{
    const long long per = kKvThreads / kLanes * kKvRows, total = (long long)P.n_rows * 2 * P.c.kv_heads;
    const dim3 grid((unsigned)((total + per - 1) / per));
    if (P.c.dtype == DSPARK_BF16) launch_pdl(kv_rows_kernel<kLanes, DSPARK_BF16, kWrite>, grid, dim3(kKvThreads), 0, s, P);
    else if (P.c.dtype == DSPARK_I8) launch_pdl(kv_rows_kernel<kLanes, DSPARK_I8, kWrite>, grid, dim3(kKvThreads), 0, s, P);
    else launch_pdl(kv_rows_kernel<kLanes, DSPARK_E4M3, kWrite>, grid, dim3(kKvThreads), 0, s, P);
}
template <bool kWrite>
static int kv_rows(const KvStep& P, cudaStream_t s)
{
    KernelTimerScope timer(kWrite ? DSPARK_K_KV_WRITE : DSPARK_K_KV_READ, s);
    if (P.c.head_dim <= 64) kv_rows_launch<8, kWrite>(P, s);
    else if (P.c.head_dim <= 128) kv_rows_launch<16, kWrite>(P, s);
    else kv_rows_launch<32, kWrite>(P, s);
    return launch_status();
}

// ---- accepted paths ----------------------------------------------------------------------------------------
// One CTA per request and (layer, K or V).  A thread owns 16 bytes of a position (or one scale) and moves them along the whole
// path, kBatch positions at a time: path[i] > i and the path ascends, so a position that is read is never one that an earlier
// batch has written, and within a batch all reads come first.  Different threads touch different bytes: no order among them.
constexpr int kCommitThreads = 128, kCommitBatch = 8;

struct KvCommit {
    KvView c;
    const int32_t* first; const int32_t* row_offsets; int R, n_rows;
    const int32_t* accepted; const int32_t* path;
    int32_t* out_first; int32_t* dev_status;
    long long layer_stride, layer_scales;                     // bytes, entries
    int n_layers;
};

__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const __grid_constant__ KvCommit P)
{
    __shared__ int s_bad;
    pdl_wait();
    const int r = blockIdx.x, tid = threadIdx.x;
    const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, kv_capacity(P.c));
    const bool tell = blockIdx.y == 0 && tid == 0;
    if (tell && q.status) atomicOr(P.dev_status, q.status);
    if (q.n <= 0) {
        if (tell && P.out_first) P.out_first[r] = q.first;
        return;
    }
    const int n = P.accepted[r];
    if (tid == 0) s_bad = (n < 0 || n >= q.n) ? 1 : 0;
    __syncthreads();
    const int32_t* path = P.path + q.row0;
    if (n > 0 && n < q.n)
        for (int i = tid; i < n; i += kCommitThreads)
            if (path[i] >= q.n || path[i] <= (i ? path[i - 1] : 0)) s_bad = 1;
    __syncthreads();
    const bool bad = s_bad != 0;
    if (tell) {
        if (bad) atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE);
        if (P.out_first) P.out_first[r] = bad ? q.first : q.first + 1 + n;
    }
    if (bad) return;
    const KvView& c = P.c;
    const int es = c.dtype == DSPARK_BF16 ? 2 : 1, per_head = c.head_dim * es / 16, pieces = per_head * c.kv_heads;
    const int scales = c.dtype == DSPARK_BF16 ? 0 : c.kv_heads;
    bool bad_page = false;
    for (int lkv = blockIdx.y; lkv < 2 * P.n_layers; lkv += gridDim.y) {
        const int layer = lkv >> 1;
        unsigned char* cache = ((lkv & 1) ? c.v : c.k) + layer * P.layer_stride;
        float* scale = (lkv & 1) ? c.v_scale : c.k_scale;
        if (scale) scale += layer * P.layer_scales;
        for (int i = tid; i < pieces + scales; i += kCommitThreads) {
            const bool row = i < pieces;
            const int head = row ? i / per_head : i - pieces, piece = row ? i - head * per_head : 0;
            for (int j0 = 0; j0 < n; j0 += kCommitBatch) {
                uint4 x[kCommitBatch];
                KvSlot to[kCommitBatch];
                bool move[kCommitBatch];
#pragma unroll
                for (int j = 0; j < kCommitBatch; ++j) {
                    move[j] = j0 + j < n && path[j0 + j] != j0 + j + 1;
                    if (!move[j]) continue;
                    KvSlot from;
                    const bool there = kv_slot(c, r, q.first + path[j0 + j], head, from);
                    move[j] = kv_slot(c, r, q.first + 1 + j0 + j, head, to[j]) && there;
                    if (!move[j]) { bad_page = true; continue; }
                    if (row) x[j] = *reinterpret_cast<const uint4*>(cache + from.at + piece * 16);
                    else x[j].x = __float_as_uint(scale[from.scale]);
                }
#pragma unroll
                for (int j = 0; j < kCommitBatch; ++j)
                    if (move[j]) {
                        if (row) *reinterpret_cast<uint4*>(cache + to[j].at + piece * 16) = x[j];
                        else scale[to[j].scale] = __uint_as_float(x[j].x);
                    }
            }
        }
    }
    if (bad_page) atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);
}

static int strides_check(long long row, long long head, int heads, int d, int n_rows, long long unit)
{
    if (row < 0 || head < 0 || (heads > 1 && head < d) || (n_rows > 1 && row < d)) return DSPARK_ERR_INVALID_ARG;
    return (row % unit || head % unit) ? DSPARK_ERR_ALIGNMENT : DSPARK_OK;
}

}  // namespace dspark

extern "C" {

int dspark_kv_write(const dspark_kv_cache_t* cache, int layer, const void* k, const void* v, int64_t row_stride, int64_t head_stride,
                    const int32_t* first, const int32_t* row_offsets, int R, int n_rows, int32_t* dev_status, void* stream)
{
    using namespace dspark;
    if (!k || !v) return DSPARK_ERR_INVALID_ARG;
    if (int e = kv_cache_check(cache, layer)) return e;
    if (int e = kv_step_check(first, row_offsets, R, n_rows, dev_status)) return e;
    if (int e = strides_check(row_stride, head_stride, cache->kv_heads, cache->head_dim, n_rows, 8)) return e;
    if (((uintptr_t)k | (uintptr_t)v) & 15) return DSPARK_ERR_ALIGNMENT;
    KvStep P = {};
    P.c = kv_view(cache, layer);
    P.first = first; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows; P.dev_status = dev_status;
    P.k = (const unsigned char*)k; P.v = (const unsigned char*)v;
    P.row_stride = row_stride * 2; P.head_stride = head_stride * 2;
    return kv_rows<true>(P, (cudaStream_t)stream);
}

int dspark_kv_read(const dspark_kv_cache_t* cache, int layer, const int32_t* first, const int32_t* row_offsets, int R, int n_rows,
                   void* out_k, void* out_v, int out_dtype, int64_t out_row_stride, int64_t out_head_stride, int32_t* dev_status, void* stream)
{
    using namespace dspark;
    if ((!out_k && !out_v) || (out_dtype != DSPARK_BF16 && out_dtype != DSPARK_F32)) return DSPARK_ERR_INVALID_ARG;
    if (int e = kv_cache_check(cache, layer)) return e;
    if (int e = kv_step_check(first, row_offsets, R, n_rows, dev_status)) return e;
    const int es = out_dtype == DSPARK_F32 ? 4 : 2;
    if (int e = strides_check(out_row_stride, out_head_stride, cache->kv_heads, cache->head_dim, n_rows, 16 / es)) return e;
    if (((uintptr_t)out_k | (uintptr_t)out_v) & 15) return DSPARK_ERR_ALIGNMENT;
    KvStep P = {};
    P.c = kv_view(cache, layer);
    P.first = first; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows; P.dev_status = dev_status;
    P.out_k = (unsigned char*)out_k; P.out_v = (unsigned char*)out_v; P.out_f32 = out_dtype == DSPARK_F32;
    P.row_stride = out_row_stride * es; P.head_stride = out_head_stride * es;
    return kv_rows<false>(P, (cudaStream_t)stream);
}

int dspark_kv_commit(const dspark_kv_cache_t* cache, const int32_t* first, const int32_t* row_offsets, int R, int n_rows,
                     const int32_t* accepted_len, const int32_t* path, int32_t* out_first, int32_t* dev_status, void* stream)
{
    using namespace dspark;
    if (!accepted_len || !path || out_first == first) return DSPARK_ERR_INVALID_ARG;
    if (int e = kv_cache_check(cache, 0)) return e;
    if (int e = kv_step_check(first, row_offsets, R, n_rows, dev_status)) return e;
    if (((uintptr_t)accepted_len | (uintptr_t)path | (uintptr_t)out_first) & 3) return DSPARK_ERR_ALIGNMENT;
    KvCommit P = {};
    P.c = kv_view(cache, 0);
    P.first = first; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows;
    P.accepted = accepted_len; P.path = path; P.out_first = out_first; P.dev_status = dev_status;
    P.layer_stride = cache->layer_stride * (cache->dtype == DSPARK_BF16 ? 2 : 1);
    P.layer_scales = (long long)cache->n_pages * cache->kv_heads * cache->page_size;
    P.n_layers = cache->n_layers;
    KernelTimerScope timer(DSPARK_K_KV_COMMIT, (cudaStream_t)stream);
    launch_pdl(kv_commit_kernel, dim3((unsigned)R, (unsigned)(2 * cache->n_layers)), dim3(kCommitThreads), 0, (cudaStream_t)stream, P);
    return launch_status();
}

}  // extern "C"
