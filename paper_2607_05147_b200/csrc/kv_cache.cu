// dspark_kv_write, dspark_kv_read, dspark_kv_commit: the paged cache of K and V rows in 16 or 8 bits.
//
// A head's row x [d] is stored with one scale,
//     int8:  s = max|x| / 127, q = rint(127 x / max|x|);      e4m3:  s = max|x| / 448, q = e4m3(448 x / max|x|),
// and read as s q.  q needs no division.  127 x and 448 x of a bf16 x have 15 and 11 significant bits, so that their quotient by a
// bf16 number, where it is not a tie of either target (at most 8 bits), is at least 2^-17 of its size away from every tie.  The product
// with an approximate reciprocal is off by less than 2^-21; rounded to 19 bits (2^-19) it is on the tie where the quotient is one,
// and on the quotient's side of it elsewhere, and rounds to the target as the exact quotient would.
//
// All three are bound by memory, or, for few rows, by a chain of dependent loads: row_offsets -> first -> block_table -> store.
// The rows are therefore read before that chain is begun.  A head's row belongs to 4, 8 or 16 neighbouring lanes, two pieces of 16
// bytes of bf16 each, so that the maximum is a few shuffles and neighbouring lanes and heads fill whole sectors; a thread has two
// such rows in flight.  For many rows instructions come next: where a row lies is worked out by one thread of the CTA.
// Prompts of 15.5 thousand rows, 8 heads of 128, int8: written in 24 us and read back in 20 (97 MB each, 4.0 and 4.8 TB/s); 8 rows of
// one request 3.2 us each way (kernels in a replayed graph; a call from Python costs some 10 us of the host's time).
#include "kv_cache.cuh"

namespace dspark {

constexpr int kKvThreads = 256;
constexpr int kKvRows = 2;                       // head rows of one thread, two pieces of 8 components each

struct KvStep {
    KvView c;
    const int32_t* first; const int32_t* row_offsets; int R, n_rows;
    uint32_t heads_reciprocal;                                 // 2^32 / kv_heads, rounded up
    int32_t* dev_status;
    const unsigned char* k; const unsigned char* v;            // kv_write: the rows
    unsigned char* out_k; unsigned char* out_v; int out_f32;   // kv_read
    long long row_stride, head_stride;                         // bytes, of either
};

// Byte offset of a head's row in the cache, and the index of its scale; false: there is no such page.
struct KvSlot { long long at, scale; };
__device__ __forceinline__ bool kv_slot(const KvView& c, int r, int position, int head, KvSlot& s)
{
    const int page_of = c.page_shift >= 0 ? position >> c.page_shift : position / c.page_size, token = position - page_of * c.page_size;
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

__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <int kDtype> __device__ constexpr float kv_whole() { return kDtype == DSPARK_I8 ? 127.f : 448.f; }
// Two times 8 of a head row's values, 8 bits each.  top: the row's largest magnitude; bad: it holds NaN or an infinity
template <int kLanes, int kDtype>
__device__ __forceinline__ void kv_quantise(const uint4 (&x)[2], uint2 (&q)[2], float& top, bool& bad)
{
    uint32_t most = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        most = max_nan_bf16x2(most, max_nan_bf16x2(max_nan_bf16x2(x[h].x & 0x7fff7fffu, x[h].y & 0x7fff7fffu),
                                                   max_nan_bf16x2(x[h].z & 0x7fff7fffu, x[h].w & 0x7fff7fffu)));
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) most = max_nan_bf16x2(most, __shfl_xor_sync(0xffffffffu, most, o));
    most = max_nan_bf16x2(most, most >> 16 | most << 16);
    top = bf16lo(most);
    bad = !(top < INFINITY);
    q[0] = q[1] = make_uint2(0, 0);
    if (bad || top == 0.f) return;
    // x and its maximum, both times a power of two where the reciprocal would leave the range of fp32
    const float by = top > 1e35f ? 0x1p-16f : top < 1e-35f ? 0x1p64f : 1.f;
    const float inverse = kv_whole<kDtype>() * rcp_approx(top * by);
    const uint64_t by2 = pack2(by, by), inverse2 = pack2(inverse, inverse);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint64_t e = pack2(bf16lo(w[i]), bf16hi(w[i]));
            if (by != 1.f) e = mul2(e, by2);
            float a, b;
            unpack2(mul2(e, inverse2), a, b);
            a = __uint_as_float((__float_as_uint(a) + 16u) & ~31u);
            b = __uint_as_float((__float_as_uint(b) + 16u) & ~31u);
            if constexpr (kDtype == DSPARK_I8) {
                // 1.5 2^23 + a: rounded to an integer, which its low bits are
                unpack2(add2(pack2(a, b), pack2(12582912.f, 12582912.f)), a, b);
                r[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
            } else
                r[i] = e4m3x2(a, b);
        }
        q[h] = make_uint2(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410));
    }
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
        // a byte + 128 in the low bits of 2^23
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t bytes = w[i >> 2] ^ 0x80808080u;
            const float a = __uint_as_float(__byte_perm(bytes, 0x4b000000u, 0x7440 | (i & 3)));
            const float b = __uint_as_float(__byte_perm(bytes, 0x4b000000u, 0x7441 | (i & 3)));
            unpack2(mul2(add2(pack2(a, b), pack2(-8388736.f, -8388736.f)), pack2(scale, scale)), e[i], e[i + 1]);
        }
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
// counts those of its first row, one load a thread, and each row goes on from there; beyond, every row is searched for.  Up to
// kKvThreads requests are kept in shared memory with their first tokens, so that no row waits for memory again before its page.
// Offsets that fall somewhere (an error, reported) lead the count and the search astray: a row for which they have found no request
// is then looked for in all of them.
constexpr int kCountRequests = 1024;
struct KvRequests {
    const int32_t* first; const int32_t* row_offsets;         // of all requests, in shared or global memory
    int R, from;                                              // from: request of the CTA's first row
};
struct KvRequestsShared { int32_t first[kKvThreads], row_offsets[kKvThreads + 1]; };
__device__ __forceinline__ KvRequests kv_requests(const int32_t* first, const int32_t* row_offsets, int R, int row, KvRequestsShared& S)
{
    KvRequests q = {first, row_offsets, R, 0};
    const int tid = threadIdx.x;
    if (R <= kKvThreads) {
        const bool in = tid < R;
        const int end = in ? row_offsets[tid + 1] : 0;
        if (in) { S.first[tid] = first[tid]; S.row_offsets[tid + 1] = end; }
        if (tid == 0) S.row_offsets[0] = row_offsets[0];
        q.from = __syncthreads_count(in && end <= row);
        q.first = S.first; q.row_offsets = S.row_offsets;
    } else if (R <= kCountRequests)
        for (int i0 = 1; i0 <= R; i0 += kKvThreads) q.from += __syncthreads_count(i0 + tid <= R && row_offsets[i0 + tid] <= row);
    return q;
}
__device__ __forceinline__ int kv_find_request(const KvRequests& q, int row)
{
    int lo = q.from;
    if (q.R <= kCountRequests) {
        while (lo < q.R && q.row_offsets[lo + 1] <= row) ++lo;
        return lo;
    }
    int hi = q.R;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (q.row_offsets[mid + 1] <= row) lo = mid + 1; else hi = mid;
    }
    return lo;
}
// Head rows [blockIdx.x * per, ...).
template <int kLanes, int kDtype, bool kWrite>
__global__ void __launch_bounds__(kKvThreads, 6) kv_rows_kernel(const __grid_constant__ KvStep P)
{
    constexpr int kPer = kKvThreads / kLanes;
    constexpr int kMost = kPer * kKvRows / 2 + 1;             // rows that a CTA has a part of
    __shared__ KvRequestsShared S;
    __shared__ KvSlot slots[kMost];                           // of head 0; at = -1: the row is left alone, -2: it has no page
    pdl_wait();
    const int tid = threadIdx.x, sub = tid & (kLanes - 1), slot = tid / kLanes;
    const int heads = P.c.kv_heads;
    // index = (row * 2 + (0: K, 1: V)) * heads + head; a product with the reciprocal divides, exact for a CTA's few thousand
    const long long total = (long long)P.n_rows * 2 * heads, base = (long long)blockIdx.x * (kPer * kKvRows);
    const int row0 = total >> 32 ? (int)(base / (2 * heads)) : (int)((uint32_t)base / (uint32_t)(2 * heads));
    const int base_in = (int)(base - (long long)row0 * 2 * heads);
    struct Place { int local, head; bool value, live; };                    // local: row - row0
    auto place = [&](int j) {
        const uint32_t i = base_in + j * kPer + slot, at = heads == 1 ? i : __umulhi(i, P.heads_reciprocal);
        return Place{(int)(at >> 1), (int)(i - at * heads), (at & 1) != 0, base + j * kPer + slot < total};
    };
    auto in = [&](int h) { return (sub + h * kLanes) * 8 < P.c.head_dim; };       // piece h of this thread exists
    uint4 x[kKvRows][2];
    if (kWrite) {
        const unsigned char* k_in = P.k + row0 * P.row_stride + sub * 16;
        const unsigned char* v_in = P.v + row0 * P.row_stride + sub * 16;
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            const Place p = place(j);
            const unsigned char* from = (p.value ? v_in : k_in) + p.local * P.row_stride + p.head * P.head_stride;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x[j][h] = make_uint4(0, 0, 0, 0);
                if (p.live && in(h)) x[j][h] = *reinterpret_cast<const uint4*>(from + h * kLanes * 16);
            }
        }
    }
    // where the CTA's rows are in the cache, one thread a row
    const long long capacity = kv_capacity(P.c);
    const KvRequests requests = kv_requests(P.first, P.row_offsets, P.R, row0, S);
    bool lost = false;                                        // no request was found for this thread's row
    auto put = [&](const KvRequest& q, int r, int row) {
        KvSlot at = {-1, 0};
        if (!kv_slot(P.c, r, q.first + (row - q.row0), 0, at)) {
            at.at = -2;
            atomicOr(P.dev_status, DSPARK_DEV_BAD_PAGE);
        }
        slots[tid] = at;
    };
    auto look_everywhere = [&](int row) {
        for (int r = 0; r < P.R; ++r) {
            const KvRequest q = kv_request(requests.first, requests.row_offsets, r, P.n_rows, capacity);
            if (q.status == DSPARK_DEV_BAD_OFFSETS || row < q.row0 || row >= requests.row_offsets[r + 1]) continue;
            if (q.n >= 0) put(q, r, row);
            return;
        }
    };
    if (tid < (kMost + 31) / 32 * 32) {
        const int row = row0 + tid, r = tid < kMost && row < P.n_rows ? kv_find_request(requests, row) : P.R;
        if (tid < kMost) slots[tid] = {-1, 0};
        lost = tid < kMost && row < P.n_rows;
        if (r < P.R) {
            const KvRequest q = kv_request(requests.first, requests.row_offsets, r, P.n_rows, capacity);
            lost = q.status == DSPARK_DEV_BAD_OFFSETS || row < q.row0;
            if (q.n >= 0 && !lost) put(q, r, row);
        }
        if (P.R <= kKvThreads && __any_sync(0xffffffffu, lost)) {
            bool falls = false;
#pragma unroll
            for (int i = 0; i < kKvThreads; i += 32) {
                const int at = min(i + (tid & 31), P.R - 1);
                falls |= requests.row_offsets[at + 1] < requests.row_offsets[at];
            }
            if (__any_sync(0xffffffffu, falls) && lost) look_everywhere(row);
        }
    }
    if (P.R > kKvThreads && __syncthreads_or(lost)) {
        bool falls = false;
        for (int i = tid; i < P.R; i += kKvThreads) falls = falls || P.row_offsets[i + 1] < P.row_offsets[i];
        if (__syncthreads_or(falls) && lost) look_everywhere(row0 + tid);
    }
    __syncthreads();

    if constexpr (kWrite) {
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            const Place p = place(j);
            const KvSlot s = slots[p.local];
            const bool store = p.live && s.at >= 0;
            unsigned char* to = (p.value ? P.c.v : P.c.k) + s.at + p.head * P.c.head_stride;
            if constexpr (kDtype == DSPARK_BF16) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (store && in(h)) *reinterpret_cast<uint4*>(to + (sub + h * kLanes) * 16) = x[j][h];
            } else {
                bool bad;
                float top;
                uint2 q[2];
                kv_quantise<kLanes, kDtype>(x[j], q, top, bad);
                if (store) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (in(h)) *reinterpret_cast<uint2*>(to + (sub + h * kLanes) * 8) = q[h];
                    if (sub == 0) (p.value ? P.c.v_scale : P.c.k_scale)[s.scale + p.head * P.c.page_size] = bad ? NAN : top / kv_whole<kDtype>();
                }
            }
        }
    } else {
        float scale[kKvRows];                               // all loads first
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            const Place p = place(j);
            const KvSlot s = slots[p.local];
            x[j][0] = x[j][1] = make_uint4(0, 0, 0, 0);
            scale[j] = 0.f;
            if (p.live && s.at >= 0) {
                const unsigned char* from = (p.value ? P.c.v : P.c.k) + s.at + p.head * P.c.head_stride;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!in(h)) continue;
                    if constexpr (kDtype == DSPARK_BF16) x[j][h] = *reinterpret_cast<const uint4*>(from + (sub + h * kLanes) * 16);
                    else {
                        const uint2 q = *reinterpret_cast<const uint2*>(from + (sub + h * kLanes) * 8);
                        x[j][h].x = q.x; x[j][h].y = q.y;
                    }
                }
                if constexpr (kDtype != DSPARK_BF16) {
                    scale[j] = (p.value ? P.c.v_scale : P.c.k_scale)[s.scale + p.head * P.c.page_size];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kKvRows; ++j) {
            const Place p = place(j);
            unsigned char* out = p.value ? P.out_v : P.out_k;
            if (!p.live || !out || slots[p.local].at == -1) continue;
            out += (row0 + p.local) * P.row_stride + p.head * P.head_stride;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (in(h)) kv_put<kDtype>(out, sub + h * kLanes, x[j][h], scale[j], P.out_f32);
        }
    }
    if (blockIdx.x == 0) kv_report(P.first, P.row_offsets, P.R, P.n_rows, capacity, P.dev_status);
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
    if (P.c.head_dim <= 64) kv_rows_launch<4, kWrite>(P, s);
    else if (P.c.head_dim <= 128) kv_rows_launch<8, kWrite>(P, s);
    else kv_rows_launch<16, kWrite>(P, s);
    return launch_status();
}

// ---- accepted paths ----------------------------------------------------------------------------------------
// A CTA has one request and some of the layers' K and V.  Where the path's rows lie, and where they go, is worked out once, a run of
// kCommitRun nodes at a time, for all layers.  A thread owns 16 bytes of a position (or one scale) and moves them along the
// path, kCommitBatch positions at a time: path[i] > i and the path ascends, so a position that is read is never one that an
// earlier batch has written, and within a batch all reads come first.  Different threads touch different bytes: no order among
// them.  64 requests, up to 7 nodes, 32 layers of 8 heads of 128 (66 MB): 15.6 us, 4.2 TB/s; a CTA for each layer's K or V worked the
// path out 64 times and took 39.5.
constexpr int kCommitThreads = 128, kCommitBatch = 8, kCommitRun = 128;

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
    __shared__ KvSlot s_from[kCommitRun], s_to[kCommitRun];   // of head 0; from.at < 0: nothing to move
    pdl_wait();
    const int r = blockIdx.x, tid = threadIdx.x;
    const KvView& c = P.c;
    const int accepted = P.accepted[r];
    const KvRequest q = kv_request(P.first, P.row_offsets, r, P.n_rows, kv_capacity(c));
    const bool tell = blockIdx.y == 0 && tid == 0;
    if (tell && q.status) atomicOr(P.dev_status, q.status);
    if (q.n <= 0) {
        if (tell && P.out_first) P.out_first[r] = q.first;
        return;
    }
    const int n = accepted;
    const int32_t* path = P.path + q.row0;
    bool bad = n < 0 || n >= q.n;
    if (!bad)
        for (int i = tid; i < n; i += kCommitThreads) bad = bad || path[i] >= q.n || path[i] <= (i ? path[i - 1] : 0);
    bad = __syncthreads_or(bad);
    if (tell) {
        if (bad) atomicOr(P.dev_status, DSPARK_DEV_BAD_TREE);
        if (P.out_first) P.out_first[r] = bad ? q.first : q.first + 1 + n;
    }
    if (bad) return;
    const int es = c.dtype == DSPARK_BF16 ? 2 : 1, per_head = c.head_dim * es / 16, pieces = per_head * c.kv_heads;
    const int scales = c.dtype == DSPARK_BF16 ? 0 : c.kv_heads;
    bool bad_page = false;
    for (int run0 = 0; run0 < n; run0 += kCommitRun) {
        const int count = min(kCommitRun, n - run0);
        for (int i = tid; i < count; i += kCommitThreads) {
            const int node = path[run0 + i];
            s_from[i].at = -1;
            if (node != run0 + i + 1) {
                KvSlot from, to;
                const bool there = kv_slot(c, r, q.first + node, 0, from);
                if (kv_slot(c, r, q.first + 1 + run0 + i, 0, to) && there) { s_from[i] = from; s_to[i] = to; }
                else bad_page = true;
            }
        }
        __syncthreads();
        for (int lkv = blockIdx.y; lkv < 2 * P.n_layers; lkv += gridDim.y) {
            const int layer = lkv >> 1;
            unsigned char* cache = ((lkv & 1) ? c.v : c.k) + layer * P.layer_stride;
            float* scale = (lkv & 1) ? c.v_scale : c.k_scale;
            if (scale) scale += layer * P.layer_scales;
            for (int i = tid; i < pieces + scales; i += kCommitThreads) {
                const bool row = i < pieces;
                const int head = row ? i / per_head : i - pieces;
                unsigned char* mine = row ? cache + head * c.head_stride + (i - head * per_head) * 16 : nullptr;
                float* my_scale = row ? nullptr : scale + (long long)head * c.page_size;
                for (int j0 = 0; j0 < count; j0 += kCommitBatch) {
                    uint4 x[kCommitBatch];
#pragma unroll
                    for (int j = 0; j < kCommitBatch; ++j)
                        if (j0 + j < count && s_from[j0 + j].at >= 0) {
                            if (row) x[j] = *reinterpret_cast<const uint4*>(mine + s_from[j0 + j].at);
                            else x[j].x = __float_as_uint(my_scale[s_from[j0 + j].scale]);
                        }
#pragma unroll
                    for (int j = 0; j < kCommitBatch; ++j)
                        if (j0 + j < count && s_from[j0 + j].at >= 0) {
                            if (row) *reinterpret_cast<uint4*>(mine + s_to[j0 + j].at) = x[j];
                            else my_scale[s_to[j0 + j].scale] = __uint_as_float(x[j].x);
                        }
                }
            }
        }
        __syncthreads();
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
    P.heads_reciprocal = (uint32_t)(((1ull << 32) + cache->kv_heads - 1) / cache->kv_heads);
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
    P.heads_reciprocal = (uint32_t)(((1ull << 32) + cache->kv_heads - 1) / cache->kv_heads);
    P.first = first; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows; P.dev_status = dev_status;
    P.out_k = (unsigned char*)out_k; P.out_v = (unsigned char*)out_v; P.out_f32 = out_dtype == DSPARK_F32;
    P.row_stride = out_row_stride * es; P.head_stride = out_head_stride * es;
    return kv_rows<false>(P, (cudaStream_t)stream);
}

int dspark_kv_commit(const dspark_kv_cache_t* cache, const int32_t* first, const int32_t* row_offsets, int R, int n_rows,
                     const int32_t* accepted_len, const int32_t* path, int32_t* out_first, int32_t* dev_status, void* stream)
{
    using namespace dspark;
    if (!accepted_len || !path) return DSPARK_ERR_INVALID_ARG;
    if (int e = kv_cache_check(cache, 0)) return e;
    if (int e = kv_step_check(first, row_offsets, R, n_rows, dev_status)) return e;
    if (((uintptr_t)accepted_len | (uintptr_t)path | (uintptr_t)out_first) & 3) return DSPARK_ERR_ALIGNMENT;
    // a request's CTAs (by layers) read these at times of their own, one of them writes its entry of out_first
    const size_t out = out_first ? (size_t)R * 4 : 0;
    if (ranges_meet(out_first, out, first, (size_t)R * 4) || ranges_meet(out_first, out, row_offsets, (size_t)R * 4 + 4) ||
        ranges_meet(out_first, out, accepted_len, (size_t)R * 4) || ranges_meet(out_first, out, path, (size_t)n_rows * 4) ||
        ranges_meet(out_first, out, dev_status, 4))
        return DSPARK_ERR_INVALID_ARG;
    KvCommit P = {};
    P.c = kv_view(cache, 0);
    P.first = first; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows;
    P.accepted = accepted_len; P.path = path; P.out_first = out_first; P.dev_status = dev_status;
    P.layer_stride = cache->layer_stride * (cache->dtype == DSPARK_BF16 ? 2 : 1);
    P.layer_scales = (long long)cache->n_pages * cache->kv_heads * cache->page_size;
    P.n_layers = cache->n_layers;
    KernelTimerScope timer(DSPARK_K_KV_COMMIT, (cudaStream_t)stream);
    // as many CTAs as the SMs hold at a time, eight each: more wait for the same path and pages over again
    const int most = 8 * current_sms() / R, all = 2 * cache->n_layers;
    const int per = most < 1 ? all : (all + most - 1) / most;             // layers' K and V of a CTA
    launch_pdl(kv_commit_kernel, dim3((unsigned)R, (unsigned)((all + per - 1) / per)), dim3(kCommitThreads), 0, (cudaStream_t)stream, P);
    return launch_status();
}

}  // extern "C"
