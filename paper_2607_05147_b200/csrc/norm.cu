// dspark_rms_norm_quant: the norm in front of the vocabulary projection, with the residual's addition and an int8
// output.  Per row of width d
//     h = round(x + residual)                         (stored; without a residual h = x)
//     y = h * rsqrt(mean(h^2) + eps) * w
//     q = rint(127 y / max|y|),   scale = max|y| / 127,     so that  q * scale ~ y.
// One pass: a row is read once into registers, its sum of squares and its largest product |h w| are reduced together
// (the norm's factor cancels in q, so q needs no second reduction), then q, h and scale are written.
//
// What bounds it: HBM (bf16: 2 + 2 bytes in, 2 + 1 out per element); one row is a chain of one load, one reduction and
// one store.  A row goes to one warp up to 1 024 elements (no block barrier; eight rows a CTA keep the loads of
// several rows in flight), to a CTA of d / 16 threads (bf16; d / 8 in fp32)
// beyond that.
//
// Rounding: q is the integer nearest to the exact quotient 127 t / max|t|, t = h w, ties to even.  One multiply-add,
// t * (127 / max|t|) + 1.5 * 2^23, leaves that integer in the low byte of its result; a second one gives the distance to
// it.  The factor and the product are off by at most 127 * 3 * 2^-24 = 2.3e-5 together, so an element whose distance is
// beyond 0.5 - 4e-5 (one in 12 000) is decided by a 64-bit division of the exact products.
#include <cuda_bf16.h>
#include <math.h>
#include <type_traits>

#include "common.cuh"

namespace dspark {

struct NormParams {
    const void* x; long long x_stride;
    const void* res; long long res_stride;      // NULL: no residual
    const void* w;
    void* h_out; long long h_stride;            // NULL: not stored
    int8_t* q; long long q_stride;
    float* scale;
    void* y; long long y_stride;                // NULL: not stored
    const int32_t* n_live;                      // NULL: all rows
    int rows, d;
    float eps;
};

constexpr int kNormVec = 16;                    // bytes of one vector of x
constexpr int kNormMaxThreads = 1024;
constexpr int kNormMaxD = 16384;
constexpr int kNormMaxStages = 8;
constexpr float kNormSmall = 1e-33f, kNormLargeRstd = 0x1p59f, kNormMark = -1.f;   // small_row()
constexpr int kNormSms = 148;                   // a B200's: what the thresholds below were measured on
constexpr int kNormStreamRows = 4 * kNormSms;   // below, a row per CTA starts sooner than a ring fills

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kPer = kNormVec / 4;
    typedef double Product;                     // exact product of two elements
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float load(const void* p, long long i) { return ((const float*)p)[i]; }
    static __device__ __forceinline__ void store(void* p, long long i, float v) { ((float*)p)[i] = v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kPer = kNormVec / 2;
    typedef float Product;                      // 8 x 8 significant bits: exact in fp32
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16lo(w[i]); f[2 * i + 1] = bf16hi(w[i]); }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float load(const void* p, long long i) { return __bfloat162float(((const __nv_bfloat16*)p)[i]); }
    static __device__ __forceinline__ void store(void* p, long long i, float v) { ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v); }
    static __device__ __forceinline__ float round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }
};

// maximum of |b| and a that keeps a NaN
__device__ __forceinline__ float max_abs_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(fabsf(b)));
    return m;
}
__device__ __forceinline__ double max_abs_nan(double a, double b)
{
    b = fabs(b);
    return (b > a || b != b) ? b : a;
}
__device__ __forceinline__ float warp_max_any(float v) { return warp_max_f32(v); }
__device__ __forceinline__ double warp_max_any(double v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The integer of an element that lies next to a half, n (with its distance's sign) the nearer one in fp32.  bf16: the
// product has 16 significant bits, so 254 t and (2 n +- 1) max|t| are exact in fp32 and their comparison decides.
// fp32: the quotient of the exact products in 64 bits.
__device__ __forceinline__ int next_to_half(float h, float w, float top, float n, float distance)
{
    float t = h * w, m = top;
    if (top > 1e36f) { t *= 0x1p-16f; m *= 0x1p-16f; }
    const float odd = 2.f * n + (distance < 0.f ? -1.f : 1.f);
    const float diff = 254.f * t - odd * m;                 // both exact, so the sign of the difference is
    const int below = (int)floorf(0.5f * odd);              // the two integers next to the half
    return diff > 0.f ? below + 1 : diff < 0.f ? below : below + (below & 1);
}
__device__ __forceinline__ int next_to_half(float h, float w, double top, float, float) { return (int)rint(((double)h * (double)w * 127.0) / top); }

// What a group of threads (a warp or a CTA) keeps of a row: vector v of a thread holds the elements of vector
// v * width + me (kVec), or its element e is column (v * kPer + e) * width + me (rows or pitches that break the 16-byte
// rule).
template <typename T, int kVpt, bool kVec>
struct NormRow {
    typedef Elem<T> E;
    typedef typename E::Product Prod;
    static constexpr int kPer = E::kPer;
    // a vector of the weight, packed as it lies in memory (kVec) or element by element
    struct Packed { uint4 v; __device__ __forceinline__ void get(float (&w)[kPer]) const { E::unpack(v, w); } };
    struct Single {
        float v[kPer];
        __device__ __forceinline__ void get(float (&w)[kPer]) const
        {
#pragma unroll
            for (int e = 0; e < kPer; ++e) w[e] = v[e];
        }
    };
    typedef typename std::conditional<kVec, Packed, Single>::type Weight;
    float h[kVpt][kPer];

    // h = x + residual from the vectors of both, rounded, and stored
    __device__ __forceinline__ void add(const uint4 (&xv)[kVpt], const uint4 (&rv)[kVpt], bool with_residual, T* h_out, int d, int width, int me)
    {
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            const int at = v * width + me;
            E::unpack(xv[v], h[v]);
            uint4 hv = xv[v];
            if (with_residual) {
                float r[kPer];
                E::unpack(rv[v], r);
#pragma unroll
                for (int e = 0; e < kPer; ++e) h[v][e] += r[e];
                hv = E::pack(h[v]);                         // rounds
                E::unpack(hv, h[v]);
            }
            if (h_out && at * kPer < d) reinterpret_cast<uint4*>(h_out)[at] = hv;
        }
    }
    __device__ __forceinline__ void statistics(const Weight (&weight)[kVpt], float& sum, Prod& top) const
    {
        sum = 0.f;
        top = 0;
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            float w[kPer];
            weight[v].get(w);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                sum = fmaf(h[v][e], h[v][e], sum);
                top = max_abs_nan(top, (Prod)h[v][e] * (Prod)w[e]);
            }
        }
        // an infinite or NaN maximum (of the row or of the weights) travels in the sum
        if (!(top <= (Prod)3.4e38)) sum = NAN;
    }
    __device__ __forceinline__ void finish(const NormParams& P, long long row, const Weight (&weight)[kVpt], float sum, float rstd, Prod top, int width, int me)
    {
        const bool bad = !(sum < INFINITY);                 // NaN or infinity in the row, or beyond fp32's range
        const float topf = (float)top;
        if (me == 0) P.scale[row] = bad ? NAN : (top == 0 ? 0.f : topf * rstd * (1.f / 127.f));
        const bool zero = bad || top == 0;
        // fp32: or the compiler keeps the 64-bit products of the statistics for the few elements next to a half, two registers
        // each (rows of 1001 elements 158 -> 293 us)
        if (sizeof(T) == 4)
#pragma unroll
            for (int v = 0; v < kVpt; ++v)
#pragma unroll
                for (int e = 0; e < kPer; ++e) asm volatile("" : "+f"(h[v][e]));
        const float inv = zero ? 0.f : 127.f / topf;
        constexpr float limit = 0.49996f;
        constexpr float kMagic = 12582912.f;                // 1.5 * 2^23: the integer ends up in the low bits
        int8_t* q_out = P.q + row * P.q_stride;
        T* y_out = P.y ? (T*)P.y + row * P.y_stride : nullptr;
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            float w[kPer];
            weight[v].get(w);
            uint32_t bits[kPer];
            float far = 0.f;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const float t = zero ? 0.f : h[v][e] * w[e];
                const float m = fmaf(t, inv, kMagic);
                far = fmaxf(far, fabsf(fmaf(t, inv, kMagic - m)));
                bits[e] = __float_as_uint(m);
            }
            if (far > limit && !zero) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float n = __uint_as_float(bits[e]) - kMagic, distance = fmaf(h[v][e] * w[e], inv, -n);
                    if (fabsf(distance) > limit) bits[e] = (uint32_t)next_to_half(h[v][e], w[e], top, n, distance);
                }
            }
            if (kVec) {
                const int at = v * width + me;
                if (at * kPer >= P.d) continue;
                uint32_t packed[kPer / 4];
#pragma unroll
                for (int i = 0; i < kPer / 4; ++i)
                    packed[i] = __byte_perm(__byte_perm(bits[4 * i], bits[4 * i + 1], 0x0040), __byte_perm(bits[4 * i + 2], bits[4 * i + 3], 0x0040), 0x5410);
                if (kPer == 8) *reinterpret_cast<uint2*>(q_out + (long long)at * 8) = make_uint2(packed[0], packed[kPer / 4 - 1]);
                else *reinterpret_cast<uint32_t*>(q_out + (long long)at * 4) = packed[0];
                if (y_out) {
                    float y[kPer];
#pragma unroll
                    for (int e = 0; e < kPer; ++e) y[e] = (h[v][e] * w[e]) * rstd;
                    reinterpret_cast<uint4*>(y_out)[at] = E::pack(y);
                }
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const int col = (v * kPer + e) * width + me;
                    if (col >= P.d) continue;
                    q_out[col] = (int8_t)(bits[e] & 255u);
                    if (y_out) E::store(y_out, col, (h[v][e] * w[e]) * rstd);
                }
            }
        }
    }
};

// Sum and maximum over a group; the CTA's group passes through shared memory (two sets in turn, so that one barrier a row
// is enough).
template <bool kWarp, typename Prod>
__device__ __forceinline__ void group_reduce(float& sum, Prod& top, float* s_sum, Prod* s_top)
{
    sum = warp_sum_f32(sum);
    top = warp_max_any(top);
    if (!kWarp) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (int)blockDim.x >> 5;
        if (lane == 0) { s_sum[warp] = sum; s_top[warp] = top; }
        __syncthreads();
        if (n_warps <= 8) {                                 // broadcast reads: a shorter chain than shuffles
            sum = 0.f;
            top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n_warps) { sum += s_sum[i]; top = s_top[i] > top ? s_top[i] : top; }
        } else {
            sum = lane < n_warps ? s_sum[lane] : 0.f;
            top = lane < n_warps ? s_top[lane] : (Prod)0;
            sum = warp_sum_f32(sum);
            top = warp_max_any(top);
        }
    }
}

// Rows at the bottom of fp32's range, in 64 bits.  Where the largest product is below kNormSmall, products next to a half and
// the maximum itself may be subnormal in fp32 and have lost the digits that decide an integer; where the mean of the squares
// and eps together are below 2^-118 (rstd above kNormLargeRstd), squares that underflow (off by 2^-150 each) show in the root.
// 64 bits hold every product of two elements.  Rows of nothing but zeros (padding) are found first, in vectors.  The row is
// read again: h from out_residual where it was stored (which may be x itself), else x + residual.  It comes last in a kernel,
// when nothing else is kept in registers: the ring marks such rows in out_scale and does them after its last row (called from
// its loop, it cost fp32 rows 13 to 30 %).
template <typename Prod>
__device__ __forceinline__ bool is_small(float sum, float rstd, Prod top)
{
    return sum < INFINITY && (top < (Prod)kNormSmall || rstd > kNormLargeRstd);
}
template <bool kWarp>
__device__ __forceinline__ void group_reduce64(double& sum, double& top)
{
    sum = warp_sum_f64(sum);
    top = warp_max_any(top);
    if (!kWarp) {
        __shared__ double s_sum[kNormMaxThreads / 32], s_top[kNormMaxThreads / 32];
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (int)blockDim.x >> 5;
        if (lane == 0) { s_sum[warp] = sum; s_top[warp] = top; }
        __syncthreads();
        sum = warp_sum_f64(lane < n_warps ? s_sum[lane] : 0.0);
        top = warp_max_any(lane < n_warps ? s_top[lane] : 0.0);
    }
}
template <typename T, bool kVec, bool kWarp>
__device__ __forceinline__ void small_row(const NormParams& P, long long row)
{
    typedef Elem<T> E;
    const int width = kWarp ? 32 : (int)blockDim.x, me = kWarp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    // out_residual was written by the whole group; the sums of the row before have been read
    if (kWarp) __syncwarp(); else __syncthreads();
    const T* x = (const T*)(P.h_out ? P.h_out : P.x) + row * (P.h_out ? P.h_stride : P.x_stride);
    const T* res = P.res && !P.h_out ? (const T*)P.res + row * P.res_stride : nullptr;
    auto load = [&](int i) { return res ? E::round(E::load(x, i) + E::load(res, i)) : E::load(x, i); };
    int8_t* q = P.q + row * P.q_stride;
    T* y = P.y ? (T*)P.y + row * P.y_stride : nullptr;
    if constexpr (kVec) {
        constexpr int kPer = E::kPer;
        bool some = false;
#pragma unroll 4
        for (int at = me; at * kPer < P.d; at += width) {
            float h[kPer], r[kPer];
            E::unpack(reinterpret_cast<const uint4*>(x)[at], h);
            E::unpack(res ? reinterpret_cast<const uint4*>(res)[at] : make_uint4(0, 0, 0, 0), r);
#pragma unroll
            for (int e = 0; e < kPer; ++e) some = some || h[e] + r[e] != 0.f;      // a sum of two numbers is not rounded to zero
        }
        if (!(kWarp ? __any_sync(0xffffffffu, some) : __syncthreads_or(some))) {
            if (me == 0) P.scale[row] = 0.f;
            for (int at = me; at * kPer < P.d; at += width) {
                if (kPer == 8) *reinterpret_cast<uint2*>(q + (long long)at * 8) = make_uint2(0, 0);
                else *reinterpret_cast<uint32_t*>(q + (long long)at * 4) = 0;
                if (y) reinterpret_cast<uint4*>(y)[at] = make_uint4(0, 0, 0, 0);
            }
            return;
        }
    }
    double sum = 0.0, top = 0.0;
#pragma unroll 1
    for (int i = me; i < P.d; i += width) {
        const double h = load(i);
        sum = fma(h, h, sum);
        top = max_abs_nan(top, h * (double)E::load(P.w, i));
    }
    group_reduce64<kWarp>(sum, top);
    const double rstd = 1.0 / sqrt(sum / P.d + (double)P.eps);
    if (me == 0) P.scale[row] = top == 0.0 ? 0.f : (float)(top * rstd / 127.0);
#pragma unroll 1
    for (int i = me; i < P.d; i += width) {
        const double t = (double)load(i) * (double)E::load(P.w, i);
        q[i] = top == 0.0 ? 0 : (int8_t)rint(t * 127.0 / top);
        if (y) E::store(y, i, top == 0.0 ? 0.f : (float)(t * rstd));
    }
}

// One row per group, loaded straight into registers: few rows, or rows that break the 16-byte rule.
// kWarp: a warp per row, several rows per CTA; otherwise a CTA per row.
template <typename T, int kVpt, bool kVec, bool kWarp, int kThreads>
__global__ void __launch_bounds__(kThreads) rms_norm_quant_kernel(const __grid_constant__ NormParams P)
{
    typedef Elem<T> E;
    typedef typename E::Product Prod;
    constexpr int kPer = E::kPer;
    __shared__ float s_sum[kNormMaxThreads / 32];
    __shared__ Prod s_top[kNormMaxThreads / 32];
    const int width = kWarp ? 32 : (int)blockDim.x;
    const int me = kWarp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const long long row = kWarp ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : (long long)blockIdx.x;
    pdl_wait();
    if (P.n_live) {
        if (row >= (long long)*P.n_live) return;            // a whole warp or CTA: nobody is left at the barrier
    }
    if (row >= P.rows) return;
    const T* x = (const T*)P.x + row * P.x_stride;
    const T* res = P.res ? (const T*)P.res + row * P.res_stride : nullptr;
    T* h_out = P.h_out ? (T*)P.h_out + row * P.h_stride : nullptr;
    NormRow<T, kVpt, kVec> r;
    typename NormRow<T, kVpt, kVec>::Weight w[kVpt];
    if constexpr (kVec) {
        uint4 xv[kVpt], rv[kVpt];
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            const int at = v * width + me;
            xv[v] = rv[v] = w[v].v = make_uint4(0, 0, 0, 0);
            if (at * kPer < P.d) {
                xv[v] = reinterpret_cast<const uint4*>(x)[at];
                if (res) rv[v] = reinterpret_cast<const uint4*>(res)[at];
                w[v].v = __ldg(reinterpret_cast<const uint4*>(P.w) + at);
            }
        }
        r.add(xv, rv, res != nullptr, h_out, P.d, width, me);
    } else {
#pragma unroll
        for (int v = 0; v < kVpt; ++v)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int col = (v * kPer + e) * width + me;
                r.h[v][e] = w[v].v[e] = 0.f;
                if (col < P.d) {
                    r.h[v][e] = E::load(x, col);
                    w[v].v[e] = E::load(P.w, col);
                    if (res) r.h[v][e] = E::round(r.h[v][e] + E::load(res, col));
                    if (h_out) E::store(h_out, col, r.h[v][e]);
                }
            }
    }
    float sum;
    Prod top;
    r.statistics(w, sum, top);
    group_reduce<kWarp>(sum, top, s_sum, s_top);
    const float rstd = rsqrtf(sum / (float)P.d + P.eps);
    if (is_small(sum, rstd, top)) small_row<T, kVec, kWarp>(P, row);
    else r.finish(P, row, w, sum, rstd, top, width, me);
}

// Many rows: persistent groups walk the rows, each with a ring of `stages` rows of x and the residual in shared memory that
// bulk copies keep filled, so that the loads of the next rows are in flight while one is reduced and written.  The barrier
// of the reduction (a warp: __syncwarp) is what frees a stage.  The weight stays in registers.
// kCtas: CTAs an SM that the registers have to allow.  Occupancy is what hides the chain of a row (shared memory,
// reduction, barrier, store).
template <typename T, int kVpt, bool kWarp, int kThreads, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas) rms_norm_quant_stream_kernel(const __grid_constant__ NormParams P, int stages, uint32_t poll_limit)
{
    typedef Elem<T> E;
    typedef typename E::Product Prod;
    constexpr int kPer = E::kPer;
    constexpr int kGroups = kWarp ? kThreads / 32 : 1;
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ __align__(8) uint64_t full[kGroups][kNormMaxStages];
    __shared__ float s_sum[2][kNormMaxThreads / 32];
    __shared__ Prod s_top[2][kNormMaxThreads / 32];
    const int group = kWarp ? (int)threadIdx.x >> 5 : 0;
    const int width = kWarp ? 32 : (int)blockDim.x;
    const int me = kWarp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const uint32_t row_bytes = (uint32_t)(P.d * sizeof(T));
    const uint32_t stage_bytes = row_bytes * (P.res ? 2 : 1);
    unsigned char* ring = s_ring + (size_t)group * stages * stage_bytes;
    if (threadIdx.x == 0) {
        for (int g = 0; g < kGroups; ++g)
            for (int s = 0; s < stages; ++s) mbar_init(&full[g][s], 1);
        mbar_fence_init();
    }
    __syncthreads();
    pdl_wait();
    // 32 bits hold a row's number and `stages` steps beyond the last one
    uint32_t live = (uint32_t)P.rows;
    if (P.n_live) { const int n = *P.n_live; live = (uint32_t)(n < 0 ? 0 : n < P.rows ? n : P.rows); }
    const uint32_t first = blockIdx.x * kGroups + group, step = gridDim.x * kGroups;
    const uint64_t pol = l2_policy_evict_first();
    auto request = [&](uint32_t row, int s) {
        mbar_arrive_expect_tx(&full[group][s], stage_bytes);
        bulk_g2s_hint(ring + s * stage_bytes, (const T*)P.x + row * P.x_stride, row_bytes, &full[group][s], pol);
        if (P.res) bulk_g2s_hint(ring + s * stage_bytes + row_bytes, (const T*)P.res + row * P.res_stride, row_bytes, &full[group][s], pol);
    };
    if (me == 0)
        for (int s = 0; s < stages; ++s)
            if (first + s * step < live) request(first + s * step, s);
    typename NormRow<T, kVpt, true>::Weight w[kVpt];
#pragma unroll
    for (int v = 0; v < kVpt; ++v) {
        const int at = v * width + me;
        w[v].v = make_uint4(0, 0, 0, 0);
        if (at * kPer < P.d) w[v].v = __ldg(reinterpret_cast<const uint4*>(P.w) + at);
    }
    int s = 0, turn = 0;
    uint32_t ph = 0;
    bool direct = false;                                    // each thread's own
    bool small = false;                                     // the same in the whole group
    uint32_t row = first;
    for (; row < live; row += step) {
        unsigned char* stage = ring + s * stage_bytes;
        // The copy is this group's own and lands.  A thread whose wait ran out all the same fetches its part of this row and of
        // all that follow itself, from where nobody else writes to where nobody else reads: a barrier that is behind by a phase
        // would pass for the one awaited.  The group's first thread, which asks for the copies, then lets those on their way
        // land (with the long bound) and asks for no more; waits of the others run out in turn.
        if (!direct && !mbar_wait_bounded(&full[group][s], ph, poll_limit)) {
            direct = true;
            if (me == 0)
                for (int i = 0; i < stages && row + i * step < live; ++i)
                    mbar_wait_bounded(&full[group][s + i < stages ? s + i : s + i - stages], s + i < stages ? ph : ph ^ 1u);
        }
        if (direct) {
#pragma unroll 1
            for (int at = me; at * kPer < P.d; at += width) {
                reinterpret_cast<uint4*>(stage)[at] = reinterpret_cast<const uint4*>((const T*)P.x + row * P.x_stride)[at];
                if (P.res) reinterpret_cast<uint4*>(stage + row_bytes)[at] = reinterpret_cast<const uint4*>((const T*)P.res + row * P.res_stride)[at];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        uint4 xv[kVpt], rv[kVpt];
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            const int at = v * width + me;
            xv[v] = rv[v] = make_uint4(0, 0, 0, 0);
            if (at * kPer < P.d) {
                xv[v] = reinterpret_cast<const uint4*>(stage)[at];
                if (P.res) rv[v] = reinterpret_cast<const uint4*>(stage + row_bytes)[at];
            }
        }
        NormRow<T, kVpt, true> r;
        r.add(xv, rv, P.res != nullptr, P.h_out ? (T*)P.h_out + row * P.h_stride : nullptr, P.d, width, me);
        float sum;
        Prod top;
        r.statistics(w, sum, top);
        group_reduce<kWarp>(sum, top, s_sum[turn & 1], s_top[turn & 1]);
        if (kWarp) __syncwarp();
        if (me == 0 && !direct && row + stages * step < live) request(row + stages * step, s);
        const float rstd = rsqrtf(sum / (float)P.d + P.eps);
        if (is_small(sum, rstd, top)) {
            small = true;
            if (me == 0) P.scale[row] = kNormMark;
        } else {
            r.finish(P, row, w, sum, rstd, top, width, me);
        }
        if (++s == stages) { s = 0; ph ^= 1u; }
        ++turn;
    }
    if (small) {
        if (kWarp) __syncwarp(); else __syncthreads();      // the marks are written
        while (row >= step) {                               // the first row is below `step`
            row -= step;
            if (*(volatile const float*)(P.scale + row) == kNormMark) small_row<T, true, kWarp>(P, row);
        }
    }
}

// Polls of a wait for a row's copy, by device, 0 standing for kWaitPollLimit (dspark_set_wait_poll_limit); a kernel argument,
// since a register for it would be spilled.  The wait for copies before they are given up keeps the long bound.
static std::atomic<uint32_t> g_norm_poll_limit[64];
int norm_set_poll_limit(uint32_t polls)
{
    int dev = 0;
    cudaGetDevice(&dev);
    g_norm_poll_limit[dev & 63].store(polls ^ kWaitPollLimit, std::memory_order_relaxed);
    return launch_status();
}

template <typename T, int kVpt, bool kWarp, int kThreads, int kCtas>
static bool norm_stream(const NormParams& P, int threads, cudaStream_t s)
{
    constexpr int kSmemPerSm = 200 * 1024, kMost = 200 * 1024;
    const int groups = kWarp ? kThreads / 32 : 1;
    const int stage = P.d * (int)sizeof(T) * (P.res ? 2 : 1) * groups;
    // as many CTAs as the registers allow, the ring cut to what they leave of the shared memory
    int ctas = kCtas * kThreads / threads;
    int stages = kSmemPerSm / ctas / stage;
    if (stages < 2) { ctas = 1; stages = kSmemPerSm / stage; }
    if (stages < 2) return false;
    if (stages > kNormMaxStages) stages = kNormMaxStages;
    static std::atomic<unsigned long long> ready{0};        // one bit per device
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(rms_norm_quant_stream_kernel<T, kVpt, kWarp, kThreads, kCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) !=
            cudaSuccess)
            return false;
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    const long long want = ((long long)P.rows + groups - 1) / groups, cap = (long long)sms * ctas;
    launch_pdl(rms_norm_quant_stream_kernel<T, kVpt, kWarp, kThreads, kCtas>, dim3((unsigned)(want < cap ? want : cap)), dim3(threads),
               (size_t)stages * stage, s, P, stages, g_norm_poll_limit[dev & 63].load(std::memory_order_relaxed) ^ kWaitPollLimit);
    return true;
}

template <typename T, bool kVec>
static void norm_launch(const NormParams& P, cudaStream_t s)
{
    constexpr int kPer = Elem<T>::kPer;
    const int vectors = (P.d + kPer - 1) / kPer;
    // a warp per row; rows of more than 256 elements only where there are enough of them to fill the SMs with warps
    if (P.d <= 256 || (P.d <= 1024 && P.rows >= 8 * kNormSms)) {
        const int per = (vectors + 31) / 32;
        if constexpr (kVec) {
            if (P.rows >= kNormStreamRows * 8) {
                bool done;
                if (per <= 1) done = norm_stream<T, 1, true, 256, 5>(P, 256, s);
                else if (per <= 2) done = norm_stream<T, 2, true, 256, 4>(P, 256, s);
                else if (kPer == 8 || per <= 4) done = norm_stream<T, 4, true, 256, 2>(P, 256, s);
                else done = norm_stream<T, kPer == 4 ? 8 : 4, true, 256, 1>(P, 256, s);
                if (done) return;
            }
        }
        const int warps = P.rows >= 8 * kNormSms ? 8 : 1;
        const dim3 grid((unsigned)((P.rows + warps - 1) / warps)), block(warps * 32);
        if (per <= 1) launch_pdl(rms_norm_quant_kernel<T, 1, kVec, true, 256>, grid, block, 0, s, P);
        else if (per <= 2) launch_pdl(rms_norm_quant_kernel<T, 2, kVec, true, 256>, grid, block, 0, s, P);
        else if (kPer == 8 || per <= 4) launch_pdl(rms_norm_quant_kernel<T, 4, kVec, true, 256>, grid, block, 0, s, P);
        else if constexpr (kPer == 4) launch_pdl(rms_norm_quant_kernel<T, 8, kVec, true, 256>, grid, block, 0, s, P);
        return;
    }
    // two vectors a thread while that fits a CTA, four beyond (fp32 rows of more than 8 192 elements)
    constexpr bool kFour = kNormMaxD / kPer > 2 * kNormMaxThreads;
    const int per = kFour && vectors > 2 * kNormMaxThreads ? 4 : 2;
    const int threads = (((vectors + per - 1) / per) + 31) & ~31;
    const dim3 grid(P.rows), block(threads);
    if constexpr (kFour)
        if (per == 4) {
            launch_pdl(rms_norm_quant_kernel<T, 4, kVec, false, kNormMaxThreads>, grid, block, 0, s, P);
            return;
        }
    if constexpr (kVec)
        if (P.rows >= kNormStreamRows) {
            const bool done = threads <= 256 ? norm_stream<T, 2, false, 256, 4>(P, threads, s)
                            : threads <= 512 ? norm_stream<T, 2, false, 512, 2>(P, threads, s) : norm_stream<T, 2, false, kNormMaxThreads, 1>(P, threads, s);
            if (done) return;
        }
    if (threads <= 512) launch_pdl(rms_norm_quant_kernel<T, 2, kVec, false, 512>, grid, block, 0, s, P);
    else launch_pdl(rms_norm_quant_kernel<T, 2, kVec, false, kNormMaxThreads>, grid, block, 0, s, P);
}

}  // namespace dspark

using namespace dspark;

extern "C" {

int dspark_rms_norm_quant(const void* x, int64_t x_row_stride, const void* residual, int64_t residual_row_stride,
                          const void* weight, int dtype, int rows, int d, float eps, const int32_t* n_live,
                          void* out_residual, int64_t out_residual_row_stride, int8_t* out_q, int64_t out_q_row_stride,
                          float* out_scale, void* out_norm, int64_t out_norm_row_stride, void* stream)
{
    if (!x || !weight || !out_q || !out_scale || rows < 1 || d < 1) return DSPARK_ERR_INVALID_ARG;
    if (dtype != DSPARK_F32 && dtype != DSPARK_BF16) return DSPARK_ERR_INVALID_ARG;
    if (!(eps >= 0.f) || isinf(eps)) return DSPARK_ERR_INVALID_ARG;
    if (x_row_stride < d || out_q_row_stride < d || (residual && residual_row_stride < d) ||
        (out_residual && out_residual_row_stride < d) || (out_norm && out_norm_row_stride < d))
        return DSPARK_ERR_INVALID_ARG;
    if (d > kNormMaxD) return DSPARK_ERR_SHAPE;
    const int es = dtype == DSPARK_BF16 ? 2 : 4;
    const uintptr_t elems = (uintptr_t)x | (uintptr_t)residual | (uintptr_t)weight | (uintptr_t)out_residual | (uintptr_t)out_norm;
    if ((elems & (uintptr_t)(es - 1)) || ((uintptr_t)out_scale & 3u) || ((uintptr_t)n_live & 3u)) return DSPARK_ERR_ALIGNMENT;
    NormParams P;
    P.x = x; P.x_stride = x_row_stride;
    P.res = residual; P.res_stride = residual_row_stride;
    P.w = weight;
    P.h_out = out_residual; P.h_stride = out_residual_row_stride;
    P.q = out_q; P.q_stride = out_q_row_stride;
    P.scale = out_scale;
    P.y = out_norm; P.y_stride = out_norm_row_stride;
    P.n_live = n_live; P.rows = rows; P.d = d; P.eps = eps;
    // 16-byte vectors of x and the rows beside it, as many bytes of q as a vector has elements
    const int per = kNormVec / es;
    bool vec = (elems & 15u) == 0 && d % per == 0 && x_row_stride % per == 0 && ((uintptr_t)out_q % per) == 0 && out_q_row_stride % per == 0;
    if (residual) vec = vec && residual_row_stride % per == 0;
    if (out_residual) vec = vec && out_residual_row_stride % per == 0;
    if (out_norm) vec = vec && out_norm_row_stride % per == 0;
    cudaStream_t s = (cudaStream_t)stream;
    KernelTimerScope timer(DSPARK_K_RMS_NORM, s);
    if (dtype == DSPARK_BF16) {
        if (vec) norm_launch<__nv_bfloat16, true>(P, s); else norm_launch<__nv_bfloat16, false>(P, s);
    } else {
        if (vec) norm_launch<float, true>(P, s); else norm_launch<float, false>(P, s);
    }
    return launch_status();
}

}  // extern "C"
