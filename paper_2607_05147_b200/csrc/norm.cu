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
__device__ __forceinline__ float warp_max_any(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ double warp_max_any(double v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A row is spread over `width` threads: vector v of a thread holds the elements of vector v * width + lane (kVec), or
// its element e is column (v * kPer + e) * width + lane (rows or pitches that break the 16-byte rule).
// kWarp: one warp per row, several rows per CTA; otherwise one CTA per row.
template <typename T, int kVpt, bool kVec, bool kWarp, int kThreads>
__global__ void __launch_bounds__(kThreads) rms_norm_quant_kernel(const __grid_constant__ NormParams P)
{
    typedef Elem<T> E;
    typedef typename E::Product Prod;
    constexpr int kPer = E::kPer;
    __shared__ float s_sum[kNormMaxThreads / 32];
    __shared__ Prod s_top[kNormMaxThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int width = kWarp ? 32 : (int)blockDim.x;
    const int me = kWarp ? lane : (int)threadIdx.x;
    const long long row = kWarp ? (long long)blockIdx.x * (blockDim.x >> 5) + warp : (long long)blockIdx.x;
    pdl_wait();
    if (P.n_live) {
        if (row >= (long long)*P.n_live) return;            // a whole warp or CTA: nobody is left at the barrier
    }
    if (row >= P.rows) return;
    const T* x = (const T*)P.x + row * P.x_stride;
    const T* res = P.res ? (const T*)P.res + row * P.res_stride : nullptr;
    T* h_out = P.h_out ? (T*)P.h_out + row * P.h_stride : nullptr;
    T* y_out = P.y ? (T*)P.y + row * P.y_stride : nullptr;
    int8_t* q_out = P.q + row * P.q_stride;

    // the row and the weight; h is stored at once, t = h w is what stays
    float h[kVpt][kPer], w[kVpt][kPer];
    if (kVec) {
        uint4 xv[kVpt], rv[kVpt], wv[kVpt];
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            const int at = v * width + me;
            xv[v] = rv[v] = wv[v] = make_uint4(0, 0, 0, 0);
            if (at * kPer < P.d) {
                xv[v] = __ldcs(reinterpret_cast<const uint4*>(x) + at);
                if (res) rv[v] = __ldcs(reinterpret_cast<const uint4*>(res) + at);
                wv[v] = __ldg(reinterpret_cast<const uint4*>(P.w) + at);
            }
        }
#pragma unroll
        for (int v = 0; v < kVpt; ++v) {
            const int at = v * width + me;
            E::unpack(wv[v], w[v]);
            E::unpack(xv[v], h[v]);
            uint4 hv = xv[v];
            if (res) {
                float r[kPer];
                E::unpack(rv[v], r);
#pragma unroll
                for (int e = 0; e < kPer; ++e) h[v][e] += r[e];
                hv = E::pack(h[v]);                         // rounds
                E::unpack(hv, h[v]);
            }
            if (h_out && at * kPer < P.d) reinterpret_cast<uint4*>(h_out)[at] = hv;
        }
    } else {
#pragma unroll
        for (int v = 0; v < kVpt; ++v)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int col = (v * kPer + e) * width + me;
                h[v][e] = w[v][e] = 0.f;
                if (col < P.d) {
                    h[v][e] = E::load(x, col);
                    w[v][e] = E::load(P.w, col);
                    if (res) h[v][e] = E::round(h[v][e] + E::load(res, col));
                    if (h_out) E::store(h_out, col, h[v][e]);
                }
            }
    }
    float sum = 0.f;
    Prod top = 0;
#pragma unroll
    for (int v = 0; v < kVpt; ++v)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            sum = fmaf(h[v][e], h[v][e], sum);
            top = max_abs_nan(top, (Prod)h[v][e] * (Prod)w[v][e]);
        }
    // an infinite or NaN maximum (of the row or of the weights) travels in the sum
    if (!(top <= (Prod)3.4e38)) sum = NAN;
    sum = warp_sum_f32(sum);
    top = warp_max_any(top);
    if (!kWarp) {
        if (lane == 0) { s_sum[warp] = sum; s_top[warp] = top; }
        __syncthreads();
        const int n_warps = (int)blockDim.x >> 5;
        sum = lane < n_warps ? s_sum[lane] : 0.f;
        top = lane < n_warps ? s_top[lane] : (Prod)0;
        sum = warp_sum_f32(sum);
        top = warp_max_any(top);
    }
    const bool bad = !(sum < INFINITY);                     // NaN or infinity in the row, or beyond fp32's range
    const float topf = (float)top;
    const float rstd = rsqrtf(sum / (float)P.d + P.eps);
    if (me == 0) P.scale[row] = bad ? NAN : (top == 0 ? 0.f : topf * rstd * (1.f / 127.f));
    const bool zero = bad || top == 0;
    float inv = zero ? 0.f : 127.f / topf;
    // products next to the smallest fp32 numbers: every element is decided by the division
    const float limit = inv < 1e35f ? 0.49996f : -1.f;
    if (!(inv < 1e35f)) inv = 0.f;
    constexpr float kMagic = 12582912.f;                    // 1.5 * 2^23: the integer ends up in the low bits
    auto divided = [&](float he, float we) -> int { return (int)rint(((double)he * (double)we * 127.0) / (double)top); };
#pragma unroll
    for (int v = 0; v < kVpt; ++v) {
        uint32_t bits[kPer];
        float far = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float t = zero ? 0.f : h[v][e] * w[v][e];
            const float m = fmaf(t, inv, kMagic);
            far = fmaxf(far, fabsf(fmaf(t, inv, kMagic - m)));
            bits[e] = __float_as_uint(m);
        }
        if (far > limit && !zero) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const float t = h[v][e] * w[v][e];
                if (fabsf(fmaf(t, inv, kMagic - __uint_as_float(bits[e]))) > limit) bits[e] = (uint32_t)divided(h[v][e], w[v][e]);
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
                for (int e = 0; e < kPer; ++e) y[e] = (h[v][e] * w[v][e]) * rstd;
                reinterpret_cast<uint4*>(y_out)[at] = E::pack(y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int col = (v * kPer + e) * width + me;
                if (col >= P.d) continue;
                q_out[col] = (int8_t)(bits[e] & 255u);
                if (y_out) E::store(y_out, col, (h[v][e] * w[v][e]) * rstd);
            }
        }
    }
}

template <typename T, bool kVec>
static void norm_launch(const NormParams& P, cudaStream_t s)
{
    constexpr int kPer = Elem<T>::kPer;
    const int vectors = (P.d + kPer - 1) / kPer;
    if (P.d <= 1024) {                                      // a warp per row, 8 rows per CTA (fewer when there are few rows)
        const int per = (vectors + 31) / 32;
        const int warps = P.rows >= 8 * 148 ? 8 : 1;
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
