// dspark_verify_tree: lossless verification of a tree of drafted tokens from given random numbers (Section 2.1's rule,
// repeated over the children of a node).
//
// At node u with target p, drafter q and children c_1, c_2, ..: a child is accepted with probability min(1, r / (Z q)) at its
// token, r being what is left of p after the rejections before it.  The residual of a rejection is max(r - Z q, 0), and
// max(max(p - a q, 0) - b q, 0) = max(p - (a + b) q, 0) for q >= 0: whatever was rejected, r = max(p - A q, 0) with one number
// A, so a rejection costs one pass over the two rows for the new Z = sum r and nothing is stored.
//
// One cluster of eight CTAs per request.  Every CTA makes the walk itself, from the scalars p(x), q(x), u of all nodes, gathered
// at once; a pass over the vocabulary is shared: 128 warps own a run of it each, and the runs' sums pass through distributed
// shared memory, so that all CTAs go on with the same numbers.  The sums of the last pass are those of the draw, which only the
// warp that owns the drawn token's run reads again.  Sums and tests are fp64: what decides is a border between tokens.
//
// Bound by the chain of dependent loads for few requests, by the rows' bytes for many (one pair of rows a request is read at
// least, two where the path ends behind an accepted second child).
#include <math.h>

#include "common.cuh"

namespace dspark {

constexpr int kVtCtas = 8, kVtWarps = 16, kVtThreads = kVtWarps * 32, kVtRuns = kVtCtas * kVtWarps;
constexpr int kVtLoads = 8;                      // vectors of a run in flight in one lane

struct VerifyTreeParams {
    const float* p; long long p_stride;
    const float* q; long long q_stride;
    int V, run;                                  // run: entries of one warp, a multiple of 128
    const int32_t* tokens; const int32_t* parents; const int32_t* row_offsets;
    int R, n_rows;
    const float* u_accept; const float* u_sample;
    int32_t* accepted_len; int32_t* out_tokens; int32_t* out_path; int32_t* dev_status;
};

enum VtAction { kVtPass = 0, kVtDraw = 1, kVtVoid = 2 };

struct VtShared {
    double sums[2][kVtWarps];                    // read by the other CTAs; one set a pass, in turn
    double all[kVtRuns];                         // inclusive sums of all runs
    double A;
    int action, node, length, n_gone, status;
    short parent[DSPARK_TREE_MAX_NODES], path[DSPARK_TREE_MAX_NODES];
    int token[DSPARK_TREE_MAX_NODES], gone[DSPARK_TREE_MAX_NODES];
    float p[DSPARK_TREE_MAX_NODES], q[DSPARK_TREE_MAX_NODES], u[DSPARK_TREE_MAX_NODES];
};

__device__ __forceinline__ void vt_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ double vt_remote(const double* local, uint32_t rank)
{
    uint32_t a;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
    return v;
}

// What is left of four entries from v on: max(p - A q, 0), or p without the rejected tokens.  Entries from `end` on: 0.
// NaN stays.
struct VtRow {
    const float* p; const float* q;
    double A;
    const int* gone; int n_gone;
    bool vectors;
    __device__ __forceinline__ void load(int v, int end, float (&a)[4], float (&b)[4]) const
    {
        if (vectors && v + 4 <= end) {
            const float4 x = *reinterpret_cast<const float4*>(p + v);
            a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w;
            if (q) {
                const float4 y = *reinterpret_cast<const float4*>(q + v);
                b[0] = y.x; b[1] = y.y; b[2] = y.z; b[3] = y.w;
            }
        } else
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = v + i < end ? p[v + i] : 0.f;
                if (q) b[i] = v + i < end ? q[v + i] : 0.f;
            }
    }
    __device__ __forceinline__ double left(int v, float a, float b) const
    {
        double r = q ? (double)a - A * (double)b : (double)a;
        if (r < 0.0) r = 0.0;
        for (int i = 0; i < n_gone; ++i)
            if (gone[i] == v) r = 0.0;
        return r;
    }
};

__global__ void __cluster_dims__(kVtCtas, 1, 1) __launch_bounds__(kVtThreads) verify_tree_kernel(const __grid_constant__ VerifyTreeParams P)
{
    __shared__ VtShared S;
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int r = blockIdx.x / kVtCtas;
    const uint32_t rank = blockIdx.x % kVtCtas;
    const int row0 = P.row_offsets[r], end = P.row_offsets[r + 1], n = end - row0;
    const bool there = row0 >= 0 && end >= row0 && end <= P.n_rows;
    if (!there || n == 0) {
        if (rank == 0 && tid == 0) { P.accepted_len[r] = 0; atomicOr(P.dev_status, DSPARK_DEV_BAD_OFFSETS); }
        return;                                  // the whole cluster
    }
    if (tid == 0) S.status = n > DSPARK_TREE_MAX_NODES ? DSPARK_DEV_BAD_OFFSETS : 0;
    __syncthreads();
    if (n <= DSPARK_TREE_MAX_NODES) {
        int bad = 0;
        for (int i = 1 + tid; i < n; i += kVtThreads) {
            const int parent = P.parents[row0 + i], x = P.tokens[row0 + i];
            const float u = P.u_accept[row0 + i];
            if (parent < 0 || parent >= i) bad |= DSPARK_DEV_BAD_TREE;
            if (x < 0 || x >= P.V) bad |= DSPARK_DEV_BAD_TOKEN;
            S.parent[i] = (short)parent;
            S.token[i] = x;
            S.u[i] = u;
            if (!bad) {
                S.p[i] = P.p[(row0 + parent) * P.p_stride + x];
                S.q[i] = P.q ? P.q[(row0 + parent) * P.q_stride + x] : 1.f;
            }
        }
        if (bad) atomicOr(&S.status, bad);
    }
    __syncthreads();

    // The walk, by warp 0 (the same in all CTAs).
    int node = 0, at = 0, length = 0, n_gone = 0;
    double A = 0.0, Z = 1.0;
    bool summed = false;                         // S.all holds the sums of (node, A, gone); uniform over the CTA
    int pass = 0;
    auto walk = [&]() {
        if (S.status) return (int)kVtVoid;
        for (;;) {
            int next = -1;
            for (int b = at + 1; b < n && next < 0; b += 32) {
                const uint32_t hit = __ballot_sync(0xffffffffu, b + lane < n && S.parent[b + lane] == node);
                if (hit) next = b + __ffs(hit) - 1;
            }
            if (next < 0) return (int)kVtDraw;
            at = next;
            const float pf = S.p[next], qf = S.q[next];
            if (!(fabsf(pf) < INFINITY) || !(fabsf(qf) < INFINITY)) {
                if (lane == 0) S.status |= DSPARK_DEV_BAD_ROW;
                return (int)kVtVoid;
            }
            const double p = pf, q = qf, u = S.u[next];
            double left = P.q ? p - A * q : p;
            if (left < 0.0) left = 0.0;
            bool taken = false;                  // the token has been rejected here before
            for (int b = 0; b < n_gone; b += 32) taken = taken || __any_sync(0xffffffffu, b + lane < n_gone && S.gone[b + lane] == S.token[next]);
            if (taken) left = 0.0;
            if (u * q * Z < left) {
                if (lane == 0) S.path[length] = (short)next;
                ++length;
                node = next;
                A = 0.0; Z = 1.0; n_gone = 0;
                continue;
            }
            if (P.q) { A += Z; return (int)kVtPass; }
            Z -= left;
            if (!taken) {
                if (lane == 0) S.gone[n_gone] = S.token[next];
                ++n_gone;
                __syncwarp();
            }
        }
    };
    VtRow row;
    int v0 = (int)(rank * kVtWarps + warp) * P.run, v1 = v0 + P.run < P.V ? v0 + P.run : P.V;
    if (v0 > P.V) v0 = P.V;
    // S.all = inclusive sums of the runs, the same in every CTA
    auto sum_rows = [&]() {
        const long long at_row = row0 + S.node;
        row.p = P.p + at_row * P.p_stride;
        row.q = P.q ? P.q + at_row * P.q_stride : nullptr;
        row.A = S.A;
        row.gone = S.gone; row.n_gone = S.n_gone;
        row.vectors = (((uintptr_t)row.p | (uintptr_t)row.q) & 15) == 0;
        double sum = 0.0;
        for (int v = v0 + lane * 4; v - lane * 4 < v1; v += kVtLoads * 128) {
            float a[kVtLoads][4], b[kVtLoads][4];
#pragma unroll
            for (int j = 0; j < kVtLoads; ++j) row.load(v + j * 128, v1, a[j], b[j]);
#pragma unroll
            for (int j = 0; j < kVtLoads; ++j) {
                double four = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i) four += row.left(v + j * 128 + i, a[j][i], b[j][i]);
                sum += four;
            }
        }
        sum = warp_sum_f64(sum);
        if (lane == 0) S.sums[pass & 1][warp] = sum;
        vt_cluster_sync();
        if (warp == 0) {
            double x[4], run = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = lane * 4 + i;
                run += vt_remote(&S.sums[pass & 1][k % kVtWarps], k / kVtWarps);
                x[i] = run;
            }
            double before = run;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += y;
            }
            before = __shfl_up_sync(0xffffffffu, before, 1);
            if (lane == 0) before = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) S.all[lane * 4 + i] = before + x[i];
        }
        ++pass;
        __syncthreads();
    };
    auto publish = [&](int action) {
        if (warp == 0 && lane == 0) { S.action = action; S.node = node; S.A = A; S.n_gone = n_gone; S.length = length; }
        __syncthreads();
    };

    for (;;) {
        const int length_before = length;
        int action = warp == 0 ? walk() : 0;
        if (warp == 0 && length != length_before) summed = false;
        // a rejection changes A; a rejected chosen token is taken out of the row
        if (warp == 0 && (action == kVtPass || n_gone > 0)) summed = false;
        if (warp == 0 && lane == 0) S.action = action | (summed ? 4 : 0);
        __syncthreads();
        const int told = S.action;
        __syncthreads();
        publish(told & 3);
        if ((told & 3) == kVtVoid) break;
        if (!(told & 4)) sum_rows();
        summed = true;
        double total = S.all[kVtRuns - 1];
        if ((told & 3) == kVtDraw && total == 0.0 && (S.A != 0.0 || S.n_gone != 0)) {
            // nothing is left (only rounding can bring this about): the target itself
            A = 0.0; n_gone = 0;
            __syncthreads();
            publish(kVtDraw);
            sum_rows();
            total = S.all[kVtRuns - 1];
        }
        if (!(total < INFINITY) || ((told & 3) == kVtDraw && !(total > 0.0))) {
            __syncthreads();
            if (tid == 0) { S.status |= DSPARK_DEV_BAD_ROW; S.action = kVtVoid; }
            __syncthreads();
            break;
        }
        Z = total;
        if ((told & 3) == kVtDraw) break;
    }
    const bool voided = S.action == kVtVoid;
    const int len = voided ? 0 : S.length;
    if (!voided) {
        // the run that the drawn token is in: the first whose inclusive sum exceeds the target, else the last with a share
        const double total = S.all[kVtRuns - 1], target = (double)P.u_sample[r] * total;
        int owner = -1, last = 0;
        for (int b = 0; b < kVtRuns; b += 32) {
            const double here = S.all[b + lane], before = b + lane ? S.all[b + lane - 1] : 0.0;
            const uint32_t over = __ballot_sync(0xffffffffu, here > target), some = __ballot_sync(0xffffffffu, here > before);
            if (owner < 0 && over) owner = b + __ffs(over) - 1;
            if (some) last = b + 31 - __clz(some);
        }
        if (owner < 0) owner = last;
        if (owner == (int)rank * kVtWarps + warp) {
            double run = owner ? S.all[owner - 1] : 0.0;
            int pick = -1, fallback = -1;
            for (int v = v0; v < v1 && pick < 0; v += 128) {
                float a[4], b[4];
                double x[4];
                row.load(v + lane * 4, v1, a, b);
                double mine = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i) { mine += row.left(v + lane * 4 + i, a[i], b[i]); x[i] = mine; }
                double before = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += y;
                }
                const double block = __shfl_sync(0xffffffffu, before, 31);
                before -= mine;
                int first = -1, with = -1;
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    if (run + (before + x[i]) > target && x[i] > (i ? x[i - 1] : 0.0)) first = v + lane * 4 + i;
                    if (with < 0 && x[i] > (i ? x[i - 1] : 0.0)) with = v + lane * 4 + i;
                }
                const uint32_t over = __ballot_sync(0xffffffffu, first >= 0), some = __ballot_sync(0xffffffffu, with >= 0);
                if (over) pick = __shfl_sync(0xffffffffu, first, __ffs(over) - 1);
                if (some) fallback = __shfl_sync(0xffffffffu, with, 31 - __clz(some));
                run += block;
            }
            if (pick < 0) pick = fallback;
            if (lane == 0) P.out_tokens[row0 + len] = pick;
        }
    }
    if (rank == 0) {
        if (tid == 0) {
            P.accepted_len[r] = len;
            if (S.status) atomicOr(P.dev_status, S.status);
        }
        for (int i = tid; i < n; i += kVtThreads) {
            const bool on = i < len;
            if (P.out_path) P.out_path[row0 + i] = on ? S.path[i] : -1;
            if (voided || i != len) P.out_tokens[row0 + i] = on ? S.token[S.path[i]] : -1;
        }
    }
    vt_cluster_sync();                           // no CTA leaves while another may read its sums
}

}  // namespace dspark

extern "C" int dspark_verify_tree(const float* target_probs, int64_t target_row_stride, const float* draft_probs, int64_t draft_row_stride,
                                  int V, const int32_t* tokens, const int32_t* parents, const int32_t* row_offsets, int R, int n_rows,
                                  const float* u_accept, const float* u_sample, int32_t* accepted_len, int32_t* out_tokens,
                                  int32_t* out_path, int32_t* dev_status, void* stream)
{
    using namespace dspark;
    if (!target_probs || !tokens || !parents || !row_offsets || !u_accept || !u_sample || !accepted_len || !out_tokens || !dev_status ||
        V < 1 || R < 1 || n_rows < 1 || target_row_stride < V || (draft_probs && draft_row_stride < V))
        return DSPARK_ERR_INVALID_ARG;
    if (V > (1 << 24) || R > (1 << 20) || n_rows > (1 << 24)) return DSPARK_ERR_SHAPE;
    if (((uintptr_t)target_probs | (uintptr_t)draft_probs | (uintptr_t)tokens | (uintptr_t)parents | (uintptr_t)row_offsets |
         (uintptr_t)u_accept | (uintptr_t)u_sample | (uintptr_t)accepted_len | (uintptr_t)out_tokens | (uintptr_t)out_path |
         (uintptr_t)dev_status) & 3)
        return DSPARK_ERR_ALIGNMENT;
    VerifyTreeParams P = {};
    P.p = target_probs; P.p_stride = target_row_stride;
    P.q = draft_probs; P.q_stride = draft_row_stride;
    P.V = V;
    P.run = ((V + kVtRuns - 1) / kVtRuns + 127) / 128 * 128;
    P.tokens = tokens; P.parents = parents; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows;
    P.u_accept = u_accept; P.u_sample = u_sample;
    P.accepted_len = accepted_len; P.out_tokens = out_tokens; P.out_path = out_path; P.dev_status = dev_status;
    cudaStream_t s = (cudaStream_t)stream;
    KernelTimerScope timer(DSPARK_K_VERIFY_TREE, s);
    launch_pdl(verify_tree_kernel, dim3((unsigned)R * kVtCtas), dim3(kVtThreads), 0, s, P);
    return launch_status();
}
