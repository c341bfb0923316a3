// dspark_verify_tree: lossless verification of a tree of drafted tokens from given random numbers (Section 2.1's rule,
// repeated over the children of a node).
//
// At node u with target p, drafter q and children c_1, c_2, ..: a child is accepted with probability min(1, r / (Z q)) at its
// token, r being what is left of p after the rejections before it.  The residual of a rejection is max(r - Z q, 0), and
// max(max(p - a q, 0) - b q, 0) = max(p - (a + b) q, 0) for q >= 0: whatever was rejected, r = max(p - A q, 0) with one number
// A, so a rejection costs one pass over the two rows for the new Z = sum r and nothing is stored.
//
// One cluster of eight CTAs per request.  Every CTA makes the walk itself, from the scalars p(x), q(x), u of all nodes, gathered
// at once; a pass over the vocabulary is shared: each warp owns a run of it, and the runs' sums pass through distributed
// shared memory, so that all CTAs go on with the same numbers.  The sums of the last pass are those of the draw, for which only the
// CTA that owns the drawn token's run reads it again.  Sums and tests are fp64: what decides is a border between tokens.
//
// Bound by the chain of dependent steps.  Clocks of one tree (16 nodes, one rejection, 129280 entries): 1300 for the offsets, 3600 for
// nodes and their scalars, 4000 for the first walk (1200 for later ones), 5000 for the pass over two rows, 2700 to join its sums,
// 2000 for the draw: 11.4 us.  128 trees of 32 nodes, 2.2 such passes each on average, the slowest 5: 58 us, 188 MB, 3.2 TB/s.
#include <math.h>

#include "common.cuh"

namespace dspark {

constexpr int kVtCtas = 8, kVtMaxWarps = 16, kVtMaxRuns = kVtCtas * kVtMaxWarps;
constexpr int kVtLoads = 4;                      // vectors of a run in flight in one lane

struct VerifyTreeParams {
    const float* p; long long p_stride;
    const float* q; long long q_stride;
    int V, run;                                  // run: entries of one warp, a multiple of 128
    int warps;                                   // of a CTA
    const int32_t* tokens; const int32_t* parents; const int32_t* row_offsets;
    int R, n_rows;
    const float* u_accept; const float* u_sample;
    int32_t* accepted_len; int32_t* out_tokens; int32_t* out_path; int32_t* dev_status;
};

enum VtAction { kVtPass = 0, kVtDraw = 1, kVtVoid = 2, kVtSummed = 4 };

struct VtShared {
    double sums[2][kVtMaxWarps];                    // read by the other CTAs; one set a pass, in turn
    double all[kVtMaxRuns];                      // inclusive sums of all runs
    double share[kVtMaxRuns];                    // the runs' own sums
    double A;
    double block[2][kVtMaxWarps];
    int action, node, length, n_gone, status, pick;
    short parent[DSPARK_TREE_MAX_NODES], path[DSPARK_TREE_MAX_NODES];
    int token[DSPARK_TREE_MAX_NODES], gone[DSPARK_TREE_MAX_NODES];
    float p[DSPARK_TREE_MAX_NODES], q[DSPARK_TREE_MAX_NODES], u[DSPARK_TREE_MAX_NODES];
};

__device__ __forceinline__ void vt_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void vt_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ double vt_remote(const double* local, uint32_t rank)
{
    uint32_t a;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
    return v;
}

// The bits of a float in a double's place: its value times 2^-896, exactly, zero and the smallest included.  Two shifts where the
// conversion, a quarter as wide, would bound the pass.  Not so for a sign, an infinity or NaN: their bits are above those of all others.
__device__ __forceinline__ double vt_scaled(uint32_t bits) { return __hiloint2double((int)(bits >> 3), (int)(bits << 29)); }
constexpr uint32_t kVtPlainBits = 0x7f800000u;

// What is left of a row: max(p - A q, 0), or p without the rejected tokens.  NaN stays.
struct VtRow {
    const float* p; const float* q;              // q == nullptr: p alone
    double A;
    const int* gone; int n_gone;
    bool vectors;
    __device__ __forceinline__ double left(int v) const
    {
        double r = q ? (double)p[v] - A * (double)q[v] : (double)p[v];
        if (r < 0.0) r = 0.0;
        for (int i = 0; i < n_gone; ++i)
            if (gone[i] == v) r = 0.0;
        return r;
    }
    // a lane's part of the sum over [v0, v1), by the warp
    __device__ double sum(int v0, int v1, int lane) const
    {
        bool any = false;
        for (int i = 0; i < n_gone; ++i) any = any || (gone[i] >= v0 && gone[i] < v1);
        if (vectors && !any) {
            double s[4] = {0.0, 0.0, 0.0, 0.0};
            uint32_t most = 0;
            for (int v = v0; v < v1; v += kVtLoads * 128) {
                uint4 a[kVtLoads], b[kVtLoads];
#pragma unroll
                for (int j = 0; j < kVtLoads; ++j) {
                    const int at = v + j * 128 + lane * 4;
                    a[j] = b[j] = make_uint4(0, 0, 0, 0);
                    if (at + 4 <= v1) {
                        a[j] = *reinterpret_cast<const uint4*>(p + at);
                        if (q) b[j] = *reinterpret_cast<const uint4*>(q + at);
                    }
                }
#pragma unroll
                for (int j = 0; j < kVtLoads; ++j) {
                    const uint32_t x[4] = {a[j].x, a[j].y, a[j].z, a[j].w}, y[4] = {b[j].x, b[j].y, b[j].z, b[j].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        most = max(most, max(x[i], y[i]));
                        const double r = vt_scaled(x[i]) - A * vt_scaled(y[i]);
                        s[i] += r < 0.0 ? 0.0 : r;
                    }
                }
            }
            double all = ((s[0] + s[1]) + (s[2] + s[3])) * 0x1p896;
            const int end = v1 & ~3;             // up to three entries are left where the row ends
            if (end >= v0 && lane < v1 - end) all += left(end + lane);
            if (!__any_sync(0xffffffffu, most >= kVtPlainBits)) return all;
        }
        double all = 0.0;
#pragma unroll 4
        for (int v = v0 + lane; v < v1; v += 32) all += left(v);
        return all;
    }
};

__global__ void __cluster_dims__(kVtCtas, 1, 1) __launch_bounds__(kVtMaxWarps * 32, 2) verify_tree_kernel(const __grid_constant__ VerifyTreeParams P)
{
    __shared__ VtShared S;
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int r = blockIdx.x / kVtCtas, rank = blockIdx.x % kVtCtas, runs = kVtCtas * P.warps;
    const int row0 = P.row_offsets[r], end = P.row_offsets[r + 1], n = end - row0;
    const bool there = row0 >= 0 && end >= row0 && end <= P.n_rows;
    if (!there || n == 0) {                      // the whole cluster; a request without rows is nothing to do
        if (rank == 0 && tid == 0) {
            P.accepted_len[r] = 0;
            if (!there) atomicOr(P.dev_status, DSPARK_DEV_BAD_OFFSETS);
        }
        return;
    }
    if (tid == 0) S.status = n > DSPARK_TREE_MAX_NODES ? DSPARK_DEV_BAD_OFFSETS : 0;
    __syncthreads();
    if (n <= DSPARK_TREE_MAX_NODES) {
        int bad = 0;
        for (int i = 1 + tid; i < n; i += blockDim.x) {
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
    int v0 = (rank * P.warps + warp) * P.run, v1 = v0 + P.run < P.V ? v0 + P.run : P.V;
    if (v0 > P.V) v0 = P.V;
    // S.all = inclusive sums of the runs, S.share their own, the same in every CTA
    auto sum_rows = [&]() {
        const long long at_row = row0 + S.node;
        row.p = P.p + at_row * P.p_stride;
        row.A = S.A;
        row.q = P.q && row.A != 0.0 ? P.q + at_row * P.q_stride : nullptr;  // nothing rejected: the target alone
        row.gone = S.gone; row.n_gone = S.n_gone;
        row.vectors = (((uintptr_t)row.p | (uintptr_t)row.q) & 15) == 0;
        const double sum = warp_sum_f64(row.sum(v0, v1, lane));
        if (lane == 0) S.sums[pass & 1][warp] = sum;
        vt_cluster_arrive();
        vt_cluster_wait();
        if (warp == 0) {
            double x[4], run = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = lane * 4 + i, at = k < runs ? k : 0;
                x[i] = vt_remote(&S.sums[pass & 1][at % P.warps], at / P.warps);
                if (k >= runs) x[i] = 0.0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                S.share[lane * 4 + i] = x[i];
                x[i] = run += x[i];
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
    // What warp 0 has come to.  The others read it before sum_rows' last barrier, behind which it may change again.
    auto publish = [&](int action) {
        if (warp == 0 && lane == 0) { S.action = action; S.node = node; S.A = A; S.n_gone = n_gone; S.length = length; }
        __syncthreads();
    };

    bool voided;
    for (;;) {
        int action = 0;
        if (warp == 0) {
            const int length_before = length;
            action = walk();
            // a rejection changes A, or takes a token out of the row
            if (length != length_before || action == kVtPass || n_gone > 0) summed = false;
        }
        publish(action | (summed ? kVtSummed : 0));
        const int told = S.action & ~kVtSummed;
        voided = told == kVtVoid;
        if (voided) break;
        if (!(S.action & kVtSummed)) sum_rows();
        summed = true;
        Z = S.all[kVtMaxRuns - 1];
        if (told == kVtDraw && Z == 0.0 && (S.A != 0.0 || S.n_gone != 0)) {
            // nothing is left (only rounding can bring this about): the target itself
            A = 0.0; n_gone = 0;
            __syncthreads();
            publish(kVtDraw);
            sum_rows();
            Z = S.all[kVtMaxRuns - 1];
        }
        if (!(Z < INFINITY) || (told == kVtDraw && !(Z > 0.0))) {
            voided = true;
            if (tid == 0) S.status |= DSPARK_DEV_BAD_ROW;
        }
        if (voided || told == kVtDraw) break;
    }
    vt_cluster_arrive();
    const int len = voided ? 0 : S.length;
    if (!voided) {
        // the run that the drawn token is in: of those with a share the first whose inclusive sum exceeds the target, else the last
        // (the inclusive sums are rounded in different orders: one without a share can be a step above the one before it)
        const double total = S.all[kVtMaxRuns - 1], target = (double)P.u_sample[r] * total;
        int owner = -1, last = 0;
        for (int b = 0; b < runs; b += 32) {
            const bool share = S.share[b + lane] > 0.0;
            const uint32_t over = __ballot_sync(0xffffffffu, share && S.all[b + lane] > target), some = __ballot_sync(0xffffffffu, share);
            if (owner < 0 && over) owner = b + __ffs(over) - 1;
            if (some) last = b + 31 - __clz(some);
        }
        if (owner < 0) owner = last;
        if (owner / P.warps == rank) {
            // The CTA that has it, a block of 128 entries a warp: the first in which the target is passed, else the last with a share.
            const int begin = owner * P.run, stop = min(begin + P.run, P.V);
            double run = owner ? S.all[owner - 1] : 0.0;
            bool found = false;
            if (tid == 0) S.pick = -1;
            int round = 0;
            for (int v = begin; v < stop && !found; v += P.warps * 128, ++round) {
                const int at = v + warp * 128 + lane * 4;
                double x[4], upto = 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double e = at + i < stop ? row.left(at + i) : 0.0;
                    x[i] = upto += e;
                }
                double before = upto;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += y;
                }
                if (lane == 31) S.block[round & 1][warp] = before;
                __syncthreads();
                // the blocks' sums up to each, by every warp
                const double block = lane < P.warps ? S.block[round & 1][lane] : 0.0;
                double blocks = block;
#pragma unroll
                for (int o = 1; o < kVtMaxWarps; o <<= 1) {
                    const double y = __shfl_up_sync(0xffffffffu, blocks, o);
                    if (lane >= o) blocks += y;
                }
                const uint32_t over = __ballot_sync(0xffffffffu, block > 0.0 && run + blocks > target), some = __ballot_sync(0xffffffffu, block > 0.0);
                found = over != 0;
                const int mine = found ? __ffs(over) - 1 : 31 - __clz(some);          // the block to look into
                const double base = run + __shfl_sync(0xffffffffu, blocks - block, warp);
                if (warp == mine) {
                    before -= upto;
                    int first = -1, last = -1;
#pragma unroll
                    for (int i = 3; i >= 0; --i) {
                        const bool share = x[i] > (i ? x[i - 1] : 0.0);
                        if (share && base + (before + x[i]) > target) first = at + i;
                        if (share && last < 0) last = at + i;
                    }
                    const uint32_t passed = __ballot_sync(0xffffffffu, first >= 0), shares = __ballot_sync(0xffffffffu, last >= 0);
                    const int pick = __shfl_sync(0xffffffffu, passed ? first : last, passed ? __ffs(passed) - 1 : 31 - __clz(shares));
                    if (lane == 0) S.pick = pick;
                }
                run += __shfl_sync(0xffffffffu, blocks, P.warps - 1);
            }
            __syncthreads();
            if (tid == 0) P.out_tokens[row0 + len] = S.pick;
        }
    }
    if (rank == 0) {
        if (tid == 0) {
            P.accepted_len[r] = len;
            if (S.status) atomicOr(P.dev_status, S.status);
        }
        for (int i = tid; i < n; i += blockDim.x) {
            const bool on = i < len;
            if (P.out_path) P.out_path[row0 + i] = on ? S.path[i] : -1;
            if (voided || i != len) P.out_tokens[row0 + i] = on ? S.token[S.path[i]] : -1;
        }
    }
    vt_cluster_wait();                           // no CTA leaves while another may read its sums
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
    // The CTAs of a cluster make the same walk from the same inputs, at times of their own: one that found a result there in place of an
    // input would take another way and meet the others at the wrong barrier.
    const size_t rows = (size_t)n_rows * 4, requests = (size_t)R * 4;
    const struct { const void* at; size_t bytes; } arrays[] = {
        {accepted_len, requests}, {out_tokens, rows}, {out_path, rows}, {dev_status, 4},       // the outputs
        {target_probs, ((size_t)(n_rows - 1) * target_row_stride + V) * 4},
        {draft_probs, draft_probs ? ((size_t)(n_rows - 1) * draft_row_stride + V) * 4 : 0},
        {tokens, rows}, {parents, rows}, {row_offsets, requests + 4}, {u_accept, rows}, {u_sample, requests}};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < (int)(sizeof arrays / sizeof arrays[0]); ++j)
            if (ranges_meet(arrays[i].at, arrays[i].bytes, arrays[j].at, arrays[j].bytes)) return DSPARK_ERR_INVALID_ARG;
    VerifyTreeParams P = {};
    P.p = target_probs; P.p_stride = target_row_stride;
    P.q = draft_probs; P.q_stride = draft_row_stride;
    P.V = V;
    // 16 warps where the requests fill the device once at most, two CTAs an SM (129280 entries: 1 tree 11.4 us, with 8 warps 12.5; 16 trees
    // 23.9 and 25.7); else 8, four CTAs an SM, so that more walks run beside each other's passes (40 trees of 32000 entries: 20.6
    // us, with 16 warps 24.8; 128 of 129280: 57.9 and 74.3)
    P.warps = R * kVtCtas <= 2 * current_sms() ? kVtMaxWarps : kVtMaxWarps / 2;
    const int runs = kVtCtas * P.warps;
    P.run = ((V + runs - 1) / runs + 127) / 128 * 128;
    P.tokens = tokens; P.parents = parents; P.row_offsets = row_offsets; P.R = R; P.n_rows = n_rows;
    P.u_accept = u_accept; P.u_sample = u_sample;
    P.accepted_len = accepted_len; P.out_tokens = out_tokens; P.out_path = out_path; P.dev_status = dev_status;
    cudaStream_t s = (cudaStream_t)stream;
    KernelTimerScope timer(DSPARK_K_VERIFY_TREE, s);
    launch_pdl(verify_tree_kernel, dim3((unsigned)R * kVtCtas), dim3(P.warps * 32), 0, s, P);
    return launch_status();
}
