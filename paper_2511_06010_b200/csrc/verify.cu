// Verification of drafted tokens against the target's probabilities (include/moska.h has the walk).
//
// A cluster of CTAs per request: every CTA follows the whole walk in its own shared memory (the probabilities of the
// tree's tokens are at most 64 numbers), and each takes an equal part of the vocabulary where a whole row is needed: the sum of
// what a failed test leaves, and the search for the next token.  Such a pass reads the row once (again, from L2, for
// each further test that fails at the same node): what is left after k failed tests is computed anew from p and
// q and the k - 1 sums before, r_{i+1} = max(r_i / Z_i - q, 0), in registers.  Sums of the CTAs meet in shared memory of the cluster, one
// barrier a pass.  Everything is summed in 64 bits: a token is picked by which side of a border a sum falls, and
// 100K terms in 32 bits would move that border over many tokens.  Every CTA adds the same numbers in the same
// order, so that all decide alike, and the results do not change from run to run.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "tree.cuh"

namespace moska {
namespace {
namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;  // the portable size
constexpr int kNodes = MOSKA_TREE_MAX_NODES;

struct VerifyArgs {
    const void* target;
    const void* draft;
    int64_t target_stride, draft_stride;
    const int32_t* tokens;
    const float* u_accept;
    const float* u_next;
    TreeRows tree;
    int32_t* path;
    int32_t* n_path;
    int32_t* next_token;
    int* status;
    int V;
};

struct VerifySmem {
    int up[kNodes], token[kNodes];
    float u[kNodes];
    float p[kNodes], q[kNodes];      // target's and draft's probability of a node's token behind its parent
    double inv[kNodes];              // 1 / Z of the failed tests at the current node
    int removed[kNodes];             // without draft probabilities: tokens that failed there
    double warp_sum[kWarps];
    double cta_sum[2][kMaxCluster];  // of all CTAs of the cluster; passes alternate
    int path[kNodes];
};

__device__ __forceinline__ float positive(float x) { return x > 0.f ? x : 0.f; }  // (NaN: 0)

// A row of probabilities from its first element on: 16-byte pieces of kVec elements that lie on 16-byte boundaries; element v
// of the row is element v + shift of the pieces.
template <class T>
struct Row {
    static constexpr int kVec = 16 / sizeof(T);
    const T* p;
    __device__ __forceinline__ int shift() const { return (int)((reinterpret_cast<uintptr_t>(p) % 16) / sizeof(T)); }
    __device__ __forceinline__ float at(int v) const
    {
        if constexpr (sizeof(T) == 4) return __ldg(reinterpret_cast<const float*>(p) + v);
        else return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p) + v) << 16);
    }
    // elements v .. v + kVec - 1, those outside [0, V) as 0; `whole`: v + this row's shift is a multiple of kVec
    __device__ __forceinline__ void load(int v, int V, bool whole, float (&x)[kVec]) const
    {
        if (whole && v >= 0 && v + kVec <= V) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(p + v));
            const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 4) {
                    x[i] = __uint_as_float(word[i]);
                } else {
                    x[2 * i] = __uint_as_float(word[i] << 16);
                    x[2 * i + 1] = __uint_as_float(word[i] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = v + i >= 0 && v + i < V ? at(v + i) : 0.f;
        }
    }
};

// What is left of p after `failed` tests.
__device__ __forceinline__ double left_of(float p, float q, int failed, const double* inv)
{
    double r = positive(p);
    const double qd = positive(q);
    for (int i = 0; i < failed; ++i) {
        r = (i == 0 ? r : r * inv[i]) - qd;
        r = r > 0.0 ? r : 0.0;
    }
    return r;
}

template <class T, bool kDraft>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs a)
{
    __shared__ VerifySmem sm;
    const cg::cluster_group cluster = cg::this_cluster();
    cluster.barrier_arrive();  // all CTAs have to have begun before one writes another's memory
    const int n_ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int r = blockIdx.x / n_ctas;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int2 rows = tree_rows(a.tree, r, a.status);
    const int n = rows.y, V = a.V;
    auto target_row = [&](int i) { return Row<T>{static_cast<const T*>(a.target) + (rows.x + i) * a.target_stride}; };
    auto draft_row = [&](int i) { return Row<T>{static_cast<const T*>(a.draft) + (rows.x + i) * a.draft_stride}; };
    if (tid < n) {
        const int up = tree_parent(a.tree, rows.x, tid, a.status), x = __ldg(a.tokens + rows.x + tid);
        const bool tried = up >= 0 && x >= 0 && x < V;
        sm.up[tid] = tried ? up : -1;
        sm.token[tid] = x;
        sm.u[tid] = __ldg(a.u_accept + rows.x + tid);
        sm.p[tid] = tried ? positive(target_row(up).at(x)) : 0.f;
        if constexpr (kDraft) sm.q[tid] = tried ? positive(draft_row(up).at(x)) : 0.f;
    }
    const double u_next = (double)__ldg(a.u_next + r);
    __syncthreads();
    cluster.barrier_wait();

    int pass = 0;
    int n_path = n > 0 ? 1 : 0, cur = 0, failed = 0;
    double z = 1.0, total = 0.0;  // total: of the last pass, if it was over what is left now
    bool summed = false;
    // this CTA's part of the vocabulary, and this warp's part of that, in pieces of kVec elements
    constexpr int kVec = Row<T>::kVec;
    int piece0 = 0, piece1 = 0, shift = 0;
    bool q_whole = true;
    auto split = [&] {  // of the current rows
        const Row<T> p = target_row(cur);
        shift = p.shift();
        if constexpr (kDraft) q_whole = draft_row(cur).shift() == shift;
        const int pieces = (V + shift + kVec - 1) / kVec;
        const int per_cta = (pieces + n_ctas - 1) / n_ctas, per_warp = (per_cta + kWarps - 1) / kWarps;
        const int c0 = min(pieces, rank * per_cta), c1 = min(pieces, c0 + per_cta);
        piece0 = min(c1, c0 + warp * per_warp);
        piece1 = min(c1, piece0 + per_warp);
    };
    // elements of piece i: what is left of them after `failed` tests
    auto left = [&](int i, double (&x)[kVec]) {
        const int v = i * kVec - shift;
        float p[kVec], q[kVec];
        target_row(cur).load(v, V, true, p);
        if constexpr (kDraft) {
            if (failed > 0) draft_row(cur).load(v, V, q_whole, q);
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[e] = left_of(p[e], q[e], failed, sm.inv);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[e] = positive(p[e]);
            for (int f = 0; f < failed; ++f) {
                const int at = sm.removed[f] - v;
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (e == at) x[e] = 0.0;
            }
        }
    };
    auto sum_pass = [&] {
        split();
        double s = 0.0;
        for (int i = piece0 + lane; i < piece1; i += 32) {
            double x[kVec];
            left(i, x);
#pragma unroll
            for (int e = 0; e < kVec; ++e) s += x[e];
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        if (lane == 0) sm.warp_sum[warp] = s;
        __syncthreads();
        double mine = 0.0;
        for (int w = 0; w < kWarps; ++w) mine += sm.warp_sum[w];
        double* slot = &sm.cta_sum[pass & 1][rank];
        if (tid < n_ctas) *cluster.map_shared_rank(slot, tid) = mine;
        cluster.sync();
        total = 0.0;
        for (int c = 0; c < n_ctas; ++c) total += sm.cta_sum[pass & 1][c];
        ++pass;
    };

    if (tid == 0 && n > 0) sm.path[0] = 0;
    for (int j = 1; j < n; ++j) {
        if (sm.up[j] != cur) continue;
        const int x = sm.token[j];
        double px;
        if constexpr (kDraft) {
            px = left_of(sm.p[j], sm.q[j], failed, sm.inv);
        } else {
            px = sm.p[j];
            for (int f = 0; f < failed; ++f)
                if (sm.removed[f] == x) px = 0.0;
        }
        const double q = kDraft ? (double)sm.q[j] : 1.0;
        if (px > 0.0 && (double)sm.u[j] * q * z < px) {
            cur = j;
            if (tid == 0) sm.path[n_path] = j;
            ++n_path;
            failed = 0;
            z = 1.0;
            summed = false;
        } else if constexpr (kDraft) {
            __syncthreads();  // (inv was read by the pass before)
            if (tid == 0) sm.inv[failed] = 1.0 / z;
            __syncthreads();
            ++failed;
            sum_pass();
            summed = true;
            if (total > 0.0) {
                z = total;
            } else {  // nothing is left: as before this test
                --failed;
                summed = false;
            }
        } else {
            __syncthreads();
            if (tid == 0) sm.removed[failed] = x;
            __syncthreads();
            ++failed;
            z -= px;
        }
    }
    if (n > 0 && !summed) sum_pass();
    __syncthreads();

    if (rank == 0) {
        if (tid < a.tree.max_nodes) a.path[(int64_t)r * a.tree.max_nodes + tid] = tid < n_path ? sm.path[tid] : -1;
        if (tid == 0) {
            a.n_path[r] = n_path;
            if (n == 0 || !(total > 0.0)) a.next_token[r] = -1;
        }
    }
    if (n == 0 || !(total > 0.0)) return;

    // ---- the next token: the CTA, then the warp, then the piece in which the sum passes the goal
    const double goal = u_next * total;
    const double* sums = sm.cta_sum[(pass - 1) & 1];
    double before = 0.0, base = 0.0;
    int cta = -1;
    for (int c = 0; c < n_ctas; ++c) {
        if (!(sums[c] > 0.0)) continue;
        cta = c;  // (the last with anything, should rounding leave none)
        base = before;
        before += sums[c];
        if (before > goal) break;
    }
    if (cta != rank) return;
    int at = -1;
    before = base;
    for (int w = 0; w < kWarps; ++w) {
        if (!(sm.warp_sum[w] > 0.0)) continue;
        at = w;
        base = before;
        before += sm.warp_sum[w];
        if (before > goal) break;
    }
    if (at != warp) return;
    int last = -1;
    for (int i0 = piece0; i0 < piece1; i0 += 32) {
        const int i = i0 + lane;
        double x[kVec], s = 0.0;
        if (i < piece1) left(i, x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            if (i >= piece1) x[e] = 0.0;
            s += x[e];
        }
        double upto = s;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += y;
        }
        double c = base + (upto - s);
        int found = -1, seen = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            c += x[e];
            if (x[e] > 0.0) {
                seen = i * kVec - shift + e;
                if (found < 0 && c > goal) found = seen;
            }
        }
        const unsigned hit = __ballot_sync(0xffffffffu, found >= 0), any = __ballot_sync(0xffffffffu, seen >= 0);
        if (hit != 0) {
            last = __shfl_sync(0xffffffffu, found, __ffs(hit) - 1);
            break;
        }
        if (any != 0) last = __shfl_sync(0xffffffffu, seen, 31 - __clz(any));
        base += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) a.next_token[r] = last;
}

}  // namespace

int launch_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, bool bf16, int V,
                  const int32_t* tokens, const float* u_accept, const float* u_next, const TreeRows& tree, int32_t* path,
                  int32_t* n_path, int32_t* next_token, int* status, cudaStream_t st)
{
    if (tree.n_requests == 0) return MOSKA_OK;
    int cluster = 1;
    while (cluster < kMaxCluster && V / cluster > 8192 && (long long)tree.n_requests * cluster < 592) cluster *= 2;
    const long long grid = (long long)tree.n_requests * cluster;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "verification grid too large");
    const VerifyArgs a{target, draft, target_stride, draft_stride, tokens, u_accept, u_next, tree, path, n_path, next_token,
                       status, V};
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)grid);
    config.blockDim = dim3(kThreads);
    config.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    config.attrs = &attr;
    config.numAttrs = 1;
    const auto kernel = bf16 ? (draft != nullptr ? verify_kernel<__nv_bfloat16, true> : verify_kernel<__nv_bfloat16, false>)
                             : (draft != nullptr ? verify_kernel<float, true> : verify_kernel<float, false>);
    MOSKA_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, a));
    return MOSKA_OK;
}

}  // namespace moska
