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
//
// What bounds it: chains of dependent passes.  64 requests of 16 nodes and 128256 tokens with draft probabilities: 54 us (memory
// traffic of 66 MB alone 10 us), as long as the request with the most failed tests takes, each 3 to 4 us: four rounds of
// loads and a barrier of the cluster.  200 requests of 5-25 nodes and 50257 tokens without: 23 us, one of 6 nodes and 32000: 8 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "tree.cuh"

namespace moska {
namespace {
namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32;
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
    int range[2];
};

__device__ __forceinline__ float positive(float x) { return x > 0.f ? x : 0.f; }  // (NaN: 0)

template <int N>
struct Values {
    float x[N];
};

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
    static __device__ __forceinline__ Values<kVec> values(const uint4& w)
    {
        Values<kVec> y;
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                y.x[i] = __uint_as_float(word[i]);
            } else {
                y.x[2 * i] = __uint_as_float(word[i] << 16);
                y.x[2 * i + 1] = __uint_as_float(word[i] & 0xffff0000u);
            }
        }
        return y;
    }
    // elements v .. v + kVec - 1, those outside [0, V) as 0; `whole`: v + this row's shift is a multiple of kVec
    __device__ __forceinline__ Values<kVec> load(int v, int V, bool whole) const
    {
        if (whole && v >= 0 && v + kVec <= V) return values(__ldg(reinterpret_cast<const uint4*>(p + v)));
        Values<kVec> y;
#pragma unroll
        for (int i = 0; i < kVec; ++i) y.x[i] = v + i >= 0 && v + i < V ? at(v + i) : 0.f;
        return y;
    }
};

// What is left of p after `failed` tests, of N elements at once.
template <int N>
__device__ __forceinline__ void left_of(const float (&p)[N], const float (&q)[N], int failed, const double* inv, double (&r)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = positive(p[e]);
    if (failed == 0) return;
    double minus_q[N];
#pragma unroll
    for (int e = 0; e < N; ++e) minus_q[e] = -(double)positive(q[e]);
#pragma unroll 1
    for (int i = 0; i < failed; ++i) {
        const double f = inv[i];  // (1 at first)
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = fmax(fma(r[e], f, minus_q[e]), 0.0);
    }
}

// (three CTAs an SM: the pieces in flight of a thread are few)
template <class T, bool kDraft>
__global__ void __launch_bounds__(kThreads, 3) verify_kernel(const VerifyArgs a)
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
    auto left_of_piece = [&](int i, const Values<kVec>& p, const Values<kVec>& q, double (&x)[kVec]) {
        if constexpr (kDraft) {
            left_of(p.x, q.x, failed, sm.inv, x);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[e] = positive(p.x[e]);
            for (int f = 0; f < failed; ++f) {
                const int at = sm.removed[f] - (i * kVec - shift);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (e == at) x[e] = 0.0;
            }
        }
    };
    auto left = [&](int i, double (&x)[kVec]) {
        Values<kVec> p, q;
        p = target_row(cur).load(i * kVec - shift, V, true);
        if constexpr (kDraft)
            if (failed > 0) q = draft_row(cur).load(i * kVec - shift, V, q_whole);
        left_of_piece(i, p, q, x);
    };
    // what is left in pieces begin .. end - 1, over the warp
    auto sum_of = [&](int begin, int end) {
        double s = 0.0;
        // Whole pieces, kAhead of a lane's in flight; then the ends of the row (and all of it where the two rows are aligned
        // differently), one by one.
        constexpr int kAhead = sizeof(T) == 4 ? 4 : 2;  // (bf16 has twice the elements in a piece: 4 spill)
        const int whole0 = q_whole ? max(begin, shift > 0 ? 1 : 0) : end, whole1 = q_whole ? min(end, (V + shift) / kVec) : end;
        const uint4* p = reinterpret_cast<const uint4*>(target_row(cur).p - shift);
        const uint4* q = kDraft ? reinterpret_cast<const uint4*>(draft_row(cur).p - shift) : nullptr;
        for (int i0 = whole0; i0 < whole1; i0 += 32 * kAhead) {
            uint4 pw[kAhead], qw[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = i0 + 32 * u + lane;
                pw[u] = i < whole1 ? __ldg(p + i) : make_uint4(0, 0, 0, 0);
                if constexpr (kDraft) qw[u] = failed > 0 && i < whole1 ? __ldg(q + i) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                double x[kVec];
                left_of_piece(i0 + 32 * u + lane, Row<T>::values(pw[u]), Row<T>::values(qw[u]), x);
#pragma unroll
                for (int e = 0; e < kVec; ++e) s += x[e];
            }
        }
        auto one = [&](int at) {
            double x[kVec];
            left(at, x);
#pragma unroll
            for (int e = 0; e < kVec; ++e) s += x[e];
        };
        for (int at = begin + lane; at < min(end, whole0); at += 32) one(at);
        for (int at = max(whole0, whole1) + lane; at < end; at += 32) one(at);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        return s;
    };
    auto sum_pass = [&] {
        split();
        const double s = sum_of(piece0, piece1);
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
            const float p1[1] = {sm.p[j]}, q1[1] = {sm.q[j]};
            double r1[1];
            left_of(p1, q1, failed, sm.inv, r1);
            px = r1[0];
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
    // the part in which `sum` (its kWarps parts' sums) passes the goal, and what is before it; the last with anything, should
    // rounding leave none
    auto part_of = [&](const double* sum) {
        int at = -1;
        double upto = base;
        for (int w = 0; w < kWarps; ++w) {
            if (!(sum[w] > 0.0)) continue;
            at = w;
            base = upto;
            upto += sum[w];
            if (upto > goal) break;
        }
        return at;
    };
    int at = part_of(sm.warp_sum);
    if (lane == 0 && warp == at) {
        sm.range[0] = piece0;
        sm.range[1] = piece1;
    }
    __syncthreads();
    // that warp's pieces among all warps once more, until one load does for what is left (one warp alone would go through them
    // for as long as a pass takes)
    int begin = sm.range[0], end = sm.range[1];
    while (end - begin > 32) {
        const int per = (end - begin + kWarps - 1) / kWarps;
        piece0 = min(end, begin + warp * per);
        piece1 = min(end, piece0 + per);
        const double mine = sum_of(piece0, piece1);
        __syncthreads();
        if (lane == 0) sm.warp_sum[warp] = mine;
        __syncthreads();
        const int next = part_of(sm.warp_sum);
        if (next >= 0) at = next;
        begin = min(end, begin + at * per);
        end = min(end, begin + per);
    }
    if (warp > 0) return;
    piece0 = begin;
    piece1 = end;
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
    // CTAs of a request, 1, 2, 4 or 8.  A pass is a chain of loads, so that more of them make it shorter while a part is more than a few
    // loads (one request of 6 nodes and 32000 tokens: 22.5, 18.4, 14.3, 12.4 us, caches flushed as in what follows).  Without draft
    // probabilities a request has one pass and a short search, and pays for CTAs that find no place (444 at a time): 5-25 nodes and
    // 50257 tokens, 100 requests 31, 25, 23, 31 us, 150 33, 26, 33, 41, 300 38, 45, 51, 67.  With them the request with the most
    // passes takes longest, and others' CTAs fill the gaps: 16 nodes and 128256 tokens, 50 requests 165, 95, 60, 52 us, 99 195, 119,
    // 85, 81, 200 213, 149, 135, 132.
    const long long most = draft != nullptr ? 1600 : 400;  // CTAs
    int cluster = 1;
    while (cluster < kMaxCluster && V / cluster > 2048 && 2LL * tree.n_requests * cluster <= most) cluster *= 2;
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
