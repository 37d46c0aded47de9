// Keeping the accepted path of a drafted tree: the rows of its nodes move to the places behind the committed
// context, as bytes.  A path is ascending and starts no earlier than its place (path[j] >= j), so that a row's new
// place is never the source of a later one: with every thread owning the same bytes of all rows, moving them in
// order (loads of up to eight rows before their stores) needs no barrier.  Bound by the chain path -> page -> row -> stores: 64
// requests of 16 nodes 5 us with the call, 512 of 64 nodes in bf16 9 to 10 us (34 MB read and written), 300 of 33 in 4 bits 11 us
// (one launch alone).
#include "tree.cuh"

namespace moska {
namespace {

constexpr int kThreads = 128, kAhead = 8;  // (512 requests of 64 nodes: 8.6 us; 9.5 with 256 threads, 10.6 with 16 rows ahead)

struct CommitArgs {
    PagedView kv;
    TreeRows tree;
    const int32_t* path;
    const int32_t* n_path;
    int32_t* kv_len_out;
    int path_stride, Hkv, parts;
};

// Items of a row: bf16, 16-byte pieces of the key row and then of the value row.  4 bits, for every head 18 pieces of D / 16
// bytes: key codes (8), value codes (8: one of each chunk), key scales, value scales.
template <int D, bool F4>
__global__ void __launch_bounds__(kThreads) commit_kernel(const CommitArgs a)
{
    __shared__ int64_t from[MOSKA_TREE_MAX_NODES], to[MOSKA_TREE_MAX_NODES];  // token rows (page * page_size + row)
    __shared__ int source[MOSKA_TREE_MAX_NODES];
    const int r = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x;
    bool good;
    const int2 rows = tree_rows(a.tree, r, a.kv.status, &good);
    const int len = __ldg(a.kv.kv_len + r);
    good &= checked_len(a.kv, len) == len;  // (with rows or a length that are none, the place of the nodes is not known)
    const int committed = good ? len - rows.y : -1;
    const int given = __ldg(a.n_path + r);
    good &= given >= 0 && given <= min(rows.y, a.path_stride);
    const int n = good ? given : 0;
    int x = 0;
    if (tid < n) {
        x = __ldg(a.path + (int64_t)r * a.path_stride + tid);
        good = x >= 0 && x < rows.y;
        source[tid] = x;
    }
    __syncthreads();
    if (tid > 0 && tid < n) good &= source[tid - 1] < x;
    const int shift = a.kv.page_shift, in_page = (1 << shift) - 1;
    const int32_t* pages = a.kv.page_table + (int64_t)r * a.kv.max_pages;
    if (tid < n && good && committed >= 0) {
        const int t = committed + tid, f = committed + x;
        const int pt = __ldg(pages + (t >> shift)), pf = __ldg(pages + (f >> shift));
        good = (unsigned)pt < (unsigned)a.kv.n_pages && (unsigned)pf < (unsigned)a.kv.n_pages;
        to[tid] = ((int64_t)pt << shift) + (t & in_page);
        from[tid] = ((int64_t)pf << shift) + (f & in_page);
    }
    good = __syncthreads_and(good);  // (else, or with a page that is not in the pool, nothing is moved)
    if (part == 0 && tid == 0) {
        a.kv_len_out[r] = good && committed >= 0 ? committed + n : len;  // (`good` of all threads: the path and its pages too)
        if (!good) atomicMin(a.kv.status, MOSKA_ERR_INVALID_ARG);
    }
    if (!good || committed < 0) return;
    int skip = 0;  // rows that are where they belong
    while (skip < n && source[skip] == skip) ++skip;

    const int item = part * kThreads + tid;
    if constexpr (!F4) {
        const int pieces = a.Hkv * D / 8;
        if (item >= 2 * pieces) return;
        uint8_t* base = (item < pieces ? a.kv.k : a.kv.v) + (int64_t)(item % pieces) * 16;
        const int64_t row_bytes = (int64_t)a.Hkv * D * 2;
        for (int j0 = skip; j0 < n; j0 += kAhead) {
            uint4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (j0 + u < n) v[u] = *reinterpret_cast<const uint4*>(base + from[j0 + u] * row_bytes);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (j0 + u < n) *reinterpret_cast<uint4*>(base + to[j0 + u] * row_bytes) = v[u];
        }
    } else {
        using B = Fp4Block<D>;
        constexpr int W = D / 16 / 4;  // words of a piece
        const int h = item / 18, piece = item % 18;
        if (h >= a.Hkv) return;
        // byte of the piece of token row `at` in the pool
        auto block = [&](int64_t at) {
            const int64_t page = at >> shift;
            const int in = (int)(at & in_page);
            return a.kv.k + (((page * a.Hkv + h) << (shift - 4)) + (in >> 4)) * B::kBytes;
        };
        auto where = [&](int t) {
            if (piece < 8) return t * (D / 2) + piece * (D / 16);
            if (piece < 16) return B::v_byte(t, (piece - 8) * (D / 8));
            return piece == 16 ? B::k_scale(t, 0) : B::v_scale(t, 0);
        };
        for (int j0 = skip; j0 < n; j0 += kAhead) {
            uint32_t v[kAhead][W];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j0 + u >= n) continue;
                const uint8_t* p = block(from[j0 + u]) + where((int)(from[j0 + u] & 15));
                if (piece < 17) {
#pragma unroll
                    for (int w = 0; w < W; ++w) v[u][w] = reinterpret_cast<const uint32_t*>(p)[w];
                } else {  // scales of a token's values lie 16 tokens apart
#pragma unroll
                    for (int w = 0; w < W; ++w)
                        v[u][w] = *reinterpret_cast<const uint16_t*>(p + 64 * w) |
                                  (uint32_t)*reinterpret_cast<const uint16_t*>(p + 64 * w + 32) << 16;
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j0 + u >= n) continue;
                uint8_t* p = block(to[j0 + u]) + where((int)(to[j0 + u] & 15));
                if (piece < 17) {
#pragma unroll
                    for (int w = 0; w < W; ++w) reinterpret_cast<uint32_t*>(p)[w] = v[u][w];
                } else {
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        *reinterpret_cast<uint16_t*>(p + 64 * w) = (uint16_t)v[u][w];
                        *reinterpret_cast<uint16_t*>(p + 64 * w + 32) = (uint16_t)(v[u][w] >> 16);
                    }
                }
            }
        }
    }
}

}  // namespace

int launch_commit_paged(const int32_t* path, int path_stride, const int32_t* n_path, const TreeRows& tree, int32_t* kv_len_out,
                        const PagedView& kv, bool fp4, const moska_shape* s, cudaStream_t st)
{
    if (tree.n_requests == 0) return MOSKA_OK;
    const long long items = fp4 ? 18LL * s->Hkv : 2LL * s->Hkv * (s->D / 8);
    const long long parts = (items + kThreads - 1) / kThreads, grid = parts * tree.n_requests;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "commit grid too large");
    const CommitArgs a{kv, tree, path, n_path, kv_len_out, path_stride, s->Hkv, (int)parts};
    const auto kernel = s->D == 128 ? (fp4 ? commit_kernel<128, true> : commit_kernel<128, false>)
                                    : (fp4 ? commit_kernel<64, true> : commit_kernel<64, false>);
    kernel<<<(unsigned)grid, kThreads, 0, st>>>(a);
    MOSKA_LAUNCH_CHECK("commit_kernel");
    return MOSKA_OK;
}

}  // namespace moska
