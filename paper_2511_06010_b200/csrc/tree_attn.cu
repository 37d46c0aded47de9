// Attention of the nodes of drafted trees over the paged contexts that they end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>

#include "tree.cuh"

namespace moska {
namespace {

constexpr int kThreads = 128;

struct TreeArgs {
    const uint16_t* q;
    PagedView kv;
    TreeRows tree;
    float* o_part;  // partial slots (nullptr: `out` gets the final rows)
    float* lse_part;
    uint16_t* out;
    float* lse_out;
    float scale;
    int Hq, Hkv, n_splits, slot0, n_slots;
};

template <int D>
__device__ __forceinline__ float e2m1_value(uint32_t code)
{
    const float mag[8] = {0.f, .5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
    return (code & 8) ? -mag[code & 7] : mag[code & 7];
}

// Element d of the key (or value) of token t
template <int D, bool F4>
__device__ __forceinline__ float element(const PagedView& kv, const int32_t* pages, int Hkv, int h, int t, int d, bool value)
{
    const int64_t page = paged_page(kv, pages, t >> kv.page_shift);
    const int in = t & ((1 << kv.page_shift) - 1);
    if constexpr (F4) {
        using B = Fp4Block<D>;
        const uint8_t* b = kv.k + (((page * Hkv + h) << (kv.page_shift - 4)) + (in >> 4)) * B::kBytes;
        const int u = in & 15;
        const int at = (value ? B::v_byte(u, d & ~7) : B::k_byte(u, d & ~7)) + (d & 7) / 2;
        const int sc = value ? B::v_scale(u, d / 32) : B::k_scale(u, d / 32);
        return e2m1_value<D>((b[at] >> (4 * (d & 1))) & 15) * __half2float(*reinterpret_cast<const __half*>(b + sc));
    } else {
        const uint16_t* x = reinterpret_cast<const uint16_t*>(value ? kv.v : kv.k);
        return __uint_as_float((uint32_t)x[(((page << kv.page_shift) + in) * Hkv + h) * D + d] << 16);
    }
}

// One CTA per (node, query head, split): scores of 128 tokens at a time, a token a thread; then the values, a
// dimension a thread.
template <int D, bool F4>
__global__ void __launch_bounds__(kThreads) tree_attn_kernel(const TreeArgs a)
{
    __shared__ float q[D], p[kThreads], red[4];
    __shared__ TreeSmem ts;
    const int hq = blockIdx.x % a.Hq, sp = (blockIdx.x / a.Hq) % a.n_splits;
    const int node = (blockIdx.x / (a.Hq * a.n_splits)) % a.tree.max_nodes;
    const int r = blockIdx.x / (a.Hq * a.n_splits) / a.tree.max_nodes;
    const int h = hq / (a.Hq / a.Hkv), tid = threadIdx.x;
    const int2 rows = tree_rows(a.tree, r, a.kv.status);
    if (node >= rows.y) return;
    const int len = paged_len(a.kv, r), committed = len - rows.y;
    const int parent = tid < rows.y ? tree_parent(a.tree, rows.x, tid, a.kv.status) : -1;
    if (tid < 64) tree_ancestors(ts, tid, parent, [] { asm volatile("bar.sync 1, 64;" ::: "memory"); });
    const int64_t row = (int64_t)(rows.x + node) * a.Hq + hq;
    if (tid < D) q[tid] = __uint_as_float((uint32_t)a.q[row * D + tid] << 16);
    __syncthreads();
    const unsigned long long sees = committed + node < 0 ? 0 : ts.bits[node];
    const int32_t* pages = a.kv.page_table + (int64_t)r * a.kv.max_pages;
    int per = (len + a.n_splits - 1) / a.n_splits;
    per = (per + kThreads - 1) / kThreads * kThreads;
    const int t0 = (int)min((long long)len, (long long)sp * per), t1 = min(len, t0 + per);
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int t = t0; t < t1; t += kThreads) {
        const int tok = t + tid;
        bool seen = tok < t1 && committed + node >= 0;
        if (seen && tok >= committed) seen = (sees >> (tok - committed)) & 1;
        float s = -INFINITY;
        if (seen) {
            s = 0.f;
            for (int d = 0; d < D; ++d) s = fmaf(q[d], element<D, F4>(a.kv, pages, a.Hkv, h, tok, d, false), s);
            s *= a.scale;
        }
        float mx = s;
        for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        if (tid % 32 == 0) red[tid / 32] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.f : mn;
        const float alpha = m == -INFINITY ? 0.f : expf(m - base);
        p[tid] = seen ? expf(s - base) : -1.f;  // -1: not seen
        __syncthreads();
        l *= alpha;
        o *= alpha;
        for (int i = 0; i < min(kThreads, t1 - t); ++i) {
            if (p[i] == -1.f) continue;
            l += p[i];
            if (tid < D) o = fmaf(p[i], element<D, F4>(a.kv, pages, a.Hkv, h, t + i, tid, true), o);
        }
        m = mn;
        __syncthreads();
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, lse = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) + logf(l);
    const int64_t slot = row * a.n_slots + a.slot0 + sp;
    if (tid < D) {
        const float x = l == 0.f ? 0.f : o * inv;
        if (a.out != nullptr) reinterpret_cast<__nv_bfloat16*>(a.out)[row * D + tid] = __float2bfloat16_rn(x);
        else a.o_part[slot * D + tid] = x;
    }
    if (tid == 0) {
        if (a.out == nullptr) a.lse_part[slot] = lse;
        else if (a.lse_out != nullptr) a.lse_out[row] = lse;
    }
}

}  // namespace

int default_tree_splits(bool, int n_requests, int nodes, int G, int Hkv, int, int max_len)
{
    const long long ctas = (long long)n_requests * nodes * G * Hkv;
    long long s = 1184 / ctas;
    if (s > (max_len + 255) / 256) s = (max_len + 255) / 256;
    return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

int launch_tree_attn(const uint16_t* q, const PagedView& kv, bool fp4, const TreeRows& tree, float* o_part, float* lse_part,
                     int slot0, int n_slots, uint16_t* out, float* lse_out, float scale, const moska_shape* s,
                     cudaStream_t st)
{
    const long long grid = (long long)tree.n_requests * tree.max_nodes * s->Hq * s->n_unique_splits;
    if (grid == 0 || tree.n_rows == 0) return MOSKA_OK;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "tree attention grid too large");
    const TreeArgs a{q, kv, tree, o_part, lse_part, out, lse_out, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0, n_slots};
    const auto kernel = s->D == 128 ? (fp4 ? tree_attn_kernel<128, true> : tree_attn_kernel<128, false>)
                                    : (fp4 ? tree_attn_kernel<64, true> : tree_attn_kernel<64, false>);
    kernel<<<(unsigned)grid, kThreads, 0, st>>>(a);
    MOSKA_LAUNCH_CHECK("tree_attn_kernel");
    return MOSKA_OK;
}

}  // namespace moska
