// Attention over a paged private store in bf16: the streaming blocks of stream_attn.cuh with the
// tile's page looked up one tile ahead of its copies.  A 16-token tile never crosses a page (a page is
// a power of two of at least 16 tokens), so one lookup serves it.  HBM-bound like the contiguous form;
// token rows of the KV heads of a page are neighbours, as in the ragged store.
#include <cuda_bf16.h>

#include <type_traits>

#include "paged.cuh"
#include "stream_attn.cuh"

namespace moska {
namespace {
using namespace stream;
static_assert(kThreads == kMaxOrdered, "a request a thread");

struct PagedTokens {
    static constexpr bool kPaged = true;
    PagedView kv;
    const int32_t* row;  // page-table row
    bool final_rows;     // results are final bf16 rows (and lse may be nullptr), not partial slots
    __device__ __forceinline__ int64_t base(int t0) const
    {
        const int i = t0 >> kv.page_shift;
        return ((int64_t)(paged_page(kv, row, i) - i)) << kv.page_shift;
    }
    __device__ __forceinline__ void store(float* o_row, float* lse_row, int d, float o, float lse) const
    {
        if (final_rows) reinterpret_cast<uint16_t*>(o_row)[d] = __bfloat16_as_ushort(__float2bfloat16_rn(o));
        else o_row[d] = o;
        if (d == 0 && lse_row != nullptr) *lse_row = lse;
    }
};

struct PagedArgs {
    const uint16_t* q;
    PagedView kv;
    float* o_part;  // partial slots (nullptr: `out` gets the final rows)
    float* lse_part;
    uint16_t* out;
    float* lse_out;
    float scale;
    int Hq, Hkv, n_splits, slot0, n_slots, q_len;
    int n_requests;
};

// One CTA per (request, KV head, split).  kMulti: several query tokens per request.
// kOrdered: requests longest context first.
template <int D, int NT, bool kMulti, bool kOrdered>
__global__ void __launch_bounds__(kThreads, D == 128 ? 2 : 3) paged_bf16_kernel(const PagedArgs a)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ TileRows<NT> rows;
    __shared__ int row_last[NT * 8];
    __shared__ typename std::conditional<kOrdered, OrderSmem, int>::type order;
    const int G = a.Hq / a.Hkv;
    const int h = blockIdx.x % a.Hkv;
    const int sp = (blockIdx.x / a.Hkv) % a.n_splits;
    int r = blockIdx.x / (a.Hkv * a.n_splits);
    dependents_may_launch();
    int len;
    if constexpr (kOrdered) r = request_at(a.kv, a.n_requests, r, order, len);
    else len = paged_len(a.kv, r);
    if (threadIdx.x < NT * 8) {
        const int j = threadIdx.x;
        const bool live = j < a.q_len * G;
        const int64_t row = ((int64_t)r * a.q_len + j / G) * a.Hq + h * G + j % G;
        const int64_t slot = row * a.n_slots + a.slot0 + sp;
        const bool final_rows = a.out != nullptr;
        rows.q[j] = live ? a.q + row * D : nullptr;
        rows.o[j] = !live ? nullptr : final_rows ? reinterpret_cast<float*>(a.out + row * D) : a.o_part + slot * D;
        rows.lse[j] = !live ? nullptr : !final_rows ? a.lse_part + slot : a.lse_out != nullptr ? a.lse_out + row : nullptr;
        row_last[j] = live ? len - 1 - (a.q_len - 1 - j / G) : 0x7fffffff;
    }
    __syncthreads();
    // equal parts rounded up to a pass of the CTA's warps
    constexpr int kPass = kWarps * kTileTokens;
    int per = (len + a.n_splits - 1) / a.n_splits;
    per = (per + kPass - 1) / kPass * kPass;
    const int t0 = (int)min((long long)len, (long long)sp * per), t1 = min(len, t0 + per);
    const int64_t stride = (int64_t)a.Hkv * D;
    const uint16_t* kb = reinterpret_cast<const uint16_t*>(a.kv.k) + (int64_t)h * D;
    const uint16_t* vb = reinterpret_cast<const uint16_t*>(a.kv.v) + (int64_t)h * D;
    const PagedTokens tokens{a.kv, a.kv.page_table + (int64_t)r * a.kv.max_pages, a.out != nullptr};
    if constexpr (D == 128)
        attend_stream_staged<NT, kMulti>(rows, kb, vb, stride, t0, t1, a.scale, ring, row_last, tokens);
    else
        attend_stream<D, NT>(rows, kb, vb, stride, t0, t1, a.scale, *reinterpret_cast<CombineSmem<D, NT>*>(ring), tokens);
}

// Final rows from the partial rows of n splits: R warps a row, each with every R-th split and eight of its
// loads in flight (the rows come from L2: latency counts), joined through shared memory.  The partial rows
// are written while this kernel may already run: no __restrict__, which would let their loads pass the wait.
constexpr int kMergeWarps = 4;
template <int D, int R>
__global__ void __launch_bounds__(kMergeWarps * 32)
paged_merge_kernel(const float* o_part, const float* lse_part, uint16_t* out, float* lse_out, long long rows, int n)
{
    constexpr int W = D / 32;  // dimensions a lane
    using Vec = typename std::conditional<W == 4, float4, float2>::type;
    __shared__ __align__(16) float part[kMergeWarps][D];
    __shared__ float sums[kMergeWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * (kMergeWarps / R) + warp / R;
    wait_for_results();
    if (row >= rows) return;  // (R = 1: no barrier follows)
    const float* lse = lse_part + row * n;
    const float* o = o_part + row * n * D + W * lane;
    float M = -INFINITY;
    for (int i = lane; i < n; i += 32) M = max_or_nan(M, lse[i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = max_or_nan(M, __shfl_xor_sync(0xffffffffu, M, off));
    const float base = M == -INFINITY ? 0.f : M;  // (all splits empty: every weight is 0)
    __align__(16) float acc[W];
    float total = 0.f;
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] = 0.f;
    for (int i0 = warp % R; i0 < n; i0 += 8 * R) {
        Vec v[8];
        float w[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u * R;
            if (i >= n) break;
            w[u] = lse[i];
            v[u] = *reinterpret_cast<const Vec*>(o + (int64_t)i * D);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i0 + u * R >= n) break;
            const float wi = __expf(w[u] - base);
            total += wi;
            const float* x = reinterpret_cast<const float*>(&v[u]);
#pragma unroll
            for (int e = 0; e < W; ++e) acc[e] = fmaf(wi, x[e], acc[e]);
        }
    }
    if constexpr (R > 1) {
        static_assert(R == kMergeWarps, "a CTA is one row");
        *reinterpret_cast<Vec*>(&part[warp][W * lane]) = *reinterpret_cast<const Vec*>(acc);
        if (lane == 0) sums[warp] = total;
        __syncthreads();
        if (warp > 0) return;
        total = 0.f;
#pragma unroll
        for (int e = 0; e < W; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < R; ++w) {
            total += sums[w];
#pragma unroll
            for (int e = 0; e < W; ++e) acc[e] += part[w][W * lane + e];
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < W; e += 2)
        *reinterpret_cast<__nv_bfloat162*>(out + row * D + W * lane + e) = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
    if (lane == 0 && lse_out != nullptr) lse_out[row] = M == -INFINITY ? -INFINITY : M + logf(total);
}

}  // namespace

int launch_paged_merge(const float* o_part, const float* lse_part, uint16_t* out, float* lse_out, const moska_shape* s,
                       cudaStream_t st)
{
    const long long rows = (long long)s->B * s->Hq;
    if (rows == 0) return MOSKA_OK;
    if (rows > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "too many rows");
    cudaLaunchConfig_t config{};
    // a row of many splits is a chain of loads: four warps share it, as long as the rows do not fill the GPU
    // (32 rows of 16 splits: 2.0 against 4.0 us; 6144 rows of 2 splits: 8 against 3)
    const int n = s->n_unique_splits;
    const bool wide = n > 4 && rows <= 4096;
    config.gridDim = dim3((unsigned)(wide ? rows : (rows + kMergeWarps - 1) / kMergeWarps));
    config.blockDim = dim3(kMergeWarps * 32);
    config.stream = st;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    const auto kernel = s->D == 128 ? (wide ? paged_merge_kernel<128, kMergeWarps> : paged_merge_kernel<128, 1>)
                                    : (wide ? paged_merge_kernel<64, kMergeWarps> : paged_merge_kernel<64, 1>);
    MOSKA_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, o_part, lse_part, out, lse_out, rows, n));
    return MOSKA_OK;
}

// `out` == nullptr: partial slots slot0 .. of n_slots; else the final rows (one split).
int launch_paged_bf16(const uint16_t* q, const PagedView& kv, float* o_part, float* lse_part, int slot0, int n_slots,
                      uint16_t* out, float* lse_out, float scale, const moska_shape* s, cudaStream_t st)
{
    const int q_len = s->q_len > 1 ? s->q_len : 1;
    const long long grid = (long long)(s->B / q_len) * s->Hkv * s->n_unique_splits;
    if (grid == 0) return MOSKA_OK;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "paged attention grid too large");
    const PagedArgs a{q, kv, o_part, lse_part, out, lse_out, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0, n_slots, q_len,
                      s->B / q_len};
    auto go = [&](auto kernel, int smem) {
        MOSKA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        kernel<<<(unsigned)grid, kThreads, smem, st>>>(a);
        MOSKA_LAUNCH_CHECK("paged_bf16_kernel");
        return (int)MOSKA_OK;
    };
    constexpr int kRing = kWarps * kStagedWarpBytes;
    auto form = [&](auto ordered) {
        constexpr bool O = decltype(ordered)::value;
        if (s->D == 64) return go(paged_bf16_kernel<64, 1, false, O>, (int)sizeof(CombineSmem<64, 1>));
        if (q_len == 1) return go(paged_bf16_kernel<128, 1, false, O>, kRing);
        if (q_len * (s->Hq / s->Hkv) <= 8) return go(paged_bf16_kernel<128, 1, true, O>, kRing);
        return go(paged_bf16_kernel<128, 2, true, O>, kRing);
    };
    return longest_first(a.n_requests, grid) ? form(std::true_type{}) : form(std::false_type{});
}

}  // namespace moska
