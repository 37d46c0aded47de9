// Attention over a paged private store in bf16: the streaming blocks of stream_attn.cuh with the
// tile's page looked up one tile ahead of its copies.  A 16-token tile never crosses a page (a page is
// a power of two of at least 16 tokens), so one lookup serves it.  HBM-bound like the contiguous form;
// token rows of the KV heads of a page are neighbours, as in the ragged store.
#include <cuda_bf16.h>

#include "paged.cuh"
#include "stream_attn.cuh"

namespace moska {
namespace {
using namespace stream;

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
};

// One CTA per (request, KV head, split).  kMulti: several query tokens per request.
template <int D, int NT, bool kMulti>
__global__ void __launch_bounds__(kThreads, D == 128 ? 2 : 3) paged_bf16_kernel(const PagedArgs a)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ TileRows<NT> rows;
    __shared__ int row_last[NT * 8];
    const int G = a.Hq / a.Hkv;
    const int h = blockIdx.x % a.Hkv;
    const int sp = (blockIdx.x / a.Hkv) % a.n_splits;
    const int r = blockIdx.x / (a.Hkv * a.n_splits);
    dependents_may_launch();
    const int len = paged_len(a.kv, r);
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

// Final rows from the partial rows of n splits (up to 64): a warp per row, D / 32 dimensions a lane; lane
// i holds the weight of splits i and i + 32.
template <int D>
__global__ void __launch_bounds__(128)
paged_merge_kernel(const float* __restrict__ o_part, const float* __restrict__ lse_part, uint16_t* __restrict__ out,
                   float* __restrict__ lse_out, int rows, int n)
{
    constexpr int W = D / 32;
    const int lane = threadIdx.x & 31;
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5);
    wait_for_results();
    if (row >= rows) return;
    const float* lse = lse_part + (int64_t)row * n;
    const float* o = o_part + (int64_t)row * n * D + W * lane;
    float l[2] = {lane < n ? lse[lane] : -INFINITY, lane + 32 < n ? lse[lane + 32] : -INFINITY};
    float M = max_or_nan(l[0], l[1]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = max_or_nan(M, __shfl_xor_sync(0xffffffffu, M, off));
    float acc[W], total = 0.f;
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] = 0.f;
    if (M != -INFINITY) {
        const float w[2] = {__expf(l[0] - M), __expf(l[1] - M)};
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float wi = __shfl_sync(0xffffffffu, i < 32 ? w[0] : w[1], i & 31);
            total += wi;
#pragma unroll
            for (int e = 0; e < W; ++e) acc[e] = fmaf(wi, o[(int64_t)i * D + e], acc[e]);
        }
        const float inv = 1.f / total;
#pragma unroll
        for (int e = 0; e < W; ++e) acc[e] *= inv;
    }
#pragma unroll
    for (int e = 0; e < W; e += 2)
        *reinterpret_cast<__nv_bfloat162*>(out + (int64_t)row * D + W * lane + e) = __floats2bfloat162_rn(acc[e], acc[e + 1]);
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
    config.gridDim = dim3((unsigned)((rows + 3) / 4));
    config.blockDim = dim3(128);
    config.stream = st;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    MOSKA_CUDA_TRY(cudaLaunchKernelEx(&config, s->D == 128 ? paged_merge_kernel<128> : paged_merge_kernel<64>, o_part,
                                      lse_part, out, lse_out, (int)rows, (int)s->n_unique_splits));
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
    const PagedArgs a{q, kv, o_part, lse_part, out, lse_out, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0, n_slots, q_len};
    auto go = [&](auto kernel, int smem) {
        MOSKA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        kernel<<<(unsigned)grid, kThreads, smem, st>>>(a);
        MOSKA_LAUNCH_CHECK("paged_bf16_kernel");
        return (int)MOSKA_OK;
    };
    constexpr int kRing = kWarps * kStagedWarpBytes;
    if (s->D == 64) return go(paged_bf16_kernel<64, 1, false>, (int)sizeof(CombineSmem<64, 1>));
    if (q_len == 1) return go(paged_bf16_kernel<128, 1, false>, kRing);
    if (q_len * (s->Hq / s->Hkv) <= 8) return go(paged_bf16_kernel<128, 1, true>, kRing);
    return go(paged_bf16_kernel<128, 2, true>, kRing);
}

}  // namespace moska
