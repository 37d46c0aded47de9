// Writing and reading back rows of a paged private store (moska_kv_append_paged,
// moska_kv_gather_paged).
//
// Append: y = rotate(x) for the queries and keys of a row, values as they are; a row's query heads go
// to q_out, its key and value heads into the page that holds its context token, in bf16 or as E2M1
// codes with one f16 scale per 32 dimensions.  Every element is read and written once: the bound is
// HBM, for a decode step (one row a request) the latency of the chain row -> request -> length -> page.
#include <cuda_bf16.h>

#include "paged.cuh"

namespace moska {
namespace {

constexpr int kAppendThreads = 256;

struct RowPlace {
    int token;      // context token, negative: padding
    int page;       // page of the token, -1: none (reported)
};

// Which request row i belongs to and which context token it is.  Every lane of a warp calls this
// with the same row.  Ragged rows: a 32-way search over row_start (two steps up to 1024 requests).
__device__ __forceinline__ RowPlace place_row(const PagedView& kv, int row, int q_len, const int32_t* row_start,
                                              int n_requests)
{
    const int lane = threadIdx.x & 31;
    int r, behind;  // request, and how many of its rows come at or after this one
    if (row_start == nullptr) {
        r = row / q_len;
        behind = q_len - (row - r * q_len);
    } else {
        // largest r with row_start[r] <= row
        int lo = 0, n = n_requests + 1;  // the answer is in [lo, lo + n)
        if (__ldg(row_start) > row) return {-1, -1};
        while (n > 1) {
            const int step = (n + 31) / 32;
            const int at = lo + lane * step;
            const bool le = at < lo + n && __ldg(row_start + at) <= row;
            const int last = __popc(__ballot_sync(0xffffffffu, le)) - 1;  // ascending: a prefix of the lanes
            const int next = lo + max(last, 0) * step;
            n = min(step, lo + n - next);
            lo = next;
        }
        if (lo >= n_requests) return {-1, -1};  // behind the last request: padding
        r = lo;
        behind = __ldg(row_start + r + 1) - row;
        if (behind <= 0) {  // row_start is not ascending
            if (lane == 0) atomicMin(kv.status, MOSKA_ERR_INVALID_ARG);
            return {-1, -1};
        }
    }
    const int len = __ldg(kv.kv_len + r);
    if (len < 0 || len > ((long long)kv.max_pages << kv.page_shift)) {
        if (lane == 0) atomicMin(kv.status, MOSKA_ERR_INVALID_ARG);
        return {-1, -1};
    }
    RowPlace out;
    out.token = len - behind;
    out.page = -1;
    if (out.token >= 0) {
        const int page = __ldg(kv.page_table + (int64_t)r * kv.max_pages + (out.token >> kv.page_shift));
        if (static_cast<unsigned>(page) < static_cast<unsigned>(kv.n_pages)) out.page = page;
        else if (lane == 0) atomicMin(kv.status, MOSKA_ERR_INVALID_ARG);
    }
    return out;
}

__device__ __forceinline__ void unpack8(const uint4& r, float (&x)[8])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// E2M1 code of x for scale s: the nearest grid value, ties to the even code.  Against products of the
// scale, not of a quotient: k/8 times an f16 is exact in fp32, so every tie and every neighbour of one
// falls on its right side.
__device__ __forceinline__ uint32_t e2m1_code(float x, float s)
{
    const float a = fabsf(x);
    uint32_t c = 0;
    c += a > 0.25f * s;
    c += a >= 0.75f * s;
    c += a > 1.25f * s;
    c += a >= 1.75f * s;
    c += a > 2.5f * s;
    c += a >= 3.5f * s;
    c += a > 5.f * s;
    return c | ((__float_as_uint(x) >> 28) & 8u);
}

template <int D, bool kFp4>
__global__ void __launch_bounds__(kAppendThreads)
append_kernel(const uint16_t* __restrict__ q, int64_t q_stride, const uint16_t* __restrict__ k, int64_t k_stride,
              const uint16_t* __restrict__ v, int64_t v_stride, const int32_t* __restrict__ positions,
              const float* __restrict__ cos_sin, int n_positions, int rot_dim, int interleaved,
              const int32_t* __restrict__ row_start, int n_requests, uint16_t* __restrict__ q_out, PagedView kv,
              int Hq, int Hkv, int q_len)
{
    constexpr int T = D / 8;                    // threads of one head: eight dimensions each
    constexpr int kHeads = kAppendThreads / T;  // heads in flight
    const int row = blockIdx.x;
    const int t = threadIdx.x % T, d0 = 8 * t;
    const RowPlace at = place_row(kv, row, q_len, row_start, n_requests);
    if (at.token < 0) return;  // padding

    // this thread's part of the rotation: y = x c + sign (partner s)
    const bool rotated = d0 < rot_dim;
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
    const int half = rot_dim / 2;
    if (rot_dim > 0) {
        const int pos = __ldg(positions + row);
        if (static_cast<unsigned>(pos) >= static_cast<unsigned>(n_positions)) {
            if (threadIdx.x == 0) atomicMin(kv.status, MOSKA_ERR_INVALID_ARG);
            return;
        }
        if (rotated) {
            const float* cs = cos_sin + (int64_t)pos * rot_dim;
            if (interleaved) {
                const float4 a = __ldg(reinterpret_cast<const float4*>(cs + d0 / 2));
                const float4 b = __ldg(reinterpret_cast<const float4*>(cs + half + d0 / 2));
                c[0] = c[1] = a.x; c[2] = c[3] = a.y; c[4] = c[5] = a.z; c[6] = c[7] = a.w;
                s[0] = s[1] = b.x; s[2] = s[3] = b.y; s[4] = s[5] = b.z; s[6] = s[7] = b.w;
            } else {
                const float* p = cs + (d0 < half ? d0 : d0 - half);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float4 a = __ldg(reinterpret_cast<const float4*>(p + 4 * i));
                    const float4 b = __ldg(reinterpret_cast<const float4*>(p + half + 4 * i));
                    c[4 * i] = a.x; c[4 * i + 1] = a.y; c[4 * i + 2] = a.z; c[4 * i + 3] = a.w;
                    s[4 * i] = b.x; s[4 * i + 1] = b.y; s[4 * i + 2] = b.z; s[4 * i + 3] = b.w;
                }
            }
        }
    }
    const bool first = d0 < half;
    // eight rotated elements from `src` (this head's row)
    auto load_rotated = [&](const uint16_t* src, float (&y)[8]) {
        float x[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(src + d0)), x);
        if (!rotated) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i];
        } else if (interleaved) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                y[i] = __fsub_rn(__fmul_rn(x[i], c[i]), __fmul_rn(x[i + 1], s[i]));
                y[i + 1] = __fadd_rn(__fmul_rn(x[i + 1], c[i]), __fmul_rn(x[i], s[i]));
            }
        } else {
            float z[8];  // the partner half's eight elements
            unpack8(__ldg(reinterpret_cast<const uint4*>(src + (first ? d0 + half : d0 - half))), z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = __fmul_rn(x[i], c[i]), b = __fmul_rn(z[i], s[i]);
                y[i] = first ? __fsub_rn(a, b) : __fadd_rn(a, b);
            }
        }
    };

    const int slot = at.token & ((1 << kv.page_shift) - 1);  // row inside the page
    const int n_q = q != nullptr ? Hq : 0, n_all = n_q + 2 * Hkv;
    for (int i = blockIdx.y * kHeads + threadIdx.x / T; i < n_all; i += gridDim.y * kHeads) {
        if (i < n_q) {
            float y[8];
            load_rotated(q + row * q_stride + (int64_t)i * D, y);
            *reinterpret_cast<uint4*>(q_out + ((int64_t)row * Hq + i) * D + d0) = pack8(y);
            continue;
        }
        const bool is_v = i >= n_q + Hkv;
        const int h = i - n_q - (is_v ? Hkv : 0);
        float y[8];
        if (is_v) unpack8(__ldg(reinterpret_cast<const uint4*>(v + row * v_stride + (int64_t)h * D + d0)), y);
        else load_rotated(k + row * k_stride + (int64_t)h * D, y);
        if constexpr (!kFp4) {
            if (at.page < 0) continue;
            const int64_t to = ((((int64_t)at.page << kv.page_shift) + slot) * Hkv + h) * D + d0;
            *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(is_v ? kv.v : kv.k) + to) = pack8(y);
        } else {
            using B = Fp4Block<D>;
            // largest magnitude of the 32 dimensions (four neighbouring threads); a NaN or an infinity
            // anywhere in them makes the sum of x - x NaN
            float top = 0.f, odd = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                top = fmaxf(top, fabsf(y[e]));
                odd += y[e] - y[e];
            }
            const unsigned group = 0xfu << (threadIdx.x & 28);
#pragma unroll
            for (int off = 1; off < 4; off <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(group, top, off));
                odd += __shfl_xor_sync(group, odd, off);
            }
            const __half sh = __float2half_rn(fminf(__fdiv_rn(top, 6.f), kFp4MaxScale) + odd);
            const float sf = __half2float(sh);
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= e2m1_code(y[e], sf) << (4 * e);
            if (at.page < 0) continue;
            const int tok = slot & (kBlockTokens - 1);
            uint8_t* blk = kv.k + ((((int64_t)at.page * Hkv + h) << (kv.page_shift - 4)) + (slot >> 4)) * B::kBytes;
            *reinterpret_cast<uint32_t*>(blk + (is_v ? B::v_byte(tok, d0) : B::k_byte(tok, d0))) = w;
            if ((t & 3) == 0)
                *reinterpret_cast<__half*>(blk + (is_v ? B::v_scale(tok, t >> 2) : B::k_scale(tok, t >> 2))) = sh;
        }
    }
}

template <int D, bool kFp4>
__global__ void __launch_bounds__(kAppendThreads)
gather_kernel(const int32_t* __restrict__ row_start, int n_requests, uint16_t* __restrict__ k_out,
              uint16_t* __restrict__ v_out, PagedView kv, int Hkv, int q_len)
{
    constexpr int T = D / 8, kHeads = kAppendThreads / T;
    const int row = blockIdx.x;
    const int t = threadIdx.x % T, d0 = 8 * t;
    const RowPlace at = place_row(kv, row, q_len, row_start, n_requests);
    if (at.token < 0) return;
    if (at.page < 0) return;  // an index outside the pool has been reported
    const int page = at.page;
    const int slot = at.token & ((1 << kv.page_shift) - 1);
    for (int i = blockIdx.y * kHeads + threadIdx.x / T; i < 2 * Hkv; i += gridDim.y * kHeads) {
        const bool is_v = i >= Hkv;
        const int h = is_v ? i - Hkv : i;
        uint4 y;
        if constexpr (!kFp4) {
            const int64_t from = ((((int64_t)page << kv.page_shift) + slot) * Hkv + h) * D + d0;
            y = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(is_v ? kv.v : kv.k) + from));
        } else {
            using B = Fp4Block<D>;
            const int tok = slot & (kBlockTokens - 1);
            const uint8_t* blk = kv.k + ((((int64_t)page * Hkv + h) << (kv.page_shift - 4)) + (slot >> 4)) * B::kBytes;
            const uint32_t w =
                __ldg(reinterpret_cast<const uint32_t*>(blk + (is_v ? B::v_byte(tok, d0) : B::k_byte(tok, d0))));
            const float s =
                __half2float(*reinterpret_cast<const __half*>(blk + (is_v ? B::v_scale(tok, t >> 2) : B::k_scale(tok, t >> 2))));
            uint32_t f[4];
            e2m1x8_to_f16x2(w, f);
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f[e]));
                x[2 * e] = p.x * s;
                x[2 * e + 1] = p.y * s;
            }
            y = pack8(x);
        }
        *reinterpret_cast<uint4*>((is_v ? v_out : k_out) + ((int64_t)row * Hkv + h) * D + d0) = y;
    }
}

// One CTA a row as long as there are rows for every SM; few rows: their heads over several CTAs.
dim3 row_grid(int rows, int heads, int heads_per_pass)
{
    const int passes = (heads + heads_per_pass - 1) / heads_per_pass;
    int y = (148 * 4 + rows - 1) / rows;
    if (y > passes) y = passes;
    return dim3((unsigned)rows, (unsigned)(y < 1 ? 1 : y));
}

}  // namespace

int launch_append_paged(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                        int64_t v_stride, const int32_t* positions, const float* cos_sin, int n_positions,
                        int rot_dim, int interleaved, const int32_t* row_start, int n_requests, uint16_t* q_out,
                        const PagedView& kv, bool fp4, const moska_shape* s, cudaStream_t st)
{
    if (s->B == 0) return MOSKA_OK;
    const int q_len = s->q_len > 1 ? s->q_len : 1;
    const dim3 grid = row_grid(s->B, (q != nullptr ? s->Hq : 0) + 2 * s->Hkv, kAppendThreads / (s->D / 8));
    auto go = [&](auto kernel) {
        kernel<<<grid, kAppendThreads, 0, st>>>(q, q_stride, k, k_stride, v, v_stride, positions, cos_sin, n_positions,
                                                rot_dim, interleaved, row_start, n_requests, q_out, kv, s->Hq, s->Hkv,
                                                q_len);
    };
    if (s->D == 128) fp4 ? go(append_kernel<128, true>) : go(append_kernel<128, false>);
    else fp4 ? go(append_kernel<64, true>) : go(append_kernel<64, false>);
    MOSKA_LAUNCH_CHECK("append_kernel");
    return MOSKA_OK;
}

int launch_gather_paged(const int32_t* row_start, int n_requests, uint16_t* k_out, uint16_t* v_out,
                        const PagedView& kv, bool fp4, const moska_shape* s, cudaStream_t st)
{
    if (s->B == 0) return MOSKA_OK;
    const int q_len = s->q_len > 1 ? s->q_len : 1;
    const dim3 grid = row_grid(s->B, 2 * s->Hkv, kAppendThreads / (s->D / 8));
    auto go = [&](auto kernel) {
        kernel<<<grid, kAppendThreads, 0, st>>>(row_start, n_requests, k_out, v_out, kv, s->Hkv, q_len);
    };
    if (s->D == 128) fp4 ? go(gather_kernel<128, true>) : go(gather_kernel<128, false>);
    else fp4 ? go(gather_kernel<64, true>) : go(gather_kernel<64, false>);
    MOSKA_LAUNCH_CHECK("gather_kernel");
    return MOSKA_OK;
}

}  // namespace moska
