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

// x / 6, correctly rounded for every x whose quotient is normal: a quotient from the rounded reciprocal and
// one correction with its exact remainder (Markstein, "Computation of elementary functions on the IBM
// RISC System/6000 processor", 1990).  Smaller quotients are below what an f16 scale can tell from 0.
__device__ __forceinline__ float sixth(float x)
{
    const float y = 1.f / 6.f;  // folded at compile time
    const float q = __fmul_rn(x, y);
    return fmaf(fmaf(-6.f, q, x), y, q);
}

// The E2M1 codes of y[0..7] for scale s, y[0] in the lowest four bits.  Products with 1 / s a little
// too small and a little too large (2^-20; their own error is below 2^-22) enclose the quotient: where
// the conversion gives both the same code that is the quotient's, elsewhere (near a tie, a few in a
// million) the codes are compared out.
__device__ __forceinline__ uint32_t e2m1x8(const float (&y)[8], float s)
{
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));  // within 2^-23; s is 0, NaN or at least 2^-24
    inv = s > 0.f ? inv : 0.f;
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float m = i == 0 ? inv * (1.f - 0x1p-20f) : inv * (1.f + 0x1p-20f);
        asm("{\n"
            ".reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3};\n"
            "}\n"
            : "=r"(w[i])
            : "f"(y[0] * m), "f"(y[1] * m), "f"(y[2] * m), "f"(y[3] * m), "f"(y[4] * m), "f"(y[5] * m),
              "f"(y[6] * m), "f"(y[7] * m));
    }
    if (w[0] != w[1]) {
        w[0] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[0] |= e2m1_code(y[e], s) << (4 * e);
    }
    return w[0];
}

struct AppendArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t* positions;
    const float* cos_sin;
    int n_positions, rot_dim;
    const int32_t* row_start;
    int n_requests;
    uint16_t* q_out;
    PagedView kv;
    int rows, Hq, Hkv, q_len;
    int warps_per_row;
};

// (a, b) -> (a c - b s, b c + a s) on two 8-element pieces.
template <bool kInterleaved>
__device__ __forceinline__ void rotate_pair(const uint4& lo, const uint4& hi, const float (&c)[8], const float (&s)[8],
                                            float (&y)[8], float (&z)[8])
{
    float a[8], b[8];
    unpack8(lo, a);
    unpack8(hi, b);
    if constexpr (kInterleaved) {  // pairs of neighbours: angles 0..3 are the first piece's, 4..7 the second's
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[2 * i] = __fsub_rn(__fmul_rn(a[2 * i], c[i]), __fmul_rn(a[2 * i + 1], s[i]));
            y[2 * i + 1] = __fadd_rn(__fmul_rn(a[2 * i + 1], c[i]), __fmul_rn(a[2 * i], s[i]));
            z[2 * i] = __fsub_rn(__fmul_rn(b[2 * i], c[4 + i]), __fmul_rn(b[2 * i + 1], s[4 + i]));
            z[2 * i + 1] = __fadd_rn(__fmul_rn(b[2 * i + 1], c[4 + i]), __fmul_rn(b[2 * i], s[4 + i]));
        }
    } else {  // the second piece is the first one's partner
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = __fsub_rn(__fmul_rn(a[i], c[i]), __fmul_rn(b[i], s[i]));
            z[i] = __fadd_rn(__fmul_rn(b[i], c[i]), __fmul_rn(a[i], s[i]));
        }
    }
}

__device__ __forceinline__ void load4(const float* p, float* x)
{
    const float4 v = __ldg(reinterpret_cast<const float4*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}

// A warp (or several, for few rows) per row.  Rotated or copied bf16 heads: D / 16 lanes a head, each with
// two 8-element pieces that are each other's partners where the head is rotated, so an element is read
// and widened once.  4-bit heads: D / 16 lanes a head too, each with sixteen neighbouring dimensions (a scale
// covers 32 of them: two lanes); their partners come from the same lines again.
// The first loads are on their way before it is known where the row goes.
template <int D, bool kFp4, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads, 3) append_kernel(const AppendArgs a)
{
    const int lane = threadIdx.x & 31;
    const int warp = blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
    const int row = warp / a.warps_per_row, part = warp - row * a.warps_per_row;
    if (row >= a.rows) return;
    const int n_q = a.q != nullptr ? a.Hq : 0;
    const int rot = a.rot_dim, half = rot / 2;
    const uint16_t* q_row = a.q + row * a.q_stride;
    const uint16_t* k_row = a.k + row * a.k_stride;
    const uint16_t* v_row = a.v + row * a.v_stride;

    constexpr int T = D / 16, kHeads = 32 / T;  // lanes of a head, heads of a pass
    constexpr int kAhead = 4;                   // passes whose loads are in flight
    const int n_k = n_q + (kFp4 ? 0 : a.Hkv), n_copy = n_k + (kFp4 ? 0 : a.Hkv);  // heads: queries, keys, values
    const int passes = (n_copy + kHeads - 1) / kHeads;
    const int t = lane % T;
    const bool rotated = t < rot / 16;
    // this lane's pieces
    const int da = rotated ? 8 * t : rot + 16 * (t - rot / 16), db = rotated && !kInterleaved ? da + half : rotated ? half + 8 * t : da + 8;
    uint4 lo[kAhead], hi[kAhead];
    auto load = [&](int pass0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = (pass0 + u * a.warps_per_row) * kHeads + lane / T;
            if (i >= n_copy) break;
            const uint16_t* src = i < n_q ? q_row + i * D : i < n_k ? k_row + (i - n_q) * D : v_row + (i - n_k) * D;
            lo[u] = __ldg(reinterpret_cast<const uint4*>(src + da));
            hi[u] = __ldg(reinterpret_cast<const uint4*>(src + db));
        }
    };
    load(part);
    const int pos = rot > 0 ? __ldg(a.positions + row) : 0;
    const bool known = rot == 0 || static_cast<unsigned>(pos) < static_cast<unsigned>(a.n_positions);
    const float* table = a.cos_sin + (int64_t)(known ? pos : 0) * rot;
    float c[8], s[8];
    if (rotated) {
        // angle of dimension d: d mod half, or d / 2 interleaved
        const int fa = kInterleaved ? da / 2 : da, fb = kInterleaved ? db / 2 : da + 4;
        load4(table + fa, c);
        load4(table + fb, c + 4);
        load4(table + half + fa, s);
        load4(table + half + fb, s + 4);
    }
    const RowPlace at = place_row(a.kv, row, a.q_len, a.row_start, a.n_requests);
    if (at.token < 0) return;  // padding
    if (!known) {
        if (lane == 0) atomicMin(a.kv.status, MOSKA_ERR_INVALID_ARG);
        return;
    }
    const int slot = at.token & ((1 << a.kv.page_shift) - 1);  // row inside the page
    const int64_t page_row = (((int64_t)at.page << a.kv.page_shift) + slot) * a.Hkv * D;  // bf16

    for (int pass0 = part; pass0 < passes; pass0 += kAhead * a.warps_per_row) {
        if (pass0 != part) load(pass0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = (pass0 + u * a.warps_per_row) * kHeads + lane / T;
            if (i >= n_copy) break;
            if (rotated && i < n_k) {
                float y[8], z[8];
                rotate_pair<kInterleaved>(lo[u], hi[u], c, s, y, z);
                lo[u] = pack8(y);
                hi[u] = pack8(z);
            }
            uint16_t* to;
            if (i < n_q) to = a.q_out + ((int64_t)row * a.Hq + i) * D;
            else if (at.page < 0) break;
            else if (i < n_k) to = reinterpret_cast<uint16_t*>(a.kv.k) + page_row + (i - n_q) * D;
            else to = reinterpret_cast<uint16_t*>(a.kv.v) + page_row + (i - n_k) * D;
            *reinterpret_cast<uint4*>(to + da) = lo[u];
            *reinterpret_cast<uint4*>(to + db) = hi[u];
        }
    }
    if constexpr (kFp4) {
        if (at.page < 0) return;
        using B = Fp4Block<D>;
        constexpr int T4 = D / 16, kHeads4 = 32 / T4;  // sixteen neighbouring dimensions a lane: two pieces
        const int n_kv = 2 * a.Hkv, passes4 = (n_kv + kHeads4 - 1) / kHeads4;
        const int t4 = lane % T4, d = 16 * t4;
        float c4[2][8], s4[2][8];  // interleaved: four angles a piece; sine negative in the first half
        int d_other[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int dp = d + 8 * p;
            const bool first = dp < half;
            d_other[p] = first ? dp + half : dp - half;
            if (dp >= rot) continue;
            const int f = kInterleaved ? dp / 2 : first ? dp : d_other[p];
            load4(table + f, c4[p]);
            load4(table + half + f, s4[p]);
            if constexpr (!kInterleaved) {
                load4(table + f + 4, c4[p] + 4);
                load4(table + half + f + 4, s4[p] + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) s4[p][e] = first ? -s4[p][e] : s4[p][e];
            }
        }
        const int tok = slot & (kBlockTokens - 1);
        uint8_t* blocks = a.kv.k + ((((int64_t)at.page * a.Hkv) << (a.kv.page_shift - 4)) + (slot >> 4)) * B::kBytes;
        const int head_bytes = B::kBytes << (a.kv.page_shift - 4);
        // the parts that have no bf16 pass left over begin; a pass's loads are one pass ahead
        int pass = (part + a.warps_per_row - passes % a.warps_per_row) % a.warps_per_row;
        uint4 own[2] = {}, other[2] = {};
        auto load_kv = [&](int next) {
            const int i = next * kHeads4 + lane / T4;
            if (i >= n_kv) return;
            const uint16_t* src = i >= a.Hkv ? v_row + (i - a.Hkv) * D : k_row + i * D;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                own[p] = __ldg(reinterpret_cast<const uint4*>(src + d + 8 * p));
                if (!kInterleaved && d + 8 * p < rot && i < a.Hkv)
                    other[p] = __ldg(reinterpret_cast<const uint4*>(src + d_other[p]));
            }
        };
        load_kv(pass);
        for (; pass < passes4; pass += a.warps_per_row) {
            const int i = pass * kHeads4 + lane / T4;
            const bool live = i < n_kv, is_v = i >= a.Hkv;
            const int h = is_v ? i - a.Hkv : i;
            float y[2][8];
            float top = 0.f;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                unpack8(own[p], y[p]);
                if (d + 8 * p < rot && !is_v) {
                    if constexpr (kInterleaved) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = y[p][2 * e], x1 = y[p][2 * e + 1];
                            y[p][2 * e] = __fsub_rn(__fmul_rn(x0, c4[p][e]), __fmul_rn(x1, s4[p][e]));
                            y[p][2 * e + 1] = __fadd_rn(__fmul_rn(x1, c4[p][e]), __fmul_rn(x0, s4[p][e]));
                        }
                    } else {
                        float z[8];
                        unpack8(other[p], z);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[p][e] = __fadd_rn(__fmul_rn(y[p][e], c4[p][e]), __fmul_rn(z[e], s4[p][e]));
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max_or_nan(top, fabsf(y[p][e]));
            }
            load_kv(pass + a.warps_per_row);
            // largest magnitude of the 32 dimensions (two lanes), NaN if one is
            top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const __half sh = __float2half_rn(top < INFINITY ? fminf(sixth(top), kFp4MaxScale) : NAN);
            const float sf = __half2float(sh);
            const uint32_t w0 = e2m1x8(y[0], sf), w1 = e2m1x8(y[1], sf);
            if (!live) continue;
            uint8_t* blk = blocks + (int64_t)h * head_bytes;
            if (is_v) {  // sixteen dimensions are one piece (D = 128) or two (D = 64) of the pair's row
                *reinterpret_cast<uint32_t*>(blk + B::v_byte(tok, d)) = w0;
                *reinterpret_cast<uint32_t*>(blk + B::v_byte(tok, d + 8)) = w1;
                if ((t4 & 1) == 0) *reinterpret_cast<__half*>(blk + B::v_scale(tok, t4 >> 1)) = sh;
            } else {
                *reinterpret_cast<uint32_t*>(blk + B::k_byte(tok, d)) = w0;
                *reinterpret_cast<uint32_t*>(blk + B::k_byte(tok, d + 8)) = w1;
                if ((t4 & 1) == 0) *reinterpret_cast<__half*>(blk + B::k_scale(tok, t4 >> 1)) = sh;
            }
        }
    }
}

// Warps of a row of append or gather: one for many rows; for few rows several, until every SM has sixteen
// warps or a warp has one pass of heads left.
int warps_per_row(int rows, int passes)
{
    const long long n = (148LL * 16 + rows - 1) / rows;
    return (int)(n < passes ? n : passes);
}

// Reading rows back: a warp (or several) per row, D / 8 lanes a head, eight elements a lane.
template <int D, bool kFp4>
__global__ void __launch_bounds__(kAppendThreads)
gather_kernel(const int32_t* __restrict__ row_start, int n_requests, uint16_t* __restrict__ k_out,
              uint16_t* __restrict__ v_out, PagedView kv, int rows, int Hkv, int q_len, int per_row)
{
    constexpr int T = D / 8, kHeads = 32 / T, kAhead = 4;
    const int lane = threadIdx.x & 31;
    const int warp = blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
    const int row = warp / per_row, part = warp - row * per_row;
    if (row >= rows) return;
    const int t = lane % T, d = 8 * t;
    const RowPlace at = place_row(kv, row, q_len, row_start, n_requests);
    if (at.token < 0 || at.page < 0) return;  // padding; an index outside the pool has been reported
    const int slot = at.token & ((1 << kv.page_shift) - 1);
    const int passes = (2 * Hkv + kHeads - 1) / kHeads;
    using B = Fp4Block<D>;
    const int tok = slot & (kBlockTokens - 1);
    const uint8_t* blocks = kv.k + ((((int64_t)at.page * Hkv) << (kv.page_shift - 4)) + (slot >> 4)) * B::kBytes;
    const int64_t head_bytes = (int64_t)B::kBytes << (kv.page_shift - 4);
    const int64_t page_row = (((int64_t)at.page << kv.page_shift) + slot) * Hkv * D;  // bf16
    const int k_at = B::k_byte(tok, d), v_at = B::v_byte(tok, d), ks_at = B::k_scale(tok, t >> 2), vs_at = B::v_scale(tok, t >> 2);
    for (int pass0 = part; pass0 < passes; pass0 += kAhead * per_row) {
        uint4 raw[kAhead];
        uint32_t code[kAhead];
        __half scale[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = (pass0 + u * per_row) * kHeads + lane / T;
            if (i >= 2 * Hkv) break;
            const bool is_v = i >= Hkv;
            const int h = is_v ? i - Hkv : i;
            if constexpr (kFp4) {
                const uint8_t* blk = blocks + h * head_bytes;
                code[u] = __ldg(reinterpret_cast<const uint32_t*>(blk + (is_v ? v_at : k_at)));
                scale[u] = __ldg(reinterpret_cast<const __half*>(blk + (is_v ? vs_at : ks_at)));
            } else {
                raw[u] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(is_v ? kv.v : kv.k) +
                                                              page_row + h * D + d));
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = (pass0 + u * per_row) * kHeads + lane / T;
            if (i >= 2 * Hkv) break;
            const bool is_v = i >= Hkv;
            const int h = is_v ? i - Hkv : i;
            if constexpr (kFp4) {
                const float s = __half2float(scale[u]);
                uint32_t f[4];
                e2m1x8_to_f16x2(code[u], f);
                float x[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f[e]));
                    x[2 * e] = p.x * s;
                    x[2 * e + 1] = p.y * s;
                }
                raw[u] = pack8(x);
            }
            *reinterpret_cast<uint4*>((is_v ? v_out : k_out) + ((int64_t)row * Hkv + h) * D + d) = raw[u];
        }
    }
}

}  // namespace

int launch_append_paged(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                        int64_t v_stride, const int32_t* positions, const float* cos_sin, int n_positions,
                        int rot_dim, int interleaved, const int32_t* row_start, int n_requests, uint16_t* q_out,
                        const PagedView& kv, bool fp4, const moska_shape* s, cudaStream_t st)
{
    if (s->B == 0) return MOSKA_OK;
    const int heads = (q != nullptr ? s->Hq : 0) + 2 * s->Hkv;
    const int per_row = warps_per_row(s->B, (heads * (s->D / 16) + 31) / 32);
    const AppendArgs args{q, k, v, q_stride, k_stride, v_stride, positions, cos_sin, n_positions, rot_dim, row_start,
                          n_requests, q_out, kv, s->B, s->Hq, s->Hkv, s->q_len > 1 ? s->q_len : 1, per_row};
    constexpr int kWarpsPerCta = kAppendThreads / 32;
    const long long warps = (long long)s->B * per_row;
    const unsigned grid = (unsigned)((warps + kWarpsPerCta - 1) / kWarpsPerCta);
    if (warps > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "too many rows");
    auto go = [&](auto kernel) { kernel<<<grid, kAppendThreads, 0, st>>>(args); };
    if (s->D == 128) {
        if (interleaved) fp4 ? go(append_kernel<128, true, true>) : go(append_kernel<128, false, true>);
        else fp4 ? go(append_kernel<128, true, false>) : go(append_kernel<128, false, false>);
    } else {
        if (interleaved) fp4 ? go(append_kernel<64, true, true>) : go(append_kernel<64, false, true>);
        else fp4 ? go(append_kernel<64, true, false>) : go(append_kernel<64, false, false>);
    }
    MOSKA_LAUNCH_CHECK("append_kernel");
    return MOSKA_OK;
}

int launch_gather_paged(const int32_t* row_start, int n_requests, uint16_t* k_out, uint16_t* v_out,
                        const PagedView& kv, bool fp4, const moska_shape* s, cudaStream_t st)
{
    if (s->B == 0) return MOSKA_OK;
    const int q_len = s->q_len > 1 ? s->q_len : 1;
    const int per_row = warps_per_row(s->B, (2 * s->Hkv * (s->D / 8) + 31) / 32);
    constexpr int kWarpsPerCta = kAppendThreads / 32;
    const long long warps = (long long)s->B * per_row;
    if (warps > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "too many rows");
    const unsigned grid = (unsigned)((warps + kWarpsPerCta - 1) / kWarpsPerCta);
    auto go = [&](auto kernel) {
        kernel<<<grid, kAppendThreads, 0, st>>>(row_start, n_requests, k_out, v_out, kv, s->B, s->Hkv, q_len, per_row);
    };
    if (s->D == 128) fp4 ? go(gather_kernel<128, true>) : go(gather_kernel<128, false>);
    else fp4 ? go(gather_kernel<64, true>) : go(gather_kernel<64, false>);
    MOSKA_LAUNCH_CHECK("gather_kernel");
    return MOSKA_OK;
}

}  // namespace moska
