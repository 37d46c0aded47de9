// Attention over a paged private store in 4 bits (E2M1 codes, one f16 scale per (token, KV head, 32
// dimensions)): a CTA per (request, KV head, split).
//
// The warps of a CTA take interleaved units of kSub 16-token blocks.  A block is one contiguous piece
// of a page (18 D bytes: key codes, value codes, scales), so one elected lane per block starts one
// bulk copy into the warp's own ring of units and an mbarrier per ring stage counts the bytes: no
// addresses per lane, no barrier between warps.  The block's byte order is the order of the MMA
// fragments, so a lane reads whole 16-byte pieces without bank conflicts.  The codes are widened to
// f16 in registers (cvt.rn.f16x2.e2m1x2, exact) for m16n8k16 MMAs with fp32 accumulation:
//   S^T  = sum_j kscale[token][j] (K4_j Q_j^T)     one accumulator per 32 dimensions, scaled after it
//   O^T += (V4 vscale[token][j])^T P               values scaled in f16, two tokens to a register
// Q is scaled per row by a power of two into f16's range: a bf16 element has eight bits and f16's steps end at
// 2^-24, so it is exact down to 2^-17 of the row's largest, and within 2^-25 of that below.  P is rounded to f16
// (half a step: 2^-11; 2^-32 of the row's largest at the lower end), row sums and statistics are fp32.
#include <cuda_bf16.h>

#include <cfloat>
#include <type_traits>

#include "paged.cuh"
#include "sm100.cuh"
#include "stream_attn.cuh"

namespace moska {
namespace {
using namespace stream;
static_assert(kThreads == kMaxOrdered, "a request a thread");

constexpr float kBelow = 7.f, kMost = 15.f;  // log2 of P: of the largest when the reference is taken, at most

// Blocks of a unit; of two column blocks four spill at 255 registers (48 x 4 query tokens: 62 us, 64 at four,
// 76 at two).
template <int NT>
constexpr int kSubOf = NT == 2 ? 3 : 4;

template <int D, int NT>
struct F4Ring {
    static constexpr int kSub = kSubOf<NT>;
    static constexpr int kDepth = 2;  // units in flight per warp
    static constexpr int kUnitBytes = kSub * Fp4Block<D>::kBytes;
    static constexpr int kBytes = kWarps * kDepth * kUnitBytes;
};

// Results of the warps before they are joined; rows padded by four floats (fewer bank conflicts).
template <int D, int NT>
struct F4Join {
    float o[kWarps][NT * 8][D + 4];
    float m[kWarps][NT * 8];  // log2 units
    float l[kWarps][NT * 8];
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
        "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t f16x2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b)
{
    const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}

// a where m has ones, b elsewhere
__device__ __forceinline__ uint32_t select_bits(uint32_t m, uint32_t a, uint32_t b)
{
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xe4;" : "=r"(y) : "r"(a), "r"(b), "r"(m));
    return y;
}

template <int N>  // N = 1, 2 or 4 words
__device__ __forceinline__ void lds_words(uint32_t addr, uint32_t (&w)[N])
{
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr));
    else if constexpr (N == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(addr));
}

// Untiled copy global -> shared; both addresses 16-byte aligned, size a multiple of 16.
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(sm100::smem_u32(bar))
                 : "memory");
}

struct AttnArgs {
    const uint16_t* q;
    PagedView kv;
    float* o_part;     // partial slots (nullptr: `out` gets the final rows)
    float* lse_part;
    uint16_t* out;
    float* lse_out;
    float scale;
    int Hq, Hkv, n_splits, slot0, n_slots, q_len;
    int n_requests;
};

// CTAs per SM.  D = 128: 164 registers (a fourth CTA would need 128: spills, slower).  D = 64: 123; four
// take 24 us over 128 contexts of 2000 tokens where three take 33.  Two column blocks: 252 registers
// (three CTAs of 168 spill: 69 us over 48 x 4 query tokens where two take 62).
template <int D, int NT>
constexpr int kCtasPerSm = NT == 2 ? 2 : D == 128 ? 3 : 4;

// kOrdered: requests longest context first.
template <int D, int NT, bool kOrdered>
__global__ void __launch_bounds__(kThreads, kCtasPerSm<D, NT>) paged_fp4_kernel(const AttnArgs a)
{
    using B = Fp4Block<D>;
    constexpr int J = B::kGroups, MT = D / 16, kSub = kSubOf<NT>;
    constexpr int kUnit = kSub * kBlockTokens, kRows = NT * 8, kDepth = F4Ring<D, NT>::kDepth;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ uint64_t full[kWarps][kDepth];
    __shared__ int gave_up;
    __shared__ typename std::conditional<kOrdered, OrderSmem, int>::type order;
    __shared__ int64_t row_of[kRows];  // result row of each query row, -1: none
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;
    const int G = a.Hq / a.Hkv;
    const int h = blockIdx.x % a.Hkv;
    const int sp = (blockIdx.x / a.Hkv) % a.n_splits;
    int r = blockIdx.x / (a.Hkv * a.n_splits);
    const int q_len = a.q_len, n_rows = q_len * G;

    dependents_may_launch();
    int len;
    if constexpr (kOrdered) r = request_at(a.kv, a.n_requests, r, order, len);
    if (threadIdx.x == 0) gave_up = 0;
    if (threadIdx.x < kRows) {
        const int j = threadIdx.x;
        row_of[j] = j < n_rows ? ((int64_t)r * q_len + j / G) * a.Hq + h * G + j % G : -1;
    }
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < kDepth; ++s) sm100::mbar_init(&full[warp][s], kSub);
        sm100::fence_mbar_init();
        sm100::fence_proxy_async_smem();
    }
    __syncthreads();

    if constexpr (!kOrdered) len = paged_len(a.kv, r);
    // this split's tokens: equal parts rounded up to a pass of the CTA's warps
    constexpr int kPass = kWarps * kUnit;
    int per = (len + a.n_splits - 1) / a.n_splits;
    per = (per + kPass - 1) / kPass * kPass;
    const int t_begin = (int)min((long long)len, (long long)sp * per), t_end = min(len, t_begin + per);
    const int n_units = (t_end - t_begin + kUnit - 1) / kUnit;
    const int mine = n_units > warp ? (n_units - warp + kWarps - 1) / kWarps : 0;

    const uint32_t ring_base = sm100::smem_u32(ring) + warp * (kDepth * F4Ring<D, NT>::kUnitBytes);
    const int32_t* pages = a.kv.page_table + (int64_t)r * a.kv.max_pages;
    const int shift = a.kv.page_shift;
    // Lane j < kSub loads block j of every unit: `ahead` is that block's token in the unit to ask for next.
    // Pages are looked up one unit before the copy that needs them.
    const bool loads = lane < kSub;
    int ahead = t_begin + warp * kUnit + lane * kBlockTokens;
    const uint32_t page_bytes = ((uint32_t)a.Hkv << (shift - 4)) * B::kBytes;
    const uint8_t* pool = a.kv.k + ((uint64_t)h << (shift - 4)) * B::kBytes;
    const uint32_t lane_slot = ring_base + lane * B::kBytes;
    auto page_ahead = [&] { return loads && ahead < t_end ? paged_page(a.kv, pages, ahead >> shift) : 0; };
    // starts the copy of the unit that `ahead` is in, into ring stage s; every loading lane arrives
    auto issue = [&](int s, int page) {
        if (loads) {
            uint64_t* bar = &full[warp][s];
            if (ahead < t_end) {
                const uint32_t block = (uint32_t)(ahead >> 4) & ((1u << (shift - 4)) - 1);
                sm100::mbar_arrive_expect_tx(bar, B::kBytes);
                bulk_load(lane_slot + s * F4Ring<D, NT>::kUnitBytes, pool + (uint64_t)(uint32_t)page * page_bytes + block * B::kBytes,
                          B::kBytes, bar);
            } else {
                sm100::mbar_arrive(bar);
            }
        }
        ahead += kWarps * kUnit;
    };
    int next_page = page_ahead();
    {
        int first[kDepth];
        first[0] = next_page;
#pragma unroll
        for (int s = 1; s < kDepth; ++s) {  // all lookups in flight before the first copy
            ahead += kWarps * kUnit;
            first[s] = page_ahead();
        }
        ahead -= (kDepth - 1) * kWarps * kUnit;
#pragma unroll
        for (int s = 0; s < kDepth; ++s)
            if (s < mine) issue(s, first[s]);
        next_page = page_ahead();
    }

    // Q as the B operand: step 2 j + u covers dimensions 32 j + 8 c + 4 u .. + 3; the row is scaled by a
    // power of two so that its largest element lies in [1, 2)
    uint32_t qf[NT][2 * J][2];
    float unit[NT][2];  // scale * log2(e) over that power, for columns 2c and 2c + 1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int j = n * 8 + g;
        const int64_t row = row_of[j];
        const bool live = row >= 0;
        float x[J][8];
        float top = 0.f;
#pragma unroll
        for (int u = 0; u < J; ++u) {
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (live)
                raw = ldg16(a.q + row * D + 32 * u + 8 * c);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[u][2 * e] = __uint_as_float(w[e] << 16);
                x[u][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                top = fmaxf(top, fmaxf(fabsf(x[u][2 * e]), fabsf(x[u][2 * e + 1])));
            }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^-e with 2^e <= top < 2^(e+1); a zero row, a denormal or a non-finite one stays in range
        const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252) - 127;
        const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int u = 0; u < J; ++u) {
            qf[n][2 * u][0] = f16x2(x[u][0] * down, x[u][1] * down);
            qf[n][2 * u][1] = f16x2(x[u][2] * down, x[u][3] * down);
            qf[n][2 * u + 1][0] = f16x2(x[u][4] * down, x[u][5] * down);
            qf[n][2 * u + 1][1] = f16x2(x[u][6] * down, x[u][7] * down);
        }
        // (neither 0 nor infinite: the -inf of a hidden token, or a score of 0, times that would be NaN)
        const float mul = fminf(fmaxf(a.scale * up * kLog2e, FLT_MIN), FLT_MAX);
        unit[n][0] = __shfl_sync(0xffffffffu, mul, (2 * c) * 4);
        unit[n][1] = __shfl_sync(0xffffffffu, mul, (2 * c + 1) * 4);
    }
    // tokens that columns 2c, 2c + 1 see: [0, seen)
    int seen[NT][2];
    const int all_see = len - (q_len - 1);  // tokens that every row sees
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int j = n * 8 + 2 * c + u;
            seen[n][u] = j < n_rows ? len - (q_len - 1 - j / G) : len;
        }

    float oacc[NT][MT][4];
    float m_run[NT][2], l_run[NT][2];  // reference of the scores (log2 units) and row sum of columns 2c, 2c + 1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m_run[n][0] = m_run[n][1] = -INFINITY;
        l_run[n][0] = l_run[n][1] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) oacc[n][mt][0] = oacc[n][mt][1] = oacc[n][mt][2] = oacc[n][mt][3] = 0.f;
    }

    // SUB blocks at `at` in the ring, from token t0; `tail`: some row's context ends in them.
    auto step = [&](auto subs, auto is_tail, uint32_t at, int t0) {
        constexpr int SUB = decltype(subs)::value;
        constexpr bool tail = decltype(is_tail)::value;
        // ---- S^T of the unit's blocks
        float sc[NT][SUB][4];
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            const uint32_t blk = at + b * B::kBytes;
            uint32_t ka[J], kb[J];
            lds_words<J>(blk + g * (D / 2) + c * (D / 8), ka);
            lds_words<J>(blk + (g + 8) * (D / 2) + c * (D / 8), kb);
            uint32_t sa[J / 2], sb[J / 2];
            lds_words<J / 2>(blk + B::k_scale(g, 0), sa);
            lds_words<J / 2>(blk + B::k_scale(g + 8, 0), sb);
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][b][0] = sc[n][b][1] = sc[n][b][2] = sc[n][b][3] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                uint32_t fa[4], fb[4];
                e2m1x8_to_f16x2(ka[j], fa);
                e2m1x8_to_f16x2(kb[j], fb);
                const float2 pa = __half22float2(*reinterpret_cast<const __half2*>(&sa[j >> 1]));
                const float2 pb = __half22float2(*reinterpret_cast<const __half2*>(&sb[j >> 1]));
                const float ksa = (j & 1) ? pa.y : pa.x, ksb = (j & 1) ? pb.y : pb.x;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_f16(acc, fa[0], fb[0], fa[1], fb[1], qf[n][2 * j][0], qf[n][2 * j][1]);
                    mma_f16(acc, fa[2], fb[2], fa[3], fb[3], qf[n][2 * j + 1][0], qf[n][2 * j + 1][1]);
                    sc[n][b][0] = fmaf(acc[0], ksa, sc[n][b][0]);
                    sc[n][b][1] = fmaf(acc[1], ksa, sc[n][b][1]);
                    sc[n][b][2] = fmaf(acc[2], ksb, sc[n][b][2]);
                    sc[n][b][3] = fmaf(acc[3], ksb, sc[n][b][3]);
                }
            }
        }
        // ---- online softmax over the unit.  P is relative to a reference (m_run) taken so that the largest P so
        // far is 2^kBelow; it moves again when one would pass 2^kMost.  Rescaling the accumulators is rare that
        // way, and f16 (steps of 2^-24 at its lower end) holds probabilities down to 2^-31 of the row's
        // largest: what rounds to 0 adds up to less than 2^-12 in a million tokens.
        float mx[NT][2];
        bool grew = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mx[n][0] = mx[n][1] = -INFINITY;
#pragma unroll
            for (int b = 0; b < SUB; ++b) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (tail)
                        if (t0 + b * 16 + g + 8 * (e >> 1) >= min(t_end, seen[n][e & 1])) sc[n][b][e] = -INFINITY;
                    mx[n][e & 1] = fmaxf(mx[n][e & 1], sc[n][b][e]);
                }
            }
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) {
                mx[n][0] = fmaxf(mx[n][0], __shfl_xor_sync(0xffffffffu, mx[n][0], off));
                mx[n][1] = fmaxf(mx[n][1], __shfl_xor_sync(0xffffffffu, mx[n][1], off));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) grew |= fmaf(mx[n][e], unit[n][e], -m_run[n][e]) > kMost;
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float alpha[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float top = mx[n][e] * unit[n][e] - kBelow;
                    // (m_run = -inf: no token seen yet, nothing to rescale; top = -inf: none in this unit either)
                    const bool moves = top > m_run[n][e];
                    alpha[e] = moves ? fast_exp2(m_run[n][e] - top) : 1.f;
                    if (moves) m_run[n][e] = top;
                    l_run[n][e] *= alpha[e];
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    oacc[n][mt][0] *= alpha[0];
                    oacc[n][mt][1] *= alpha[1];
                    oacc[n][mt][2] *= alpha[0];
                    oacc[n][mt][3] *= alpha[1];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // a row that has seen no token yet: keep its (empty) state free of inf - inf
            const float ms0 = tail && m_run[n][0] == -INFINITY ? 0.f : m_run[n][0];
            const float ms1 = tail && m_run[n][1] == -INFINITY ? 0.f : m_run[n][1];
#pragma unroll
            for (int b = 0; b < SUB; ++b) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc[n][b][e] = fast_exp2(fmaf(sc[n][b][e], unit[n][e & 1], (e & 1) ? -ms1 : -ms0));
                l_run[n][0] += sc[n][b][0] + sc[n][b][2];
                l_run[n][1] += sc[n][b][1] + sc[n][b][3];
            }
        }
        // ---- O^T += V^T P.  Where a token that not every row sees holds NaN, the block is passed once for each
        // query token over the values that it sees, kept in its columns only: 0 times NaN is NaN.
        // (Rows behind the whole context hold anything; codes are finite, so zero scales make them 0.)
        int passes = 1;
        if constexpr (tail) {
            // (SUB is 1 here) a scale above the largest that append writes, infinities and NaN included
            uint32_t s0[1], s1[1];
            lds_words<1>(at + B::v_scale(2 * c, g * J / 8), s0);
            lds_words<1>(at + B::v_scale(2 * c + 8, g * J / 8), s1);
            const int t = t0 + 2 * c;
            auto odd = [&](uint32_t bits, int tok) { return (bits & 0x7fffu) > 0x7154u && tok >= all_see && tok < t_end; };
            const bool bad = odd(s0[0], t) || odd(s0[0] >> 16, t + 1) || odd(s1[0], t + 8) || odd(s1[0] >> 16, t + 9);
            if (__any_sync(0xffffffffu, bad)) passes = q_len;
        }
        for (int pass = 0; pass < passes; ++pass) {
            // tail: values of tokens from here on are hidden
            const int limit = passes == 1 ? len : len - (q_len - 1 - pass);
#pragma unroll
            for (int b = 0; b < SUB; ++b) {
                const uint32_t blk = at + b * B::kBytes;
                uint32_t pb0[NT], pb1[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    pb0[n] = movmatrix_trans(f16x2(sc[n][b][0], sc[n][b][1]));
                    pb1[n] = movmatrix_trans(f16x2(sc[n][b][2], sc[n][b][3]));
                }
                // value chunk g of token pairs c (tokens 2c, 2c+1) and c + 4; first token's bytes, then the second's
                constexpr int W = J / 2;  // words of a token's chunk
                uint32_t va[2 * W], vb[2 * W], s0[1], s1[1];
                const uint32_t chunk = (g ^ B::v_swap(c)) * (D / 8);
                lds_words<2 * W>(blk + B::kV + c * D + chunk, va);
                lds_words<2 * W>(blk + B::kV + (c + 4) * D + chunk, vb);
                constexpr int kLanesPerGroup = 8 / J;  // lane groups g that share a scale
                lds_words<1>(blk + B::v_scale(2 * c, g / kLanesPerGroup), s0);
                lds_words<1>(blk + B::v_scale(2 * c + 8, g / kLanesPerGroup), s1);
                if constexpr (tail) {
                    const int t = t0 + b * 16 + 2 * c, end = min(t_end, limit);
                    s0[0] &= (t < end ? 0xffffu : 0u) | (t + 1 < end ? 0xffff0000u : 0u);
                    s1[0] &= (t + 8 < end ? 0xffffu : 0u) | (t + 9 < end ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    // byte e: dimension 8 w + 2 e (even) or 8 w + 2 e + 1 (odd) of both tokens of a pair
                    const uint32_t m = 0x0f0f0f0fu;
                    const uint32_t a_even = select_bits(m, va[w], va[W + w] << 4);
                    const uint32_t a_odd = select_bits(m, va[w] >> 4, va[W + w]);
                    const uint32_t b_even = select_bits(m, vb[w], vb[W + w] << 4);
                    const uint32_t b_odd = select_bits(m, vb[w] >> 4, vb[W + w]);
                    uint32_t f0[4], f1[4], f2[4], f3[4];
                    e2m1x8_to_f16x2(a_even, f0);
                    e2m1x8_to_f16x2(a_odd, f1);
                    e2m1x8_to_f16x2(b_even, f2);
                    e2m1x8_to_f16x2(b_odd, f3);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t a0 = hmul2(f0[e], s0[0]), a1 = hmul2(f1[e], s0[0]);
                        const uint32_t a2 = hmul2(f2[e], s1[0]), a3 = hmul2(f3[e], s1[0]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float(&acc)[4] = oacc[n][4 * w + e];
                            if (!tail || passes == 1) {
                                mma_f16(acc, a0, a1, a2, a3, pb0[n], pb1[n]);
                            } else {
                                float x[4] = {acc[0], acc[1], acc[2], acc[3]};
                                mma_f16(x, a0, a1, a2, a3, pb0[n], pb1[n]);
#pragma unroll
                                for (int y = 0; y < 4; ++y)
                                    if (seen[n][y & 1] == limit) acc[y] = x[y];
                            }
                        }
                    }
                }
            }
        }
    };

    int i = 0, s = 0, t0 = t_begin + warp * kUnit;
    uint32_t parity = 0;
    const int masked = min(t_end, all_see);  // units that reach past this token go block by block, with masks
    for (; i < mine; ++i, t0 += kWarps * kUnit) {
        if (!__all_sync(0xffffffffu, sm100::mbar_wait(&full[warp][s], parity, &gave_up))) {
            if (lane == 0) atomicMin(a.kv.status, MOSKA_ERR_TIMEOUT);
            break;
        }
        const uint32_t at = ring_base + s * F4Ring<D, NT>::kUnitBytes;
        if (t0 + kUnit <= masked) {
            step(std::integral_constant<int, kSub>{}, std::false_type{}, at, t0);
        } else {
            for (int t = t0; t < min(t_end, t0 + kUnit); t += kBlockTokens)
                step(std::integral_constant<int, 1>{}, std::true_type{}, at + ((t - t0) / kBlockTokens) * B::kBytes, t);
        }
        __syncwarp();  // every lane has read the stage into registers: refill it
        if (i + kDepth < mine) issue(s, next_page);
        next_page = page_ahead();
        if (++s == kDepth) {
            s = 0;
            parity ^= 1;
        }
    }
    // gave up on unit i: the copies in flight end (each wait again has a limit) before the ring is reused
    for (int stop = min(mine, i + kDepth); i < stop; ++i) {
        int never = 0;
        sm100::mbar_wait(&full[warp][i % kDepth], (i / kDepth) & 1, &never);
    }

    // ---- combine the warps through the (now idle) ring
    __syncthreads();
    F4Join<D, NT>& sm = *reinterpret_cast<F4Join<D, NT>*>(ring);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
            l_run[n][0] += __shfl_xor_sync(0xffffffffu, l_run[n][0], off);
            l_run[n][1] += __shfl_xor_sync(0xffffffffu, l_run[n][1], off);
        }
    static_assert(sizeof(F4Join<D, NT>) <= F4Ring<D, NT>::kBytes, "the join reuses the ring");
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n * 8 + 2 * c >= n_rows) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int j = n * 8 + 2 * c + u;
            if (g == 0) {
                sm.m[warp][j] = m_run[n][u];
                sm.l[warp][j] = l_run[n][u];
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)  // rows g and g + 8 of block mt: dimensions d and d + 1
                *reinterpret_cast<float2*>(&sm.o[warp][j][g * (D / 8) + 2 * mt]) = make_float2(oacc[n][mt][u], oacc[n][mt][2 + u]);
        }
    }
    __syncthreads();
    // four dimensions a thread
    for (int i = threadIdx.x; i < n_rows * (D / 4); i += kThreads) {
        const int j = i / (D / 4), d = i % (D / 4) * 4;
        const int64_t row = row_of[j];
        float M = sm.m[0][j];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sm.m[w][j]);
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            // (all maxima -inf: no token, or NaN scores alone, whose sum is NaN)
            const float al = M != -INFINITY ? fast_exp2(sm.m[w][j] - M) : 1.f;
            const float4 o = *reinterpret_cast<const float4*>(&sm.o[w][j][d]);
            num.x = fmaf(al, o.x, num.x);
            num.y = fmaf(al, o.y, num.y);
            num.z = fmaf(al, o.z, num.z);
            num.w = fmaf(al, o.w, num.w);
            den = fmaf(al, sm.l[w][j], den);
        }
        const float inv = den == 0.f ? 0.f : 1.f / den;
        const float lse = den == 0.f ? -INFINITY : M * kLn2 + logf(den);
        num = make_float4(num.x * inv, num.y * inv, num.z * inv, num.w * inv);
        if (a.out != nullptr) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(num.x, num.y), hi = __floats2bfloat162_rn(num.z, num.w);
            *reinterpret_cast<uint2*>(a.out + row * D + d) =
                make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            if (d == 0 && a.lse_out != nullptr) a.lse_out[row] = lse;
        } else {
            const int64_t slot = row * a.n_slots + a.slot0 + sp;
            *reinterpret_cast<float4*>(a.o_part + slot * D + d) = num;
            if (d == 0) a.lse_part[slot] = lse;
        }
    }
}

}  // namespace

// `out` == nullptr: partial slots slot0 .. of n_slots; else the final rows (one split).
int launch_paged_fp4(const uint16_t* q, const PagedView& kv, float* o_part, float* lse_part, int slot0, int n_slots,
                     uint16_t* out, float* lse_out, float scale, const moska_shape* s, cudaStream_t st)
{
    const int q_len = s->q_len > 1 ? s->q_len : 1;
    const long long grid = (long long)(s->B / q_len) * s->Hkv * s->n_unique_splits;
    if (grid == 0) return MOSKA_OK;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "paged attention grid too large");
    const AttnArgs a{q, kv, o_part, lse_part, out, lse_out, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0, n_slots, q_len,
                     s->B / q_len};
    auto go = [&](auto kernel, int ring) {
        MOSKA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring));
        kernel<<<(unsigned)grid, kThreads, ring, st>>>(a);
        MOSKA_LAUNCH_CHECK("paged_fp4_kernel");
        return (int)MOSKA_OK;
    };
    const bool two = q_len * (s->Hq / s->Hkv) > 8;
    auto form = [&](auto ordered) {
        constexpr bool O = decltype(ordered)::value;
        if (s->D == 128)
            return two ? go(paged_fp4_kernel<128, 2, O>, F4Ring<128, 2>::kBytes) : go(paged_fp4_kernel<128, 1, O>, F4Ring<128, 1>::kBytes);
        return two ? go(paged_fp4_kernel<64, 2, O>, F4Ring<64, 2>::kBytes) : go(paged_fp4_kernel<64, 1, O>, F4Ring<64, 1>::kBytes);
    };
    return longest_first(a.n_requests, grid) ? form(std::true_type{}) : form(std::false_type{});
}

}  // namespace moska
