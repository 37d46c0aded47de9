// Attention of the nodes of drafted trees over the paged contexts that they end, on the 5th-generation tensor cores.
//
// The T G query rows of a request's KV head (T nodes, G heads each) share one context.  A CTA takes up to 128 of them
// (whole nodes) and a split of the context, in tiles of 128 tokens:
//   S = Q K^T          tcgen05.mma, both operands in shared memory, 128 x 128 scores in tensor memory
//   P = exp2(S - m)    a thread per row: TMEM -> registers -> 16 bits, back over the columns of S
//   O += P V           tcgen05.mma, P from TMEM, V from shared memory, a 64-dimension half at a time
// Two CTAs share an SM (half of its shared and of its tensor memory each): while one is in its softmax the other
// has the tensor cores, and one's prologue and epilogue run under the other's tiles.  The CTAs of a KV head's row tiles
// are neighbours in the grid, so that the second and later read the context from L2.
//
// Warps 0-3: softmax (thread i: row i = TMEM lane i).  Warp 4: copies.  Warp 5: MMAs.  4-bit pages: warps 6-9 widen.
// Operands lie in a ring of 16 KB slots (128 tokens x 64 dimensions, rows of 128 bytes with the 128-byte swizzle).
//   bf16: one TMA box of min(page_size, 128) tokens a page and half.
//   4 bits: bulk copies of the key part or the value part (codes, then scales) of four 16-token blocks into a ring of their
//   own; a warp per block widens them to f16 operands, code times scale (half a step: 2^-11).  Queries are f16 too,
//   scaled by a power of two per row.
//
// What a node sees: committed tokens, and of the last T tokens those whose bit is set in its 64-bit word of ancestors.
// Only tiles that reach past the committed tokens look at it.  0 times NaN is NaN, so values of such tiles that are
// not finite are taken out of the operands (a bit per token remembers), and put into the rows that see them at the end.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <mutex>

#include "sm100.cuh"
#include "tree.cuh"

namespace moska {
namespace {
using namespace sm100;

constexpr int kTile = 128;                 // tokens of a tile
constexpr int kSlotBytes = kTile * 64 * 2;  // 64 dimensions of a tile
constexpr int kTileRows = 128;             // query rows of a CTA
constexpr int kLoadWarp = 4, kMmaWarp = 5, kWidenWarp0 = 6;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRescaleAt = 8.f;  // log2 units that a row's maximum may grow before its sums are rescaled

template <int D, bool F4>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kThreads = F4 ? 320 : 192;
    static constexpr int kSlots = F4 ? (D == 128 ? 4 : 5) : (D == 128 ? 5 : 6);
    static constexpr int kUnitBlocks = 4;              // 16-token blocks of a unit of codes
    static constexpr int kPartBytes = 9 * D;           // codes and scales of a block's keys, or of its values
    static constexpr int kUnitBytes = kUnitBlocks * kPartBytes;
    static constexpr int kUnits = F4 ? (D == 128 ? 3 : 6) : 0;
};

// One CTA's shared memory: half of an SM's.
template <int D, bool F4>
struct Smem {
    using C = Cfg<D, F4>;
    uint8_t q[C::kHalves][kSlotBytes];
    uint8_t slot[C::kSlots][kSlotBytes];
    uint8_t unit[F4 ? C::kUnits * C::kUnitBytes : 16];
    float row_unit[F4 ? kTileRows : 4];  // log2 units of one score of a row
    uint64_t full[C::kSlots], empty[C::kSlots];
    uint64_t unit_full[F4 ? C::kUnits : 1], unit_empty[F4 ? C::kUnits : 1];
    uint64_t q_full, s_full, p_full, o_full;
    unsigned long long bad;  // tree tokens with values that are not finite
    uint32_t tmem_base;
    int gave_up;
};
constexpr int kMostSmem = 115712;  // 2 x (that + 1 KB that the system takes) = 228 KB
static_assert(sizeof(Smem<128, false>) <= kMostSmem && sizeof(Smem<128, true>) <= kMostSmem &&
                  sizeof(Smem<64, false>) <= kMostSmem && sizeof(Smem<64, true>) <= kMostSmem,
              "two CTAs share an SM");
static_assert(sizeof(TreeSmem) <= kSlotBytes, "the ancestors' scratch lies where the queries come");

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
    int row_tiles;       // of the largest tree
    int nodes_per_tile;  // 128 / G
};

__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float fmax3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint32_t f16x2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b)
{
    const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ void tma_load_3d(void* dst, const void* map, int x, int y, int z, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// The calling warp waits; false if the CTA has given up.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* gave_up)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, gave_up));
}

// What all roles of a CTA know.
struct Work {
    int first, nodes;   // the request's rows
    int len, committed;
    int h, r, split;
    int node0, rows;    // first node of the row tile, its rows
    int tile0, tiles;   // tiles of the split
};

__device__ __forceinline__ Work work_of(const TreeArgs& a)
{
    Work w;
    int x = blockIdx.x;
    const int rt = x % a.row_tiles;
    x /= a.row_tiles;
    w.h = x % a.Hkv;
    x /= a.Hkv;
    w.split = x % a.n_splits;
    w.r = x / a.n_splits;
    const int2 rows = tree_rows(a.tree, w.r, a.kv.status);
    w.first = rows.x;
    w.nodes = rows.y;
    w.len = paged_len(a.kv, w.r);
    w.committed = w.len - w.nodes;
    w.node0 = rt * a.nodes_per_tile;
    w.rows = min(a.nodes_per_tile, max(0, w.nodes - w.node0)) * (a.Hq / a.Hkv);
    const int all = (w.len + kTile - 1) / kTile, per = (all + a.n_splits - 1) / a.n_splits;
    w.tile0 = min(all, w.split * per);
    w.tiles = min(all, w.tile0 + per) - w.tile0;
    return w;
}

// Rows of a query tile: bf16 as they are, or f16 times a power of two that brings the row's largest element into
// [1, 2) (exact down to 2^-17 of it, within 2^-25 of it below); 128-byte swizzled operand rows, 0 where there is no row.
template <int D, bool F4>
__device__ __forceinline__ void stage_queries(Smem<D, F4>& sm, const TreeArgs& a, const Work& w, int warp, int lane)
{
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // lanes of a row, rows at once
    const int G = a.Hq / a.Hkv, ch = lane % kLanes;
#pragma unroll 4
    for (int i0 = 0; i0 < 32; i0 += kRows) {
        const int i = warp * 32 + i0 + lane / kLanes;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (i < w.rows)
            x = __ldg(reinterpret_cast<const uint4*>(
                a.q + ((int64_t)(w.first + w.node0 + i / G) * a.Hq + w.h * G + i % G) * D + 8 * ch));
        if constexpr (F4) {
            const uint32_t word[4] = {x.x, x.y, x.z, x.w};
            float f[8], top = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[2 * e] = __uint_as_float(word[e] << 16);
                f[2 * e + 1] = __uint_as_float(word[e] & 0xffff0000u);
                top = fmaxf(top, fmaxf(fabsf(f[2 * e]), fabsf(f[2 * e + 1])));
            }
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252) - 127;
            const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
            // (neither 0 nor infinite: the -inf of a hidden token, or a score of 0, times that would be NaN)
            if (ch == 0) sm.row_unit[i] = fminf(fmaxf(a.scale * up * kLog2e, FLT_MIN), FLT_MAX);
            x = make_uint4(f16x2(f[0] * down, f[1] * down), f16x2(f[2] * down, f[3] * down), f16x2(f[4] * down, f[5] * down),
                           f16x2(f[6] * down, f[7] * down));
        }
        *reinterpret_cast<uint4*>(&sm.q[ch >> 3][i * 128 + (((ch & 7) ^ (i & 7)) << 4)]) = x;
    }
}

// Columns 32 c .. 32 c + 31 of a tile that begins at token t0: those that a row sees.
__device__ __forceinline__ uint32_t seen_columns(int t, int committed, int len, unsigned long long sees)
{
    if (t + 32 <= committed) return 0xffffffffu;
    uint32_t bits;
    const int behind = t - committed;  // first column's place behind the committed tokens
    if (behind >= 0) {
        bits = behind < 64 ? (uint32_t)(sees >> behind) : 0u;
    } else {
        bits = (uint32_t)(sees << -behind) | ((1u << -behind) - 1u);
    }
    return t + 32 <= len ? bits : len > t ? bits & ((1u << (len - t)) - 1u) : 0u;
}

template <int D, bool F4>
__device__ __forceinline__ void softmax_role(Smem<D, F4>& sm, const TreeArgs& a, const Work& w, uint32_t tmem, int warp, int lane)
{
    using C = Cfg<D, F4>;
    const int i = threadIdx.x, G = a.Hq / a.Hkv;
    int* gave_up = &sm.gave_up;

    // ---- what this row sees: the ancestors' words, in memory that the queries take next
    TreeSmem& ts = *reinterpret_cast<TreeSmem*>(sm.q[0]);
    if (i < MOSKA_TREE_MAX_NODES)
        tree_ancestors(ts, i, i < w.nodes ? tree_parent(a.tree, w.first, i, a.kv.status) : -1,
                       [] { asm volatile("bar.sync 2, 64;" ::: "memory"); });
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const bool live = i < w.rows;
    const int node = w.node0 + i / G;
    unsigned long long sees = 0;
    if (live && w.committed + node >= 0) sees = ts.bits[node];
    if (w.committed < 0) sees &= ~0ull << min(63, -w.committed);  // nodes without a token
    asm volatile("bar.sync 1, 128;" ::: "memory");
    stage_queries<D, F4>(sm, a, w, warp, lane);
    fence_proxy_async_smem();
    mbar_arrive(&sm.q_full);

    const int64_t row = (int64_t)(w.first + node) * a.Hq + w.h * G + i % G;
    const int64_t slot = row * a.n_slots + a.slot0 + w.split;
    const uint32_t t_s = tmem + (static_cast<uint32_t>(warp * 32) << 16), t_o = t_s + kTile;
    const bool warp_live = warp * 32 < w.rows;
    if constexpr (F4) asm volatile("bar.sync 1, 128;" ::: "memory");  // row_unit
    const float unit = F4 ? sm.row_unit[F4 ? i : 0] : a.scale * kLog2e;
    float m_ref = -INFINITY, l_sum = 0.f;
    bool alive = true;
    for (int j = 0; j < w.tiles; ++j) {
        const int t0 = (w.tile0 + j) * kTile;
        const bool ends = t0 + kTile > w.committed;  // some row does not see all of the tile
        if constexpr (!F4) {
            if (ends) {
                // Values behind the context, and those of drafted tokens that are not finite, become 0: token row i here
                const int t = t0 + i;
                const int seq = j * 2 * C::kHalves + C::kHalves;
#pragma unroll
                for (int hv = 0; hv < C::kHalves; ++hv)
                    alive = alive && warp_wait(&sm.full[(seq + hv) % C::kSlots], ((seq + hv) / C::kSlots) & 1, gave_up);
                if (!alive) break;
                if (t >= w.committed) {
#pragma unroll
                    for (int hv = 0; hv < C::kHalves; ++hv) {
                        uint8_t* at = &sm.slot[(seq + hv) % C::kSlots][i * 128];
#pragma unroll 1
                        for (int x = 0; x < 8; ++x) {
                            uint4* p = reinterpret_cast<uint4*>(at + (((x + i) & 7) << 4));
                            const uint4 v = t < w.len ? *p : make_uint4(0, 0, 0, 0);
                            uint32_t word[4] = {v.x, v.y, v.z, v.w};
                            bool odd = false;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((word[e] & 0x7f80u) == 0x7f80u) { word[e] &= 0xffff0000u; odd = true; }
                                if ((word[e] & 0x7f800000u) == 0x7f800000u) { word[e] &= 0xffffu; odd = true; }
                            }
                            if (odd) atomicOr(&sm.bad, 1ull << (t - w.committed));
                            if (odd || t >= w.len) *p = make_uint4(word[0], word[1], word[2], word[3]);
                        }
                    }
                }
                fence_proxy_async_smem();
            }
        }
        alive = warp_wait(&sm.s_full, j & 1, gave_up);
        if (!alive) break;
        if (warp_live) {
            tc_fence_after_sync();
            uint32_t see[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (ends)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    see[c] = w.committed + node >= 0 ? seen_columns(t0 + 32 * c, w.committed, w.len, sees) : 0u;
            float mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t s[32];
                tmem_ld32(t_s + 32 * c, s);
                tmem_ld_wait();
                if (ends)
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        if (!((see[c] >> x) & 1)) s[x] = 0xff800000u;
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, mx};
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    m4[x & 3] = fmax3(m4[x & 3], __uint_as_float(s[2 * x]), __uint_as_float(s[2 * x + 1]));
                mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            }
            if (j == 0) {
                m_ref = mx;
            } else {
                const bool need = live && (mx - m_ref) * unit > kRescaleAt;
                if (__any_sync(0xffffffffu, need)) {
                    // all MMAs issued before these scores, O's last among them, have completed
                    const float alpha = need ? fast_exp2((m_ref - mx) * unit) : 1.f;
                    if (need) m_ref = mx;
                    l_sum *= alpha;
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(t_o + 32 * c, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                        tmem_st32(t_o + 32 * c, o);
                    }
                }
            }
            const float base = m_ref == -INFINITY ? 0.f : m_ref * unit;  // (nothing seen yet)
            float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t s[32], pk[16];
                tmem_ld32(t_s + 32 * c, s);
                tmem_ld_wait();
                if (ends)
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        if (!((see[c] >> x) & 1)) s[x] = 0xff800000u;
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const float p0 = fast_exp2(fmaf(__uint_as_float(s[2 * x]), unit, -base));
                    const float p1 = fast_exp2(fmaf(__uint_as_float(s[2 * x + 1]), unit, -base));
                    l4[2 * (x & 1)] += p0;
                    l4[2 * (x & 1) + 1] += p1;
                    pk[x] = F4 ? f16x2(p0, p1) : bf16x2(p0, p1);
                }
                tmem_st16(t_s + 16 * c, pk);  // over columns that have been read
            }
            l_sum += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            tmem_st_wait();
        }
        tc_fence_before_sync();
        mbar_arrive(&sm.p_full);
    }

    // ---- the row's result
    if (alive && w.tiles > 0) alive = warp_wait(&sm.o_full, 0, gave_up);
    asm volatile("bar.sync 1, 128;" ::: "memory");  // `bad` is complete
    if (!alive || !warp_live) return;
    tc_fence_after_sync();
    const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;
    const float base = m_ref == -INFINITY ? 0.f : m_ref * unit;
    unsigned long long odd = l_sum == 0.f ? 0 : sm.bad & sees;
    const int32_t* pages = a.kv.page_table + (int64_t)w.r * a.kv.max_pages;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        if (w.tiles > 0) {
            tmem_ld32(t_o + 32 * c, o);
            tmem_ld_wait();
        }
        float x[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = l_sum == 0.f ? 0.f : __uint_as_float(o[e]) * inv;
        for (unsigned long long left = odd; left != 0; left &= left - 1) {  // values that were taken out
            const int t = w.committed + __ffsll(left) - 1, in = t & ((1 << a.kv.page_shift) - 1);
            const int64_t page = paged_page(a.kv, pages, t >> a.kv.page_shift);
            if constexpr (F4) {
                using B = Fp4Block<D>;
                const uint8_t* b = a.kv.k + (((page * a.Hkv + w.h) << (a.kv.page_shift - 4)) + (in >> 4)) * B::kBytes;
                const uint32_t sc = *reinterpret_cast<const uint16_t*>(b + B::v_scale(in & 15, c));
                if ((sc & 0x7fffu) <= 0x7154u) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t f[4];
                    e2m1x8_to_f16x2(*reinterpret_cast<const uint32_t*>(b + B::v_byte(in & 15, 32 * c + 8 * e)), f);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t v = hmul2(f[y], sc * 0x10001u);
                        x[8 * e + 2 * y] += __half2float(__ushort_as_half((unsigned short)v));
                        x[8 * e + 2 * y + 1] += __half2float(__ushort_as_half((unsigned short)(v >> 16)));
                    }
                }
            } else {
                const uint16_t* v = reinterpret_cast<const uint16_t*>(a.kv.v) +
                                    (((page << a.kv.page_shift) + in) * a.Hkv + w.h) * D + 32 * c;
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if ((v[e] & 0x7f80u) == 0x7f80u) x[e] += __uint_as_float((uint32_t)v[e] << 16);
            }
        }
        if (!live) continue;
        if (a.out != nullptr) {
            uint4* to = reinterpret_cast<uint4*>(a.out + row * D + 32 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                to[e] = make_uint4(bf16x2(x[8 * e], x[8 * e + 1]), bf16x2(x[8 * e + 2], x[8 * e + 3]),
                                   bf16x2(x[8 * e + 4], x[8 * e + 5]), bf16x2(x[8 * e + 6], x[8 * e + 7]));
        } else {
            float4* to = reinterpret_cast<float4*>(a.o_part + slot * D + 32 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
        }
    }
    if (!live) return;
    const float lse = l_sum == 0.f ? -INFINITY : base * kLn2 + logf(l_sum);
    if (a.out == nullptr) a.lse_part[slot] = lse;
    else if (a.lse_out != nullptr) a.lse_out[row] = lse;
}

template <int D, bool F4>
__device__ __forceinline__ void load_role(Smem<D, F4>& sm, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const TreeArgs& a,
                                          const Work& w, int lane)
{
    using C = Cfg<D, F4>;
    const int32_t* pages = a.kv.page_table + (int64_t)w.r * a.kv.max_pages;
    const int shift = a.kv.page_shift;
    const int end = w.len;
    if constexpr (!F4) {
        const int box = min(kTile, 1 << shift);  // tokens of a copy; lane b < kTile / box copies the b-th of a tile
        const int boxes = kTile / box;
        auto page_of = [&](int j) {
            const int t = (w.tile0 + j) * kTile + lane * box;
            return lane < boxes && j < w.tiles && t < end ? paged_page(a.kv, pages, t >> shift) : -1;
        };
        int next = page_of(0), seq = 0;
        bool ok = true;
        for (int j = 0; j < w.tiles && ok; ++j) {
            const int page = next;
            next = page_of(j + 1);
            const int t = (w.tile0 + j) * kTile + lane * box;
            const int there = __popc(__ballot_sync(0xffffffffu, page >= 0));
            const int z = (page << shift) + (t & ((1 << shift) - 1));
#pragma unroll
            for (int x = 0; x < 2 * C::kHalves; ++x, ++seq) {
                const int s = seq % C::kSlots;
                if (seq >= C::kSlots) ok = warp_wait(&sm.empty[s], ((seq / C::kSlots) - 1) & 1, &sm.gave_up);
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(&sm.full[s], there * box * 128);
                __syncwarp();
                if (page >= 0)
                    tma_load_3d(sm.slot[s] + lane * box * 128, x < C::kHalves ? &tm_k : &tm_v, 64 * (x % C::kHalves), w.h, z,
                                &sm.full[s]);
            }
        }
        if (*static_cast<volatile int*>(&sm.gave_up))  // the copies in flight end before the CTA leaves (each wait again has a limit)
            for (int x = max(0, seq - C::kSlots); x < seq; ++x) {
                int never = 0;
                mbar_wait(&sm.full[x % C::kSlots], (x / C::kSlots) & 1, &never);
            }
    } else {
        using B = Fp4Block<D>;
        // units: keys of tokens 0 .. 63 of a tile, of 64 .. 127, then the values; lane 2 b + c copies block b's codes
        // (c = 0) or scales (c = 1)
        const int b = lane >> 1, c = lane & 1;
        const int64_t page_bytes = ((int64_t)a.Hkv << (shift - 4)) * B::kBytes;
        const uint8_t* pool = a.kv.k + ((int64_t)w.h << (shift - 4)) * B::kBytes;
        auto page_of = [&](int j, int half) {
            const int t = (w.tile0 + j) * kTile + 64 * half + 16 * b;
            return lane < 2 * C::kUnitBlocks && j < w.tiles && t < end ? paged_page(a.kv, pages, t >> shift) : -1;
        };
        int next[2] = {page_of(0, 0), page_of(0, 1)}, seq = 0;
        bool ok = true;
        for (int j = 0; j < w.tiles && ok; ++j) {
            const int page[2] = {next[0], next[1]};
            next[0] = page_of(j + 1, 0);
            next[1] = page_of(j + 1, 1);
#pragma unroll
            for (int x = 0; x < 4; ++x, ++seq) {
                const int half = x & 1;
                const bool value = x >= 2;
                const int u = seq % C::kUnits;
                if (seq >= C::kUnits) ok = warp_wait(&sm.unit_empty[u], ((seq / C::kUnits) - 1) & 1, &sm.gave_up);
                if (!ok) break;
                const int there = __popc(__ballot_sync(0xffffffffu, page[half] >= 0)) / 2;
                if (lane == 0) mbar_arrive_expect_tx(&sm.unit_full[u], there * C::kPartBytes);
                __syncwarp();
                if (page[half] >= 0) {
                    const int t = (w.tile0 + j) * kTile + 64 * half + 16 * b;
                    const int block = (t & ((1 << shift) - 1)) >> 4;
                    const uint8_t* from = pool + page[half] * page_bytes + (int64_t)block * B::kBytes;
                    from += c == 0 ? (value ? B::kV : 0) : (value ? B::kVScale : B::kKScale);
                    bulk_load(sm.unit + u * C::kUnitBytes + b * C::kPartBytes + (c == 0 ? 0 : 8 * D), from, c == 0 ? 8 * D : D,
                              &sm.unit_full[u]);
                }
            }
        }
        if (*static_cast<volatile int*>(&sm.gave_up))
            for (int x = max(0, seq - C::kUnits); x < seq; ++x) {
                int never = 0;
                mbar_wait(&sm.unit_full[x % C::kUnits], (x / C::kUnits) & 1, &never);
            }
    }
}

template <int D, bool F4>
__device__ __forceinline__ void mma_role(Smem<D, F4>& sm, const Work& w, uint32_t tmem)
{
    using C = Cfg<D, F4>;
    constexpr int H = C::kHalves;
    const uint32_t id_qk = F4 ? idesc_f16_f32(128, kTile, false) : idesc_bf16_f32(128, kTile, false);
    const uint32_t id_pv = F4 ? idesc_f16_f32(128, 64, true) : idesc_bf16_f32(128, 64, true);
    const uint64_t d_k = smem_desc_sw128(0, 16, 1024), d_n = smem_desc_sw128(0, kSlotBytes, 1024);
    const uint32_t hi_k = static_cast<uint32_t>(d_k >> 32), hi_n = static_cast<uint32_t>(d_n >> 32);
    const uint32_t lo_q = static_cast<uint32_t>(d_k) + (smem_u32(sm.q[0]) >> 4);
    const uint32_t lo_k = static_cast<uint32_t>(d_k) + (smem_u32(sm.slot[0]) >> 4);
    const uint32_t lo_v = static_cast<uint32_t>(d_n) + (smem_u32(sm.slot[0]) >> 4);
    auto desc = [](uint32_t hi, uint32_t lo) { return (static_cast<uint64_t>(hi) << 32) | lo; };
    int* gave_up = &sm.gave_up;
    auto scores = [&](int j) {
#pragma unroll
        for (int hv = 0; hv < H; ++hv) {
            const int seq = j * 2 * H + hv, s = seq % C::kSlots;
            if (!mbar_wait(&sm.full[s], (seq / C::kSlots) & 1, gave_up)) return false;
            tc_fence_after_sync();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                mma_ss(tmem, desc(hi_k, lo_q + ((hv * kSlotBytes + ks * 32) >> 4)), desc(hi_k, lo_k + ((s * kSlotBytes + ks * 32) >> 4)),
                       id_qk, hv > 0 || ks > 0);
            tc_commit(&sm.empty[s]);
        }
        tc_commit(&sm.s_full);
        return true;
    };
    bool ok = mbar_wait(&sm.q_full, 0, gave_up) && scores(0);
    for (int j = 0; j < w.tiles && ok; ++j) {
        ok = mbar_wait(&sm.p_full, j & 1, gave_up);
#pragma unroll
        for (int hv = 0; hv < H && ok; ++hv) {
            const int seq = j * 2 * H + H + hv, s = seq % C::kSlots;
            ok = mbar_wait(&sm.full[s], (seq / C::kSlots) & 1, gave_up);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int ks = 0; ks < kTile / 16; ++ks)
                mma_ts(tmem + kTile + 64 * hv, tmem + 8 * ks, desc(hi_n, lo_v + ((s * kSlotBytes + ks * 2048) >> 4)), id_pv,
                       j > 0 || ks > 0);
            tc_commit(&sm.empty[s]);
        }
        if (!ok) break;
        if (j + 1 < w.tiles) ok = scores(j + 1);
        else tc_commit(&sm.o_full);
    }
}

// Codes of one block (a warp) of every unit -> f16 operand rows in the slots.
template <int D>
__device__ __forceinline__ void widen_role(Smem<D, true>& sm, const Work& w, int block, int lane)
{
    using C = Cfg<D, true>;
    constexpr int H = C::kHalves, J = D / 32;
    int* gave_up = &sm.gave_up;
    int unit = 0, seq = 0;
    bool ok = true;
    for (int j = 0; j < w.tiles && ok; ++j) {
        const int t0 = (w.tile0 + j) * kTile;
        const bool ends = t0 + kTile > w.committed;
#pragma unroll 1
        for (int kind = 0; kind < 2 && ok; ++kind, seq += H) {
            uint8_t* to[H];
#pragma unroll
            for (int hv = 0; hv < H; ++hv) {
                const int s = (seq + hv) % C::kSlots;
                to[hv] = sm.slot[s];
                if (seq + hv >= C::kSlots) ok = ok && warp_wait(&sm.empty[s], (((seq + hv) / C::kSlots) - 1) & 1, gave_up);
            }
#pragma unroll 1
            for (int half = 0; half < 2 && ok; ++half, ++unit) {
                ok = warp_wait(&sm.unit_full[unit % C::kUnits], (unit / C::kUnits) & 1, gave_up);
                if (!ok) break;
                const uint8_t* from = sm.unit + (unit % C::kUnits) * C::kUnitBytes + block * C::kPartBytes;
                const int row0 = 64 * half + 16 * block;
                if (kind == 0) {
                    // Keys: the D / 8 bytes of (token, c) are dimensions 32 g + 8 c .. + 7 for each group g.  Eight lanes that
                    // go to memory together have tokens x and x ^ 5: their loads and their swizzled stores both fall on
                    // eight different 16-byte pieces of the banks.
#pragma unroll
                    for (int it = 0; it < 2; ++it) {
                        const int l = lane & 7, c = l & 3, qd = lane >> 3, t = 8 * it + ((l >> 2) ? (qd ^ 5) : qd);
                        uint32_t code[J], sc[J / 2];
                        if constexpr (J == 4) {
                            const uint4 x = *reinterpret_cast<const uint4*>(from + t * (D / 2) + c * (D / 8));
                            code[0] = x.x; code[1] = x.y; code[2] = x.z; code[3] = x.w;
                            const uint2 y = *reinterpret_cast<const uint2*>(from + 8 * D + 2 * t * J);
                            sc[0] = y.x; sc[1] = y.y;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2*>(from + t * (D / 2) + c * (D / 8));
                            code[0] = x.x; code[1] = x.y;
                            sc[0] = *reinterpret_cast<const uint32_t*>(from + 8 * D + 2 * t * J);
                        }
                        const int row = row0 + t;
#pragma unroll
                        for (int g = 0; g < J; ++g) {
                            uint32_t f[4];
                            e2m1x8_to_f16x2(code[g], f);
                            const uint32_t s2 = __byte_perm(sc[g >> 1], 0, (g & 1) ? 0x3232 : 0x1010);
                            *reinterpret_cast<uint4*>(to[g >> 1] + row * 128 + (((4 * (g & 1) + c) ^ (row & 7)) << 4)) =
                                make_uint4(hmul2(f[0], s2), hmul2(f[1], s2), hmul2(f[2], s2), hmul2(f[3], s2));
                        }
                    }
                } else {
                    // Values: chunk x (D / 8 dimensions) of a pair of tokens, first token's bytes, then the second's
#pragma unroll
                    for (int it = 0; it < 2; ++it) {
                        const int x = lane & 7, p = 4 * it + (lane >> 3);
                        constexpr int W = D / 64;  // words of a token's chunk
                        uint32_t code[2 * W];
                        const uint8_t* at = from + p * D + (x ^ Fp4Block<D>::v_swap(p)) * (D / 8);
                        if constexpr (W == 2) {
                            const uint4 y = *reinterpret_cast<const uint4*>(at);
                            code[0] = y.x; code[1] = y.y; code[2] = y.z; code[3] = y.w;
                        } else {
                            const uint2 y = *reinterpret_cast<const uint2*>(at);
                            code[0] = y.x; code[1] = y.y;
                        }
                        uint32_t sc = *reinterpret_cast<const uint32_t*>(from + 8 * D + 2 * ((x * (D / 8) / 32) * 16 + 2 * p));
#pragma unroll
                        for (int tok = 0; tok < 2; ++tok) {
                            const int row = row0 + 2 * p + tok, t = t0 + row;
                            uint32_t s1 = tok == 0 ? sc & 0xffffu : sc >> 16;
                            if (ends && t >= w.committed) {
                                if (t >= w.len) {
                                    s1 = 0;
                                } else if ((s1 & 0x7fffu) > 0x7154u) {  // above what appends write, infinities and NaN included
                                    atomicOr(&sm.bad, 1ull << (t - w.committed));
                                    s1 = 0;
                                }
                            }
                            const uint32_t s2 = s1 * 0x10001u;
                            uint4 v[W];
#pragma unroll
                            for (int y = 0; y < W; ++y) {
                                uint32_t f[4];
                                e2m1x8_to_f16x2(code[tok * W + y], f);
                                v[y] = make_uint4(hmul2(f[0], s2), hmul2(f[1], s2), hmul2(f[2], s2), hmul2(f[3], s2));
                            }
                            if constexpr (W == 2) {
                                // (lanes of the other half store their pieces the other way round: different banks)
                                const int first = x >> 2, piece = 2 * (x & 3);
                                uint8_t* base = (first ? to[H - 1] : to[0]) + row * 128;
                                *reinterpret_cast<uint4*>(base + (((piece + first) ^ (row & 7)) << 4)) = first ? v[W - 1] : v[0];
                                *reinterpret_cast<uint4*>(base + (((piece + 1 - first) ^ (row & 7)) << 4)) = first ? v[0] : v[W - 1];
                            } else {
                                *reinterpret_cast<uint4*>(to[0] + row * 128 + ((x ^ (row & 7)) << 4)) = v[0];
                            }
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.unit_empty[unit % C::kUnits]);
            }
            if (!ok) break;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0)
                for (int hv = 0; hv < H; ++hv) mbar_arrive(&sm.full[(seq + hv) % C::kSlots]);
        }
    }
}

template <int D, bool F4>
__global__ void __launch_bounds__(Cfg<D, F4>::kThreads, 2)
tree_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const TreeArgs a)
{
    using C = Cfg<D, F4>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem<D, F4>& sm = *reinterpret_cast<Smem<D, F4>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    dependents_may_launch();
    if ((smem_u32(smem_raw) & 1023u) != 0) {  // (operand tiles lie on 1024-byte boundaries)
        if (tid == 0) atomicMin(a.kv.status, (int)MOSKA_ERR_CUDA);
        return;
    }
    const Work w = work_of(a);
    if (w.rows <= 0) return;
    if (tid == 0) {
        for (int s = 0; s < C::kSlots; ++s) {
            mbar_init(&sm.full[s], F4 ? 4 : 1);  // 4 bits: one arrival per widening warp
            mbar_init(&sm.empty[s], 1);
        }
        if constexpr (F4)
            for (int u = 0; u < C::kUnits; ++u) {
                mbar_init(&sm.unit_full[u], 1);
                mbar_init(&sm.unit_empty[u], 4);
            }
        mbar_init(&sm.q_full, 128);
        mbar_init(&sm.s_full, 1);
        mbar_init(&sm.p_full, 128);
        mbar_init(&sm.o_full, 1);
        sm.bad = 0;
        sm.gave_up = 0;
        fence_mbar_init();
        fence_proxy_async_smem();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&sm.tmem_base, 256);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sm.tmem_base;

    if (warp < 4) {
        softmax_role<D, F4>(sm, a, w, tmem, warp, lane);
    } else if (warp == kLoadWarp) {
        load_role<D, F4>(sm, tm_k, tm_v, a, w, lane);
    } else if (warp == kMmaWarp) {
        if (lane == 0 && w.tiles > 0) mma_role<D, F4>(sm, w, tmem);
        __syncwarp();
    } else {
        if constexpr (F4) widen_role<D>(sm, w, warp - kWidenWarp0, lane);
    }

    tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 256);
    if (tid == 0 && sm.gave_up) atomicMin(a.kv.status, (int)MOSKA_ERR_TIMEOUT);
}

// ---- host side ------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up through the runtime (no link against libcuda).
int encoder(EncodeTiledFn* out)
{
    static EncodeTiledFn fn = nullptr;
    static std::mutex mtx;
    std::lock_guard<std::mutex> lock(mtx);
    if (fn == nullptr) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult res;
        MOSKA_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &res));
        if (sym == nullptr || res != cudaDriverEntryPointSuccess)
            return fail(MOSKA_ERR_CUDA, "the driver does not provide cuTensorMapEncodeTiled");
        fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    *out = fn;
    return MOSKA_OK;
}

// Pages as [tokens][Hkv][D]: boxes of 64 dimensions of one head, a page's tokens or 128 of them.
int make_page_map(CUtensorMap* tm, const void* pool, const PagedView& kv, int Hkv, int D)
{
    EncodeTiledFn enc = nullptr;
    MOSKA_TRY_STATUS(encoder(&enc));
    const int page = 1 << kv.page_shift;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)Hkv, (cuuint64_t)kv.n_pages << kv.page_shift};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)Hkv * D * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)(page < kTile ? page : kTile)};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(pool), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(MOSKA_ERR_CUDA, "cuTensorMapEncodeTiled failed for pages (%d)", (int)r);
    return MOSKA_OK;
}

}  // namespace

int default_tree_splits(bool, int n_requests, int nodes, int G, int Hkv, int, int max_len)
{
    // as many CTAs as there are places, two tiles at least
    const long long row_tiles = (nodes + kTileRows / G - 1) / (kTileRows / G);
    long long s = 296 / (n_requests * Hkv * row_tiles);
    const long long cap = ((long long)max_len + 2 * kTile - 1) / (2 * kTile);
    if (s > cap) s = cap;
    return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

int launch_tree_attn(const uint16_t* q, const PagedView& kv, bool fp4, const TreeRows& tree, float* o_part, float* lse_part,
                     int slot0, int n_slots, uint16_t* out, float* lse_out, float scale, const moska_shape* s,
                     cudaStream_t st)
{
    if (tree.n_rows == 0) return MOSKA_OK;
    const int G = s->Hq / s->Hkv, per_tile = kTileRows / G, row_tiles = (tree.max_nodes + per_tile - 1) / per_tile;
    const long long grid = (long long)tree.n_requests * s->Hkv * s->n_unique_splits * row_tiles;
    if (grid > 0x7fffffffLL) return fail(MOSKA_ERR_UNSUPPORTED, "tree attention grid too large");
    if (((long long)kv.n_pages << kv.page_shift) > 0x7fffffffLL)
        return fail(MOSKA_ERR_UNSUPPORTED, "a pool of more than 2^31 tokens");
    const TreeArgs a{q, kv, tree, o_part, lse_part, out, lse_out, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0, n_slots,
                     row_tiles, per_tile};
    CUtensorMap tm_k{}, tm_v{};
    if (!fp4) {
        MOSKA_TRY_STATUS(make_page_map(&tm_k, kv.k, kv, s->Hkv, s->D));
        MOSKA_TRY_STATUS(make_page_map(&tm_v, kv.v, kv, s->Hkv, s->D));
    }
    auto go = [&](auto kernel, int threads, int smem) {
        MOSKA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        kernel<<<(unsigned)grid, threads, smem, st>>>(tm_k, tm_v, a);
        MOSKA_LAUNCH_CHECK("tree_attn_kernel");
        return (int)MOSKA_OK;
    };
    auto form = [&](auto d, auto f4) {
        constexpr int D = decltype(d)::value;
        constexpr bool F4 = decltype(f4)::value;
        return go(tree_attn_kernel<D, F4>, Cfg<D, F4>::kThreads, (int)sizeof(Smem<D, F4>));
    };
    const std::integral_constant<int, 128> d128;
    const std::integral_constant<int, 64> d64;
    if (s->D == 128) return fp4 ? form(d128, std::true_type{}) : form(d128, std::false_type{});
    return fp4 ? form(d64, std::true_type{}) : form(d64, std::false_type{});
}

}  // namespace moska
