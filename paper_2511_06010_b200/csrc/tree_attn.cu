// Attention of the nodes of drafted trees over the paged contexts that they end, on the 5th-generation tensor cores.
//
// The T G query rows of a request's KV head (T nodes, G heads each) share one context.  Work comes in units: up to 128 of
// these rows (whole nodes) and the context in tiles of 128 tokens:
//   S = Q K^T          tcgen05.mma, Q in tensor memory, K in shared memory: 128 x 64 scores (half a tile) in tensor memory
//   P = exp2(S - m)    a thread per row: TMEM -> registers -> 16 bits, back over the columns of S
//   O += P V           tcgen05.mma, P from TMEM, V from shared memory
// Two groups of softmax warps take turns at the halves: while one has the special function units (512 cycles of exponentials a
// half), the other reads its scores, finds their maxima and stores.  Scores have four buffers, so that products run ahead.  A
// third group stages the next unit's queries and writes the last unit's rows.  TMEM: O 128, S 4 x 64, Q 2 x 64 = 512 columns.
//
// What bounds it.  A tile of 128 rows and 128 tokens is 1024 cycles of MMA (D = 128), as many of exponentials, and in 4 bits
// some 1800 cycles of shared memory (operands written, and read by the MMAs) and 512 more of MMA.  A half takes a group about 1900 cycles from
// scores to probabilities, of which 900 are exponentials that the other group's slow down, so a tile takes 1900 cycles instead of
// 1024.  Times in long runs, at the clock that the power cap leaves: bf16, 24 requests of 60 nodes and 1K-16K tokens 0.52 ms, 0.79
// PFLOP/s (one launch alone 0.44 ms, tensor pipe 52 % busy).  Up to 64 rows bf16 waits for memory (64 requests of 16 nodes and
// 4096 tokens: 202 us, 5.4 TB/s; alone 181).  4 bits, 32 requests of 64 nodes and 1K-8K tokens: 526 us (488), 3300 cycles a tile:
// its keys wait for the product before (their second operand has one buffer), and issue slots are 63 % full.  One request of
// 8 nodes and 1000 tokens: 17 us, of which 3.7 find the part, 1.3 bring the queries, 3 are the tile, 1.2 its rows, and the
// rest the two launches.
// Not kept (short runs): a third softmax group (bf16 471 us for 437: registers), products of 128 tokens (one MMA warp waits for
// the other's operands), the next scores read between a step's exponentials (468 for 434), part of the exponentials as
// polynomials (all of them left out saves 10 %).
//
// One CTA per SM.  For each row tile (first 128 rows of every request, second 128, ..) the tiles of all its units, request after
// request and head after head, form a line.  Lines get CTAs by their lengths and are cut into equal parts, one per CTA,
// whatever the contexts' lengths: a CTA walks the units in its part.  A unit that a cut divides leaves partial rows, which a
// second kernel joins.  (With trees of one size the lines are alike and their CTAs walk the same contexts at the same time, so
// that all but the first find them in L2; cut as one line, each fetched them from memory: 24 requests of 60 nodes
// read 3.45 GB instead of 0.9.)
//
// Warps, in this order: groups of four for the softmax (thread i: row i % 128 = TMEM lane), four for queries and results, one for
// copies, one for the MMAs of Q K^T and one for those of P V (one warp for both left the tensor cores idle while it waited).  4-bit
// pages: twelve that widen.  Operands lie in a ring of slots, a K or a V tile each, as halves of 64 dimensions in rows of
// 128 bytes with the 128-byte swizzle.
//   bf16: one TMA box of min(page_size, 128) tokens a page and half.
//   4 bits: a bulk copy a page into a ring of tiles of codes, which are widened to operands, code times scale.  Values: f16 (half
//   a step, 2^-11).  Keys: two bf16 operands, code times the scale's upper 6 bits and code times the rest of it, exact
//   for every finite scale, and bf16 queries as they are, so that scores are exact but for their sums.  (With a key as one
//   f16 operand lse was off by 2e-6 relative in contexts of 4096 tokens, 1e-5 in short ones; two f16 ones, the product and
//   what is left of it, are 14 instructions less for 8 codes, 205 us for 64 requests of 8 nodes instead of 214 and 511 for 32
//   of 64 instead of 558, but give inf - inf above a scale of 10912 and steps of 2^-24.)  Rows of queries are scaled
//   by a power of two.
//
// What a node sees: committed tokens, and of the last T tokens those whose bit is set in its 64-bit word of ancestors.
// Only tiles that reach past the committed tokens look at it.  0 times NaN is NaN, so values of such tiles that are
// not finite are taken out of the operands (a bit per token remembers), and put into the rows that see them at the end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <type_traits>

#include "sm100.cuh"
#include "tensor_map.cuh"
#include "tree.cuh"

namespace moska {
namespace {
using namespace sm100;

constexpr int kTile = 128;      // tokens of a tile
constexpr int kStep = 64;       // tokens whose scores are computed at once
constexpr int kTileRows = 128;  // query rows of a unit
constexpr int kHalfBytes = kTile * 64 * 2;
constexpr int kFindThreads = 256;  // of those that find a CTA's part
constexpr int kMaxRowTiles = 4;  // 64 nodes of up to 8 heads
constexpr int kMaxCtas = 148;    // parts of the line of tiles
constexpr uint32_t kColO = 0, kColS = 128, kColQ = 384;  // tensor-memory columns
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kStagePitch = 144;  // 128 bytes and 16: a row's pieces and a piece's rows both fall on different banks
constexpr float kRescaleAt = 8.f;  // log2 units that a row's maximum may grow before its sums are rescaled
// 4 bits: log2 of P at a row's reference, so that P is at most 2^15.  f16 ends in steps of 2^-24: with P = 1 at the reference,
// many tokens of less than 2^-25 each beside one that holds most of a row's weight (3 % of a row of a million tokens) would
// count in its sum and not in its result.  So they are held down to 2^-32 of the row's largest, as in moska_unique_attn_paged.
constexpr float kBelowF16 = 7.f;

template <int D, bool F4>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kGroups = 2;  // of softmax warps
    static constexpr int kRowWarp0 = 4 * kGroups, kLoadWarp = kRowWarp0 + 4, kScoreWarp = kLoadWarp + 1, kValueWarp = kLoadWarp + 2,
                         kWidenWarp0 = kLoadWarp + 4, kKeyWarps = 8, kValueWarps = 4, kWidenWarps = kKeyWarps + kValueWarps;
    static constexpr int kThreads = 32 * (F4 ? kWidenWarp0 + kWidenWarps : kWidenWarp0);
    // Registers of a thread: at the launch, and of the groups of four warps after it.
    static constexpr int kLaunchRegs = F4 ? 72 : 128;
    static constexpr int kSoftmaxRegs = F4 ? 112 : 152, kRowRegs = F4 ? 96 : 128, kIssueRegs = F4 ? 40 : 80, kWidenRegs = 48;
    static_assert(128 * (kGroups * kSoftmaxRegs + kRowRegs + kIssueRegs + (F4 ? kWidenWarps / 4 * kWidenRegs : 0)) <= kThreads * kLaunchRegs,
                  "setmaxnreg: more than the CTA was launched with would be waited for without end");
    static constexpr int kSlotBytes = kHalves * kHalfBytes;
    static constexpr int kSlots = F4 ? (D == 128 ? 4 : 8) : (D == 128 ? 6 : 12);
    static constexpr int kBlocks = kTile / kBlockTokens;  // 16-token blocks of a tile
    static constexpr int kCodeBytes = kBlocks * fp4_block_bytes(D);
    static constexpr int kCodeSlots = F4 ? (D == 128 ? 2 : 6) : 1;
};

// Units of few rows have each row P times, in lanes kTileRows / P apart: the i-th has the i-th part of every step's tokens, with a
// reference, a sum and an O of its own, as if a context were cut into P.  The four warps of a group have a P-th of the
// scores each then, where one warp of live rows would have had them all (4 bits, 64 requests of 4096 tokens: 32 rows 214 us with
// P = 4, 216 with 2, 239 without; with D = 64 74 and 76; 64 rows 232 with 2, 256 without.  bf16 waits for memory there, 182,
// 182, 183 us and 190, 192; it has P = 1 alone).
template <int P>
struct Spread {
    static constexpr int kRows = kTileRows / P, kCols = kStep / P;
};

// Tiles of request r's context (an empty one counts as one, so that its rows are written) and its row tiles.
struct Request {
    int first, nodes, len, tiles, row_tiles;
};
// A CTA's part of the line of its row tile.
struct Part {
    long long p0, p1, per;  // tiles p0 .. p1 - 1; `per` in a full part
    long long start;        // first tile of the unit that p0 is in: (row tile, request, head)
    int rt, r, h;
    Request q;
    int cta0;               // the line's first CTA
    int cost;               // of a unit, in tiles
    int longest[kFindThreads / 32];
    long long sums[kMaxRowTiles][kFindThreads / 32];  // of each warp's requests
};

// A unit that cuts divide, for the kernel that joins its rows: its first node's batch row, its KV head, rows (0: none) and the
// CTAs of its parts.
struct __align__(16) CutUnit {
    int first, h, rows, c0, c1, unused[3];
};

// What the softmax needs of a unit.
struct UnitInfo {
    int committed, len, tile0, tiles, rows, more;
};

template <int D, bool F4>
struct Smem {
    using C = Cfg<D, F4>;
    uint8_t slot[C::kSlots][C::kSlotBytes];
    uint8_t rest[F4 ? C::kSlotBytes : 1024];  // one tile's second operand of keys
    uint8_t code[F4 ? C::kCodeSlots * C::kCodeBytes : 16];
    float ref[C::kGroups][kTileRows];       // the reference of a row's probabilities after a step of each softmax group
    float2 stat[2][C::kGroups][kTileRows];  // (reference, sum) of a unit's rows by each group; units take turns
    UnitInfo info[2];                // units take turns
    unsigned long long sees[2][kTileRows];
    float row_unit[2][kTileRows];
    uint8_t stage[4][32][kStagePitch];  // pieces of 128 bytes of each warp's rows, on their way to and from global memory
    void* row_to[4][32];                // where the rows of a unit go
    TreeSmem tree;
    uint64_t full[C::kSlots], empty[C::kSlots];
    uint64_t code_full[C::kCodeSlots], code_empty[C::kCodeSlots];
    uint64_t q_full[2], s_full[4], p_full[4], stat_full[2], ref_full[C::kGroups][4], pv_done[4], o_full, o_free;
    uint64_t rest_empty[2], key_full[C::kSlots][2];  // (4 bits: halves of a tile of keys)
    unsigned long long bad[8];  // tree tokens with values that are not finite; units take turns
    Part part;
    uint32_t tmem_base;
    uint32_t step;  // that the first softmax group is at
    int gave_up;
};
constexpr int kMostSmem = 232448;
static_assert(sizeof(Smem<128, false>) <= kMostSmem && sizeof(Smem<128, true>) <= kMostSmem &&
                  sizeof(Smem<64, false>) <= kMostSmem && sizeof(Smem<64, true>) <= kMostSmem,
              "an SM's shared memory");

struct TreeArgs {
    const uint16_t* q;
    PagedView kv;
    TreeRows tree;
    float* o_part;  // partial slots of the rows (nullptr: `out` gets the final rows)
    float* lse_part;
    uint16_t* out;
    float* lse_out;
    float* o_cut;   // partial rows of units that a cut divides [CTA][2][128][D] (final rows only)
    float* lse_cut;
    CutUnit* cut;   // [CTA]: the unit whose second part is the CTA's first
    float scale;
    int Hq, Hkv, n_splits, slot0, n_slots;
    int row_tiles;       // of the largest tree
    int nodes_per_tile;  // 128 / G
};

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

__device__ __forceinline__ uint32_t bmul2(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
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

// The same for the end of a unit, whose steps may be many: the limit of a wait begins anew when `step` moves (2^29 tokens in one
// part take 5 s).
__device__ __forceinline__ bool unit_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* step, volatile int* gave_up)
{
    bool ok = false;
    uint64_t since = 0;
    uint32_t seen = 0;
    for (uint32_t polls = 1; !ok; ++polls) {
        ok = mbar_try_wait(bar, parity);
        if (ok || (polls & 1023u) != 0) continue;
        if (*gave_up) break;
        const uint64_t now = global_timer_ns();
        const uint32_t at = *step;
        if (since == 0 || at != seen) {
            since = now;
            seen = at;
        } else if (now - since > kWaitLimitNs) {
            *gave_up = 1;
            break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void find_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// Of the third group; true if all of its threads say so.  (No thread leaves on its own: the others would wait for it.)
__device__ __forceinline__ bool row_barrier(bool ok = true)
{
    uint32_t all;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "barrier.cta.red.and.pred q, 2, 128, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(all)
        : "r"(ok ? 1u : 0u)
        : "memory");
    return all != 0;
}

// True in one lane of the calling warp (converged).  With it, and loops that the whole warp runs, descriptors stay in
// uniform registers: under `lane == 0` an MMA took about 90 cycles to issue.
__device__ __forceinline__ bool elect_one()
{
    uint32_t yes;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(yes));
    return yes != 0;
}

// ---- the line of tiles ------------------------------------------------------------------------------
// On the line a unit is longer than its tiles by what its beginning and its end cost, in tiles (bf16 24 requests of 60 nodes 554 us
// with 0, 545 with 1, 529 with 2, 525 with 4; 4 bits 32 of 64 nodes 597, 578, 571, 580; bf16 100 of 5-33 nodes, D = 64, 75, 76, 76,
// 78); where parts would be shorter than kShortPart by nothing, as they would be longer for it then (bf16 requests of 8 nodes and
// 4000 tokens, always counted and from 2, 4, 8 and 16 tiles on: one 20.9, 22.5 us, two 23.3, 23.3, 22.9, 22.6, 22.7, four 28.6, 28.7, 28.7,
// 29.5, 29.7, eight 39.5, 39.4, 39.5, 39.4, 40.6).
constexpr int kUnitCost = 2, kShortPart = 4;
// Tiles and units of a stretch of requests in one number.
constexpr int kUnitBit = 40;
// (64-bit divisions are long: 32 bits where they do)
__device__ __forceinline__ long long divide(long long a, long long b)
{
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ long long places(long long packed, int cost)
{
    return (packed & ((1ll << kUnitBit) - 1)) + (packed >> kUnitBit) * cost;
}

__device__ __forceinline__ Request request_of(const TreeArgs& a, int r)
{
    Request q;
    const int2 rows = tree_rows(a.tree, r, a.kv.status);
    q.first = rows.x;
    q.nodes = rows.y;
    q.len = paged_len(a.kv, r);
    q.tiles = max(1, (int)(((unsigned)q.len + kTile - 1) / kTile));
    q.row_tiles = (q.nodes + a.nodes_per_tile - 1) / a.nodes_per_tile;
    return q;
}

// Finds part `cta` of `ctas`: for kFindThreads threads, in shared memory that all of the CTA may read after its next
// barrier (p0 >= p1: nothing).  Each thread counts a stretch of requests; what is before a warp, a lane and a request is
// then added up.  kTiles: row tiles of the largest tree at most.
template <int kTiles>
__device__ __forceinline__ void find_part(const TreeArgs& a, int cta, int ctas, Part& part)
{
    constexpr int kWarps = kFindThreads / 32;
    const int i = threadIdx.x, warp = i >> 5, lane = i & 31, R = a.tree.n_requests;
    const int stretch = (R + kFindThreads - 1) / kFindThreads;
    const int r0 = (int)min((long long)R, (long long)i * stretch), r1 = min(R, r0 + stretch);
    long long mine[kTiles] = {}, upto[kTiles] = {};
    int longest = 0;
    for (int r = r0; r < r1; ++r) {
        const Request q = request_of(a, r);
        if (q.row_tiles > 0) longest = max(longest, q.tiles);
#pragma unroll
        for (int k = 0; k < kTiles; ++k)
            if (k < q.row_tiles) mine[k] += q.tiles + (1ll << kUnitBit);
    }
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        if (k >= a.row_tiles) continue;
        upto[k] = mine[k];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto[k], off);
            if (lane >= off) upto[k] += y;
        }
        if (lane == 31) part.sums[k][warp] = upto[k];
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 0) part.longest[warp] = longest;
    find_barrier();
    long long line[kTiles] = {}, total = 0;
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        if (k >= a.row_tiles) continue;
        for (int x = 0; x < kWarps; ++x) line[k] += part.sums[k][x];
        total += places(line[k], 0);
    }
    for (int x = 0; x < kWarps; ++x) longest = max(longest, part.longest[x]);
    const int cost = total * a.Hkv >= (long long)ctas * kShortPart ? kUnitCost : 0;
    total = 0;
#pragma unroll
    for (int k = 0; k < kTiles; ++k) total += places(line[k], cost);
    // CTAs of the lines: by their lengths, one at least; the first line, the longest, gets what is over
    int rt = 0, cta0 = 0, n = ctas;
    long long mine_all = line[0];
#pragma unroll
    for (int k = kTiles - 1; k > 0; --k) {
        if (line[k] == 0 || rt != 0) continue;
        const int c = max(1, (int)divide(ctas * places(line[k], cost), total));
        n -= c;
        if (cta >= n) {
            rt = k;
            cta0 = n;
            n = c;
            mine_all = line[k];
        }
    }
    const long long all = places(mine_all, cost) * a.Hkv;
    // equal parts, in each at least one tile of a unit that begins in it; no unit in more of them than there may be
    long long per = divide(all + n - 1, n);
    if (a.n_splits > 1) per = max(per, divide((long long)longest + cost + a.n_splits - 2, a.n_splits - 1));
    per = max((long long)cost + 1, per);
    const long long p0 = (cta - cta0) * per, p1 = min(all, p0 + per);
    if (i == 0) {
        part.p0 = p0;
        part.p1 = p1;
        part.per = per;
        part.cost = cost;
        part.rt = rt;
        part.cta0 = cta0;
    }
    long long at = 0;
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
        if (k != rt) continue;
        for (int x = 0; x < warp; ++x) at += part.sums[k][x];
        at = places(at + upto[k] - mine[k], cost) * a.Hkv;
        if (p0 >= p1 || p0 < at || p0 >= at + places(mine[k], cost) * a.Hkv) continue;
        for (int r = r0; r < r1; ++r) {  // one thread: the part begins in its stretch
            const Request q = request_of(a, r);
            if (q.row_tiles <= k) continue;
            const long long long_is = q.tiles + cost;
            if (p0 < at + long_is * a.Hkv) {
                part.r = r;
                part.q = q;
                part.h = (int)divide(p0 - at, long_is);
                part.start = at + part.h * long_is;
                break;
            }
            at += long_is * a.Hkv;
        }
    }
}

// The units of a part, one after another.
struct Walk {
    int rt, r, h;
    Request q;
    long long start;   // of the unit, on the line
    int tile0, tiles;  // of its tiles, those in this part

    __device__ __forceinline__ int committed() const { return q.len - q.nodes; }
    __device__ __forceinline__ int node0(const TreeArgs& a) const { return rt * a.nodes_per_tile; }
    __device__ __forceinline__ int rows(const TreeArgs& a) const
    {
        return min(a.nodes_per_tile, q.nodes - node0(a)) * (a.Hq / a.Hkv);
    }
    // first and last CTA that has tiles of the unit (from the line's first)
    __device__ __forceinline__ int first_cta(const Part& p) const { return (int)divide(start + p.cost, p.per); }
    __device__ __forceinline__ int last_cta(const Part& p) const { return (int)divide(start + p.cost + q.tiles - 1, p.per); }
    // false if none of its tiles is in this part
    __device__ __forceinline__ bool cut(const TreeArgs& a, const Part& p)
    {
        tile0 = 0;
        tiles = q.tiles;
        if (a.n_splits == 1) return true;  // units are not divided: the part in which one begins takes it
        const long long first = start + p.cost;  // place of its first tile
        tile0 = (int)max(0ll, p.p0 - first);
        tiles = (int)(min(p.p1, first + q.tiles) - first) - tile0;
        return tiles > 0;
    }
    __device__ __forceinline__ bool next(const TreeArgs& a, const Part& p)
    {
        start += q.tiles + p.cost;
        if (start >= p.p1) return false;
        if (++h == a.Hkv) {
            h = 0;
            do {
                if (++r == a.tree.n_requests) return false;
                q = request_of(a, r);
            } while (q.row_tiles <= rt);
        }
        return cut(a, p);
    }
    // the first one; false if there is none
    __device__ __forceinline__ bool begin(const TreeArgs& a, const Part& p)
    {
        if (p.p0 >= p.p1) return false;
        rt = p.rt;
        r = p.r;
        h = p.h;
        start = p.start;
        q = p.q;
        if (a.n_splits == 1 && start < p.p0) return next(a, p);
        return cut(a, p);
    }
};

// Tokens t .. t + 31: bits of those that a row sees.
__device__ __forceinline__ uint32_t seen_tokens(int t, int committed, int len, unsigned long long sees)
{
    if (t <= committed - 32) return 0xffffffffu;
    uint32_t bits;
    const int behind = t - committed;  // the first one's place behind the committed tokens
    if (behind >= 0) {
        bits = behind < 64 ? (uint32_t)(sees >> behind) : 0u;
    } else {
        bits = (uint32_t)(sees << -behind) | ((1u << -behind) - 1u);
    }
    return t <= len - 32 ? bits : len > t ? bits & ((1u << (len - t)) - 1u) : 0u;
}

// ---- softmax ----------------------------------------------------------------------------------------
// Values of half a tile behind the context, and those of drafted tokens that are not finite, become 0 (bf16): two threads per
// token row.
template <int D>
__device__ __forceinline__ bool clean_values(Smem<D, false>& sm, const UnitInfo& u, int t0, uint32_t step, uint32_t n_unit, int i)
{
    using C = Cfg<D, false>;
    const uint32_t seq = step | 1u;
    if (!warp_wait(&sm.full[seq % C::kSlots], (seq / C::kSlots) & 1, &sm.gave_up)) return false;
    const int token = i & (kStep - 1), t = t0 + token, behind = t - u.committed;
    if (behind >= 0) {
        // 16-byte pieces: of a half of the dimensions (D = 128), every second one (D = 64)
        uint8_t* at = sm.slot[seq % C::kSlots] + (C::kHalves == 2 ? (i >> 6) * kHalfBytes : 0) + ((step & 1) * kStep + token) * 128;
#pragma unroll 4
        for (int x = C::kHalves == 2 ? 0 : i >> 6; x < 8; x += C::kHalves == 2 ? 1 : 2) {
            uint4* p = reinterpret_cast<uint4*>(at + (((x + i) & 7) << 4));
            if (t >= u.len) {
                *p = make_uint4(0, 0, 0, 0);
                continue;
            }
            const uint4 v = *p;
            const uint32_t m = 0x7fff7fffu;
            const uint32_t top = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
            if (__vmaxu2(top, 0x7f7f7f7fu) == 0x7f7f7f7fu) continue;  // all below an infinity
            uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((word[e] & 0x7f80u) == 0x7f80u) word[e] &= 0xffff0000u;
                if ((word[e] & 0x7f800000u) == 0x7f800000u) word[e] &= 0xffffu;
            }
            atomicOr(&sm.bad[n_unit & 7], 1ull << behind);
            *p = make_uint4(word[0], word[1], word[2], word[3]);
        }
    }
    fence_proxy_async_smem();
    return true;
}

// Scores of every kGroups-th step (half a tile) -> probabilities.  A row's reference m passes from step to step; it moves when a
// step's maximum passes it by 2^8, and whoever moves it rescales O.  Each group keeps its own sum, relative to the reference
// that it saw last.  The reference is handed on when half of a step's exponentials are done, which also keeps the groups out of
// step: handed on before them, both have their exponentials at one time and wait at another, and after all of them it comes too
// late (bf16 24 requests of 60 nodes 552 us before, 529 halfway, 550 after; 4 bits with D = 64, 100 of 5-33 nodes 88, 86, 94).
// 4 bits with D = 128 have the reference handed on first: the tensor cores wait for keys there, and halfway costs more than
// it orders (32 of 64 nodes 529 us before, 581 halfway, 534 after).
template <int D, bool F4, int P>
__device__ __forceinline__ void softmax_role(Smem<D, F4>& sm, uint32_t tmem, int group, int warp, int i)
{
    constexpr int kGroups = Cfg<D, F4>::kGroups;
    // 4 bits: scores are read twice, 32 at a time, and loops are rolled.  The roles' code shares the instruction caches, and the
    // widening takes its part (64 scores at once and unrolled: 32 requests of 64 nodes 591 us, rolled 571, with the reference
    // handed on halfway in both; bf16 24 of 60 nodes 529 us unrolled, 537 rolled).
    constexpr int kKeep = F4 ? 0 : 1;
    constexpr bool kHandOnFirst = P > 1 || (F4 && D == 128);
    int* gave_up = &sm.gave_up;
    const int before_me = group == 0 ? kGroups - 1 : group - 1;  // the group of the step before
    uint32_t mine = group;             // this group's next step, and how many it had
    uint32_t turn = 0;
    uint32_t unit0 = 0;                // first step of the unit
    for (uint32_t n_unit = 0;; ++n_unit) {
        if (!warp_wait(&sm.q_full[n_unit & 1], (n_unit >> 1) & 1, gave_up)) return;
        const UnitInfo u = sm.info[n_unit & 1];
        const unsigned long long sees = sm.sees[n_unit & 1][i];
        const float unit = sm.row_unit[n_unit & 1][i];  // log2 units of one score
        const bool live = i % Spread<P>::kRows < u.rows, warp_live = (warp & 3) * 32 % Spread<P>::kRows < u.rows;
        float m = -INFINITY, l = 0.f;
        const uint32_t end = unit0 + 2 * u.tiles;
        for (; mine < end; mine += kGroups, ++turn) {
            const int t0 = u.tile0 * kTile + (int)(mine - unit0) * kStep;
            const bool ends = t0 > u.committed - kStep;  // some row does not see all of it
            if constexpr (!F4)
                if (ends && !clean_values<D>(sm, u, t0, mine, n_unit, i)) return;
            if (!warp_wait(&sm.s_full[mine & 3], (mine >> 2) & 1, gave_up)) return;
            if (group == 0 && i == 0) *static_cast<volatile uint32_t*>(&sm.step) = mine;
            tc_fence_after_sync();
            const uint32_t t_s = tmem + kColS + (mine & 3) * kStep;
            if (P == 1 && ends && warp_live) {  // scores of what the row does not see, in place
#pragma unroll 1
                for (int c = 0; c < kStep / 16; ++c) {
                    const uint32_t see = sees == 0 ? 0u : seen_tokens(t0 + 16 * c, u.committed, u.len, sees);
                    uint32_t x[16];
                    tmem_ld16(t_s + 16 * c, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!((see >> e) & 1)) x[e] = 0xff800000u;
                    tmem_st16(t_s + 16 * c, x);
                }
                tmem_st_wait();
            }
            float mx = -INFINITY;
            uint32_t s[1 + kKeep][32];
            constexpr int kCols = Spread<P>::kCols;
            const uint32_t part = i / Spread<P>::kRows;  // (the same for the warp)
            uint32_t few[kCols];
            if constexpr (P > 1) {
                if (warp_live) {
                    if constexpr (P == 4) tmem_ld16(t_s + kCols * part, few);
                    else tmem_ld32(t_s + kCols * part, few);
                    tmem_ld_wait();
                    if (ends) {
                        const uint32_t see = sees == 0 ? 0u : seen_tokens(t0 + kCols * part, u.committed, u.len, sees);
#pragma unroll
                        for (int e = 0; e < kCols; ++e)
                            if (!((see >> e) & 1)) few[e] = 0xff800000u;
                    }
                    float m2[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int e = 0; e < kCols / 2; ++e)
                        m2[e & 1] = fmax3(m2[e & 1], __uint_as_float(few[2 * e]), __uint_as_float(few[2 * e + 1]));
                    mx = fmaxf(m2[0], m2[1]);
                }
            } else if (warp_live) {
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto most = [&](const uint32_t (&x)[32]) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        m4[e & 3] = fmax3(m4[e & 3], __uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]));
                };
                if constexpr (kKeep) {
                    tmem_ld32(t_s, s[0]);
                    tmem_ld32(t_s + 32, s[kKeep]);
                    tmem_ld_wait();
                    most(s[0]);
                    most(s[kKeep]);
                } else {
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        tmem_ld32(t_s + 32 * c, s[0]);
                        tmem_ld_wait();
                        most(s[0]);
                    }
                }
                mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            }
            // the reference of the step before
            if (mine > 0 && !warp_wait(&sm.ref_full[before_me][warp & 3], (group == 0 ? turn - 1 : turn) & 1, gave_up)) return;
            const float before = mine == unit0 ? mx : sm.ref[before_me][i];
            const bool need = mine != unit0 && live && (mx - before) * unit > kRescaleAt;
            const float now = need ? mx : before;
            sm.ref[group][i] = now;
            if (kHandOnFirst || !warp_live) mbar_arrive(&sm.ref_full[group][warp & 3]);
            if (warp_live) {
                if (__any_sync(0xffffffffu, need)) {
                    // the last product has left O (its barrier's turn before, four steps back, is over: these scores came behind it)
                    if (!warp_wait(&sm.pv_done[(mine - 1) & 3], ((mine - 1) >> 2) & 1, gave_up)) return;
                    tc_fence_after_sync();
                    const float alpha = need ? fast_exp2((before - now) * unit) : 1.f;
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld16(tmem + kColO + 16 * c, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                        tmem_st16(tmem + kColO + 16 * c, o);
                    }
                }
                if (now != m) l *= fast_exp2((m - now) * unit);
                m = now;
                // (the product rounded before the difference, as lse has it)
                const float base = m == -INFINITY ? 0.f : __fmul_rn(m, unit) - (F4 ? kBelowF16 : 0.f);  // (nothing seen yet)
                const float2 unit2 = make_float2(unit, unit), base2 = make_float2(-base, -base);
                float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                auto exponentials_of = [&](const auto& x, auto& pk) {
#pragma unroll
                    for (int e = 0; e < (int)(sizeof(pk) / 4); ++e) {
                        float2 p = ffma2(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), unit2, base2);
                        p.x = fast_exp2(p.x);
                        p.y = fast_exp2(p.y);
                        l2[e & 1] = fadd2(l2[e & 1], p);
                        pk[e] = F4 ? f16x2(p.x, p.y) : bf16x2(p.x, p.y);
                    }
                };
                auto exponentials = [&](const uint32_t (&x)[32], int c) {
                    uint32_t pk[16];
                    exponentials_of(x, pk);
                    tmem_st16(t_s + 16 * c, pk);  // over columns that have been read
                };
                if constexpr (P > 1) {
                    uint32_t pk[kCols / 2], none[kCols / 2] = {};
                    exponentials_of(few, pk);
#pragma unroll
                    for (uint32_t c = 1; c < P; ++c) {  // the other parts' tokens
                        const uint32_t at = t_s + kCols / 2 * ((part + c) % P);
                        if constexpr (P == 4) tmem_st8(at, none);
                        else tmem_st16(at, none);
                    }
                    if constexpr (P == 4) tmem_st8(t_s + kCols / 2 * part, pk);
                    else tmem_st16(t_s + kCols / 2 * part, pk);
                } else if constexpr (kKeep) {
                    static_assert(!kHandOnFirst, "handed on once");
                    exponentials(s[0], 0);
                    mbar_arrive(&sm.ref_full[group][warp & 3]);
                    exponentials(s[kKeep], 1);
                } else {
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        tmem_ld32(t_s + 32 * c, s[0]);
                        tmem_ld_wait();
                        exponentials(s[0], c);
                        if (c == 0 && !kHandOnFirst) mbar_arrive(&sm.ref_full[group][warp & 3]);
                    }
                }
                l += (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
                tmem_st_wait();
            }
            tc_fence_before_sync();
            mbar_arrive(&sm.p_full[mine & 3]);
        }
        unit0 = end;
        sm.stat[n_unit & 1][group][i] = make_float2(m, l);
        mbar_arrive(&sm.stat_full[n_unit & 1]);
        if (!u.more) return;
    }
}

// ---- queries and results ----------------------------------------------------------------------------
template <int D, bool F4, int P>
struct Rows {
    using C = Cfg<D, F4>;
    Smem<D, F4>& sm;
    const TreeArgs& a;
    const uint32_t tmem;  // with this warp's lanes
    const int i;          // row
    const int warp = i >> 5, lane = i & 31;
    const int ir = i % Spread<P>::kRows;  // row of the unit

    // 128 bytes of every row of the warp, from its lane's registers to where the row goes (row_to), at `offset`: eight lanes a
    // row (rows of the warp's lanes one by one: 3600 cycles a unit).
    __device__ __forceinline__ void store_pieces(const uint32_t (&x)[32], int offset)
    {
        uint8_t(*stage)[kStagePitch] = sm.stage[warp];
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(&stage[lane][16 * e]) = make_uint4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
        __syncwarp();
        uint8_t* to[8];
        uint4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = 4 * e + (lane >> 3);
            to[e] = static_cast<uint8_t*>(sm.row_to[warp][row]);
            v[e] = *reinterpret_cast<const uint4*>(&stage[row][16 * (lane & 7)]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (to[e] != nullptr) *reinterpret_cast<uint4*>(to[e] + offset + 16 * (lane & 7)) = v[e];
    }

    // A unit's rows: what they see, and their queries into tensor memory.  With 4-bit pages times a power of two that brings
    // the row's largest element into [2^16, 2^17): scores stay finite, keys being up to 6 * 65504 2^-16.
    __device__ __forceinline__ void prepare(const Walk& w, bool new_request, bool more, uint32_t n_unit)
    {
        if (new_request) {
            row_barrier();
            if (i < MOSKA_TREE_MAX_NODES)
                tree_ancestors(sm.tree, i, i < w.q.nodes ? tree_parent(a.tree, w.q.first, i, a.kv.status) : -1,
                               [] { asm volatile("bar.sync 3, 64;" ::: "memory"); });
            row_barrier();
        }
        const int G = a.Hq / a.Hkv, node = w.node0(a) + ir / G, committed = w.committed(), rows = w.rows(a);
        const bool live = ir < rows;
        unsigned long long sees = live && committed + node >= 0 ? sm.tree.bits[node] : 0;
        if (committed < 0) sees &= ~0ull << min(63, -committed);  // nodes without a token
        sm.sees[n_unit & 1][i] = sees;
        if (i == 0) sm.info[n_unit & 1] = UnitInfo{committed, w.q.len, w.tile0, w.tiles, rows, more};
        // Rows come in pieces of 64 dimensions: eight lanes a row, by way of shared memory (a lane that reads its own row touches
        // another line in each of 16 loads).
        const int64_t at = live ? ((int64_t)(w.q.first + node) * a.Hq + w.h * G + ir % G) * D : -1;
        const uint32_t rows_here = __ballot_sync(0xffffffffu, live);
        auto load = [&](int c, uint4 (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (a row that is none reads the batch's first one: no branch keeps a load waiting for the one before)
                const int64_t from = __shfl_sync(0xffffffffu, max(at, (int64_t)0), 4 * e + (lane >> 3));
                v[e] = __ldg(reinterpret_cast<const uint4*>(a.q + from + 64 * c + 8 * (lane & 7)));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!((rows_here >> (4 * e + (lane >> 3))) & 1)) v[e] = make_uint4(0, 0, 0, 0);
        };
        // 4 bits: once for the rows' largest elements, then for the operands.  (Rolled, with a row's elements in its lane: the code
        // is cold when a CTA begins.  Maxima of pieces, joined by shuffles, took 11000 cycles.)
        if constexpr (!F4) sm.row_unit[n_unit & 1][i] = fminf(a.scale * kLog2e, FLT_MAX);  // (a score of 0 times an infinity is NaN)
        float down = 1.f;
        uint32_t top = 0;
        uint8_t(*stage)[kStagePitch] = sm.stage[warp];
#pragma unroll 1
        for (int it = F4 ? 0 : D / 64; it < 2 * (D / 64); ++it) {
            const int c = it % (D / 64);
            uint4 v[8];
            load(c, v);
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(&stage[4 * e + (lane >> 3)][16 * (lane & 7)]) = v[e];
            __syncwarp();
            uint32_t x[32];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint4 y = *reinterpret_cast<const uint4*>(&stage[lane][16 * e]);
                x[4 * e] = y.x;
                x[4 * e + 1] = y.y;
                x[4 * e + 2] = y.z;
                x[4 * e + 3] = y.w;
            }
            if constexpr (F4) {
                if (it < D / 64) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) top = __vmaxu2(top, x[e] & 0x7fff7fffu);
                    if (it + 1 == D / 64) {
                        const int e2 = min(max((int)(max(top >> 16, top & 0xffffu) >> 7), 17), 252) - 127;
                        down = __uint_as_float((uint32_t)(127 + 16 - e2) << 23);
                        // (neither 0 nor infinite: the -inf of a hidden token, or a score of 0, times that would be NaN)
                        sm.row_unit[n_unit & 1][i] =
                            fminf(fmaxf(a.scale * __uint_as_float((uint32_t)(127 + e2) << 23) * kLog2e, FLT_MIN), FLT_MAX);
                    }
                    continue;
                }
                // dimensions e and e + 4 of eight together, as in the keys' operands
                auto lower = [&](uint32_t y) { return __uint_as_float(y << 16) * down; };
                auto upper = [&](uint32_t y) { return __uint_as_float(y & 0xffff0000u) * down; };
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const uint32_t y[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        x[e + 2 * u] = bf16x2(lower(y[u]), lower(y[u + 2]));  // (exact)
                        x[e + 2 * u + 1] = bf16x2(upper(y[u]), upper(y[u + 2]));
                    }
                }
            }
            tmem_st32(tmem + kColQ + (n_unit & 1) * 64 + 32 * c, x);
        }
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(&sm.q_full[n_unit & 1]);
    }

    // Adds the values that were taken out of the operands to a row that sees them, 0 or not: whatever is added to is not finite
    // then.  Rare, and out of the way of what is not.
    __device__ __forceinline__ void put_back(const int32_t* pages, int h, int committed, unsigned long long odd, void* to,
                                             bool is_bf16) const
    {
#pragma unroll 1
        for (unsigned long long left = odd; left != 0; left &= left - 1) {
            const int t = committed + __ffsll(left) - 1, in = t & ((1 << a.kv.page_shift) - 1);
            const int64_t page = paged_page(a.kv, pages, t >> a.kv.page_shift);
#pragma unroll 1
            for (int d = 0; d < D; ++d) {
                float v;
                if constexpr (F4) {
                    using B = Fp4Block<D>;
                    const uint8_t* b = a.kv.k + (((page * a.Hkv + h) << (a.kv.page_shift - 4)) + (in >> 4)) * B::kBytes;
                    const uint16_t sc = *reinterpret_cast<const uint16_t*>(b + B::v_scale(in & 15, d / 32));
                    if ((sc & 0x7fffu) <= 0x7154u) continue;
                    uint32_t f[4];
                    e2m1x8_to_f16x2(*reinterpret_cast<const uint32_t*>(b + B::v_byte(in & 15, d & ~7)), f);
                    const uint32_t code2 = (d & 4) ? ((d & 2) ? f[3] : f[2]) : ((d & 2) ? f[1] : f[0]);
                    const uint32_t x = hmul2(code2, sc * 0x10001u);
                    const uint32_t bits = (d & 1) ? x >> 16 : x & 0xffffu;
                    if ((bits & 0x7c00u) != 0x7c00u) continue;
                    v = __half2float(__ushort_as_half((unsigned short)bits));
                } else {
                    const uint16_t x = reinterpret_cast<const uint16_t*>(a.kv.v)[(((page << a.kv.page_shift) + in) * a.Hkv + h) * D + d];
                    if ((x & 0x7f80u) != 0x7f80u) continue;
                    v = __uint_as_float((uint32_t)x << 16);
                }
                if (is_bf16) {
                    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(to) + d;
                    *o = __float2bfloat16_rn(__bfloat162float(*o) + v);
                } else {
                    static_cast<float*>(to)[d] += v;
                }
            }
        }
    }

    // The unit's rows: final ones, partial ones of a cut unit, or partial slots.
    __device__ __forceinline__ bool finish(const Walk& w, uint32_t n_unit, uint32_t last)
    {
        bool ok = unit_wait(&sm.stat_full[n_unit & 1], (n_unit >> 1) & 1, &sm.step, &sm.gave_up);
        // the group of the last step has the row's reference; the others' sums are brought to it
        const float unit = sm.row_unit[n_unit & 1][i];
        const float mine = sm.stat[n_unit & 1][last % C::kGroups][i].x;
        float m = mine;
#pragma unroll
        for (int p = 0; p < (P > 1 ? P : 0); ++p) m = fmaxf(m, sm.stat[n_unit & 1][last % C::kGroups][ir + p * Spread<P>::kRows].x);
        float l = 0.f;
#pragma unroll
        for (int x = 0; x < C::kGroups; ++x)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float2 part = sm.stat[n_unit & 1][x][ir + p * Spread<P>::kRows];
                l += part.x == m ? part.y : part.y * fast_exp2((part.x - m) * unit);
            }
        const int G = a.Hq / a.Hkv, node = w.node0(a) + ir / G;
        const bool live = i < w.rows(a);
        const int64_t row = (int64_t)(w.q.first + node) * a.Hq + w.h * G + ir % G;
        float inv = l == 0.f ? 0.f : 1.f / l;
        if (P > 1 && mine != m) inv *= fast_exp2((mine - m) * unit);  // (0 for a part that has seen nothing)
        const float lse = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m * unit * kLn2) + logf(F4 ? l * 0.0078125f : l);
        static_assert(kBelowF16 == 7.f, "l is 2^7 times the sum relative to the reference");
        const bool final_row = a.out != nullptr && w.tiles == w.q.tiles;  // (the same for all rows)
        void* to = a.out + row * D;
        float* lse_to = a.lse_out != nullptr ? a.lse_out + row : nullptr;
        int spare = 0;  // slots behind this one that hold nothing
        if (!final_row && a.out == nullptr) {
            const int c0 = w.first_cta(sm.part);
            const int k = a.n_splits == 1 ? 0 : (int)blockIdx.x - sm.part.cta0 - c0;
            const int parts = a.n_splits == 1 ? 1 : w.last_cta(sm.part) - c0 + 1;
            const int64_t slot = row * a.n_slots + a.slot0 + k;
            to = a.o_part + slot * D;
            lse_to = a.lse_part + slot;
            if (k == parts - 1) spare = a.n_splits - parts;
        } else if (!final_row) {
            const int64_t slot = (int64_t)(2 * blockIdx.x + (w.tile0 == 0 ? 1 : 0)) * kTileRows + i;
            to = a.o_cut + slot * D;
            lse_to = a.lse_cut + slot;
        }
        sm.row_to[warp][lane] = live ? to : nullptr;
        ok = ok && warp_wait(&sm.o_full, n_unit & 1, &sm.gave_up);
        if (!row_barrier(ok)) return false;
        tc_fence_after_sync();
        if constexpr (P > 1) {
            // the sum of the parts, by way of shared memory: thread x has dimensions 8 (x % 4) .. of row x / 4 (P = 4), or 16 of row x / 2
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(tmem + kColO + 32 * c, o);
                tmem_ld_wait();
                if (c + 1 == D / 32) {
                    tc_fence_before_sync();
                    mbar_arrive(&sm.o_free);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float y[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) y[x] = inv == 0.f ? 0.f : __uint_as_float(o[4 * e + x]) * inv;
                    *reinterpret_cast<float4*>(&sm.stage[warp][lane][16 * e]) = make_float4(y[0], y[1], y[2], y[3]);
                }
                row_barrier();
                constexpr int kLanes = kTileRows / Spread<P>::kRows, kDims = 32 / kLanes;  // threads of a row, dimensions of each
                const int r = i / kLanes, d0 = (i % kLanes) * kDims;
                float y[kDims] = {};
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int x = 0; x < kDims; x += 4) {
                        const int from = r + p * Spread<P>::kRows;
                        const float4 v = *reinterpret_cast<const float4*>(&sm.stage[from >> 5][from & 31][4 * (d0 + x)]);
                        y[x] += v.x; y[x + 1] += v.y; y[x + 2] += v.z; y[x + 3] += v.w;
                    }
                uint8_t* row_to = static_cast<uint8_t*>(sm.row_to[r >> 5][r & 31]);
                if (row_to != nullptr) {
#pragma unroll
                    for (int x = 0; x < kDims; x += 8) {
                        if (final_row) {
                            *reinterpret_cast<uint4*>(row_to + 2 * (32 * c + d0 + x)) =
                                make_uint4(bf16x2(y[x], y[x + 1]), bf16x2(y[x + 2], y[x + 3]), bf16x2(y[x + 4], y[x + 5]),
                                           bf16x2(y[x + 6], y[x + 7]));
                        } else {
                            float4* to4 = reinterpret_cast<float4*>(row_to + 4 * (32 * c + d0 + x));
                            to4[0] = make_float4(y[x], y[x + 1], y[x + 2], y[x + 3]);
                            to4[1] = make_float4(y[x + 4], y[x + 5], y[x + 6], y[x + 7]);
                        }
                    }
                }
                row_barrier();
            }
        } else if (final_row) {
            uint32_t y[D / 64][32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(tmem + kColO + 32 * c, o);
                tmem_ld_wait();
                // (a row that has seen nothing: its O is 0 or was never written)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    y[c >> 1][16 * (c & 1) + e] =
                        l == 0.f ? 0u : bf16x2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
            }
            tc_fence_before_sync();
            mbar_arrive(&sm.o_free);  // O may be written again
#pragma unroll
            for (int c = 0; c < D / 64; ++c) store_pieces(y[c], 128 * c);
        } else {
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(tmem + kColO + 32 * c, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
                store_pieces(o, 128 * c);
            }
            tc_fence_before_sync();
            mbar_arrive(&sm.o_free);
        }
        if (live)
#pragma unroll 1
            for (int k = 1; k <= spare; ++k) {
                lse_to[k] = -INFINITY;
#pragma unroll 1
                for (int d = 0; d < D; d += 4)
                    *reinterpret_cast<float4*>(static_cast<float*>(to) + k * D + d) = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        __syncwarp();
        if (live && lse_to != nullptr) *lse_to = lse;
        const unsigned long long odd =
            l == 0.f ? 0 : *static_cast<volatile unsigned long long*>(&sm.bad[n_unit & 7]) & sm.sees[n_unit & 1][i];
        if (live && odd != 0)
            put_back(a.kv.page_table + (int64_t)w.r * a.kv.max_pages, w.h, w.committed(), odd, to, final_row);
        row_barrier();  // all have read `bad`
        if (i == 0) sm.bad[n_unit & 7] = 0;
        return true;
    }

    // One unit is prepared ahead of the one that is finished.
    __device__ __forceinline__ void run(Walk w)
    {
        Walk after = w;
        bool more = after.next(a, sm.part);
        prepare(w, true, more, 0);
        uint32_t steps = 0;
        for (uint32_t n_unit = 0;; ++n_unit) {
            Walk then = after;
            const bool go_on = more;
            if (go_on) {
                more = then.next(a, sm.part);
                prepare(after, after.r != w.r, more, n_unit + 1);
            }
            steps += 2 * w.tiles;
            if (!finish(w, n_unit, steps - 1) || !go_on) return;
            w = after;
            after = then;
        }
    }
};

// ---- copies -----------------------------------------------------------------------------------------
template <int D, bool F4>
__device__ __forceinline__ void load_role(Smem<D, F4>& sm, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const TreeArgs& a,
                                          Walk w, int lane)
{
    using C = Cfg<D, F4>;
    const int shift = a.kv.page_shift;
    uint32_t seq = 0;
    bool ok = true;
    do {
        const int32_t* pages = a.kv.page_table + (int64_t)w.r * a.kv.max_pages;
        if constexpr (!F4) {
            const int box = min(kTile, 1 << shift);  // tokens of a copy; lane b < kTile / box copies the b-th of a tile
            const int boxes = kTile / box;
            auto page_of = [&](int j) {
                const int t = (w.tile0 + j) * kTile + lane * box;
                return lane < boxes && j < w.tiles && t < w.q.len ? paged_page(a.kv, pages, t >> shift) : -1;
            };
            int ahead = page_of(0);
            for (int j = 0; j < w.tiles && ok; ++j) {
                const int page = ahead;
                ahead = page_of(j + 1);
                const int t = (w.tile0 + j) * kTile + lane * box;
                const int there = __popc(__ballot_sync(0xffffffffu, page >= 0));
                const int z = (page << shift) + (t & ((1 << shift) - 1));
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    const uint32_t s = seq % C::kSlots;
                    if (seq >= C::kSlots) ok = warp_wait(&sm.empty[s], ((seq / C::kSlots) - 1) & 1, &sm.gave_up);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(&sm.full[s], there * box * 128 * C::kHalves);
                    __syncwarp();
                    if (page >= 0)
#pragma unroll
                        for (int hv = 0; hv < C::kHalves; ++hv)
                            tma_load_3d(sm.slot[s] + hv * kHalfBytes + lane * box * 128, kind == 0 ? &tm_k : &tm_v, 64 * hv, w.h, z,
                                        &sm.full[s]);
                    ++seq;
                }
            }
        } else {
            using B = Fp4Block<D>;
            // A page's blocks of a head are neighbours: one copy of min(page_size, 128) tokens, up to the context's last block.
            // (Copies of key and value parts, block by block, kept the tensor cores waiting: a copy costs its warp about 60 cycles.)
            const int box = min(kTile, 1 << shift), boxes = kTile / box;
            const int64_t page_bytes = ((int64_t)a.Hkv << (shift - 4)) * B::kBytes;
            const uint8_t* pool = a.kv.k + ((int64_t)w.h << (shift - 4)) * B::kBytes;
            auto page_of = [&](int j) {
                const int t = (w.tile0 + j) * kTile + lane * box;
                return lane < boxes && j < w.tiles && t < w.q.len ? paged_page(a.kv, pages, t >> shift) : -1;
            };
            int ahead = page_of(0);
            for (int j = 0; j < w.tiles; ++j) {
                const int page = ahead;
                ahead = page_of(j + 1);
                const int t0 = (w.tile0 + j) * kTile, t = t0 + lane * box;
                const uint32_t s = seq % C::kCodeSlots;
                if (seq >= C::kCodeSlots) ok = warp_wait(&sm.code_empty[s], ((seq / C::kCodeSlots) - 1) & 1, &sm.gave_up);
                if (!ok) break;
                const int there = (min(kTile, w.q.len - t0) + 15) >> 4;  // blocks (0: an empty context)
                if (lane == 0) mbar_arrive_expect_tx(&sm.code_full[s], max(0, there) * B::kBytes);
                __syncwarp();
                if (page >= 0)
                    bulk_load(sm.code + s * C::kCodeBytes + lane * (box >> 4) * B::kBytes,
                              pool + page * page_bytes + (int64_t)((t & ((1 << shift) - 1)) >> 4) * B::kBytes,
                              min(box >> 4, there - lane * (box >> 4)) * B::kBytes, &sm.code_full[s]);
                ++seq;
            }
        }
    } while (ok && w.next(a, sm.part));
    if (*static_cast<volatile int*>(&sm.gave_up)) {
        // the copies in flight end before the CTA leaves (each wait again has a limit)
        constexpr uint32_t kRing = F4 ? C::kCodeSlots : C::kSlots;
        for (uint32_t x = seq > kRing ? seq - kRing : 0; x < seq; ++x) {
            int never = 0;
            mbar_wait(F4 ? &sm.code_full[x % kRing] : &sm.full[x % kRing], (x / kRing) & 1, &never);
        }
    }
}

// ---- MMAs -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t descriptor(uint32_t hi, uint32_t lo) { return (static_cast<uint64_t>(hi) << 32) | lo; }

// Scores of step after step, into the buffer of the step four before, when its probabilities have been used.
template <int D, bool F4>
__device__ __forceinline__ void score_role(Smem<D, F4>& sm, uint32_t tmem)
{
    using C = Cfg<D, F4>;
    const uint32_t id = idesc_bf16_f32(128, kStep, false);
    const uint64_t d = smem_desc_sw128(0, 16, 1024);
    const uint32_t hi = static_cast<uint32_t>(d >> 32), lo = static_cast<uint32_t>(d) + (smem_u32(sm.slot[0]) >> 4);
    const uint32_t rest = static_cast<uint32_t>(d) + (smem_u32(sm.rest) >> 4);
    int* gave_up = &sm.gave_up;
    uint32_t step = 0;
    for (uint32_t n_unit = 0;; ++n_unit) {
        if (!warp_wait(&sm.q_full[n_unit & 1], (n_unit >> 1) & 1, gave_up)) return;
        const int steps = 2 * sm.info[n_unit & 1].tiles, more = sm.info[n_unit & 1].more;
        const uint32_t q = tmem + kColQ + (n_unit & 1) * 64;
        for (int j = 0; j < steps; ++j, ++step) {
            const uint32_t seq = step & ~1u, s = seq % C::kSlots, half = step & 1;  // (tile step / 2: slots 2 (step / 2) and the next)
            if (step >= 4 && !warp_wait(&sm.pv_done[step & 3], ((step >> 2) - 1) & 1, gave_up)) return;
            if constexpr (F4) {
                if (!warp_wait(&sm.key_full[s][half], (seq / C::kSlots) & 1, gave_up)) return;
            } else {
                if (half == 0 && !warp_wait(&sm.full[s], (seq / C::kSlots) & 1, gave_up)) return;
            }
            tc_fence_after_sync();
            if (elect_one()) {
                const uint32_t to = tmem + kColS + (step & 3) * kStep;
                const uint32_t k = lo + ((s * C::kSlotBytes + half * kStep * 128) >> 4);
                if constexpr (F4) {  // the second operand first: its buffer is wanted
                    const uint32_t r = rest + ((half * kStep * 128) >> 4);
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        mma_ts(to, q + 8 * ks, descriptor(hi, r + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4)), id, ks > 0);
                    tc_commit(&sm.rest_empty[half]);
                }
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    mma_ts(to, q + 8 * ks, descriptor(hi, k + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4)), id, F4 || ks > 0);
                tc_commit(&sm.s_full[step & 3]);
                if (half == 1) tc_commit(&sm.empty[s]);
            }
            __syncwarp();
        }
        if (!more) return;
    }
}

template <int D, bool F4>
__device__ __forceinline__ void value_role(Smem<D, F4>& sm, uint32_t tmem)
{
    using C = Cfg<D, F4>;
    const uint32_t id = F4 ? idesc_f16_f32(128, D, true) : idesc_bf16_f32(128, D, true);
    const uint64_t d = smem_desc_sw128(0, kHalfBytes, 1024);
    const uint32_t hi = static_cast<uint32_t>(d >> 32), lo = static_cast<uint32_t>(d) + (smem_u32(sm.slot[0]) >> 4);
    int* gave_up = &sm.gave_up;
    uint32_t step = 0;
    for (uint32_t n_unit = 0;; ++n_unit) {
        if (!warp_wait(&sm.q_full[n_unit & 1], (n_unit >> 1) & 1, gave_up)) return;
        const int steps = 2 * sm.info[n_unit & 1].tiles, more = sm.info[n_unit & 1].more;
        for (int j = 0; j < steps; ++j, ++step) {
            const uint32_t seq = step | 1u, s = seq % C::kSlots, half = step & 1;
            if (!warp_wait(&sm.p_full[step & 3], (step >> 2) & 1, gave_up)) return;
            if (half == 0 && !warp_wait(&sm.full[s], (seq / C::kSlots) & 1, gave_up)) return;
            // (a unit's first product overwrites O, which the rows of the unit before have to have left)
            if (j == 0 && n_unit > 0 && !warp_wait(&sm.o_free, (n_unit - 1) & 1, gave_up)) return;
            tc_fence_after_sync();
            if (elect_one()) {
                const uint32_t p = tmem + kColS + (step & 3) * kStep, v = lo + ((s * C::kSlotBytes + half * kStep * 128) >> 4);
#pragma unroll
                for (int ks = 0; ks < kStep / 16; ++ks)
                    mma_ts(tmem + kColO, p + 8 * ks, descriptor(hi, v + ((ks * 2048) >> 4)), id, j > 0 || ks > 0);
                tc_commit(&sm.pv_done[step & 3]);
                if (half == 1) tc_commit(&sm.empty[s]);
                if (j + 1 == steps) tc_commit(&sm.o_full);
            }
            __syncwarp();
        }
        if (!more) return;
    }
}

// ---- 4 bits: codes -> operand rows --------------------------------------------------------------------
// Keys of a block.  The D / 8 bytes of (token, c) are dimensions 32 x + 8 c .. + 7 for each group x.  Eight lanes that
// go to memory together have tokens y and y ^ 5: their loads and their swizzled stores both fall on eight different
// 16-byte pieces of the banks.
template <int D>
__device__ __forceinline__ void widen_keys(const uint8_t* code_tile, uint8_t* to, uint8_t* rest, int block, int lane)
{
    using B = Fp4Block<D>;
    constexpr int J = D / 32;
    const int l = lane & 7, c = l & 3, qd = lane >> 3, token = (l >> 2) ? (qd ^ 5) : qd;
#pragma unroll
    for (int it = 0; it < 2; ++it) {
        const int t = 8 * it + token, row = 16 * block + t;
        const uint8_t* from = code_tile + block * B::kBytes;
        uint32_t code[J], sc[J / 2];
        if constexpr (J == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(from + t * (D / 2) + c * (D / 8));
            code[0] = x.x; code[1] = x.y; code[2] = x.z; code[3] = x.w;
            const uint2 y = *reinterpret_cast<const uint2*>(from + B::k_scale(t, 0));
            sc[0] = y.x; sc[1] = y.y;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(from + t * (D / 2) + c * (D / 8));
            code[0] = x.x; code[1] = x.y;
            sc[0] = *reinterpret_cast<const uint32_t*>(from + B::k_scale(t, 0));
        }
#pragma unroll
        for (int x = 0; x < J; ++x) {
            // A scale has 11 bits and a code 2: the upper 6 bits of the one times the other are a bf16 number, and so are the lower
            // 5 times it.  A code's bits (s e e m) in bf16's places are the bf16 number 2^-126 times it, 0.5 a subnormal
            // one; a scale has 2^110, and the queries the 2^16 that are left.
            const uint16_t bits = (uint16_t)((x & 1) ? sc[x >> 1] >> 16 : sc[x >> 1]);
            const float scale = __half2float(__ushort_as_half(bits)) * 0x1p110f;
            const uint32_t upper = __float_as_uint(scale) & 0xfffc0000u, lower = __float_as_uint(scale - __uint_as_float(upper));
            const uint32_t upper2 = __byte_perm(upper, 0, 0x3232), lower2 = __byte_perm(lower, 0, 0x3232);
            const int at = (x >> 1) * kHalfBytes + row * 128 + (((4 * (x & 1) + c) ^ (row & 7)) << 4);
            uint32_t y[4], left[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // dimensions e and e + 4 of the eight: s to bit 15, e e m to bits 8 .. 6 of each half
                const uint32_t two = (e < 2 ? code[x] : code[x] >> 8) & (e & 1 ? 0x00f000f0u : 0x000f000fu);
                const uint32_t c2 = two * (e & 1 ? 0x104u : 0x1040u) & 0x81c081c0u;
                y[e] = bmul2(c2, upper2);
                left[e] = bmul2(c2, lower2);
            }
            *reinterpret_cast<uint4*>(to + at) = make_uint4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<uint4*>(rest + at) = make_uint4(left[0], left[1], left[2], left[3]);
        }
    }
}

// Chunk x (D / 8 dimensions) of a pair of tokens of a block: first token's bytes, then the second's.
template <int D>
struct ValueChunk {
    using B = Fp4Block<D>;
    static constexpr int W = D / 64;  // words of a token's chunk
    int block, p, x;
    __device__ __forceinline__ ValueChunk(int block0, int it, int lane) : block(block0 + (it >> 1)), p(4 * (it & 1) + (lane >> 3)), x(lane & 7) {}
    __device__ __forceinline__ const uint8_t* codes(const uint8_t* tile) const
    {
        return tile + block * B::kBytes + B::kV + p * D + (x ^ B::v_swap(p)) * (D / 8);
    }
    __device__ __forceinline__ uint32_t scales(const uint8_t* tile) const  // of both tokens
    {
        return *reinterpret_cast<const uint32_t*>(tile + block * B::kBytes + B::v_scale(2 * p, x * (D / 8) / 32));
    }
    __device__ __forceinline__ int row(int tok) const { return 16 * block + 2 * p + tok; }
    // where the operand's 16 bytes of word y of the token's chunk go
    __device__ __forceinline__ uint8_t* piece(uint8_t* to, int tok, int y) const
    {
        const int at = W == 2 ? 2 * (x & 3) + y : x;
        return to + (W == 2 ? (x >> 2) * kHalfBytes : 0) + row(tok) * 128 + ((at ^ (row(tok) & 7)) << 4);
    }
};

// The same for drafted tokens with a scale above what appends write, after widen_values has made them 0: products that are finite
// as they are.  (Of its own and rolled: in the loop of all values 32 requests of 64 nodes took 636 us instead of 558.)
template <int D>
__device__ __forceinline__ void widen_odd_values(const uint8_t* code_tile, uint8_t* to, int block0, int lane, int behind, int nodes,
                                                 unsigned long long* bad)
{
    constexpr int W = ValueChunk<D>::W;
#pragma unroll 1
    for (int n = 0; n < 8 * W; ++n) {
        const int tok = n & 1, y = W == 2 ? (n >> 1) & 1 : 0;
        const ValueChunk<D> c(block0, n / (2 * W), lane);
        const int node = behind + c.row(tok);
        const uint32_t s2 = __byte_perm(c.scales(code_tile), 0, tok ? 0x3232 : 0x1010);
        if (node < 0 || node >= nodes || (s2 & 0x7fffu) <= 0x7154u) continue;
        uint32_t f[4], out = 0;
        e2m1x8_to_f16x2(*reinterpret_cast<const uint32_t*>(c.codes(code_tile) + 4 * (tok * W + y)), f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = hmul2(f[e], s2);
            const uint32_t gone = ((f[e] & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((f[e] & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u);
            f[e] &= ~gone;
            out |= gone;
        }
        if (out != 0) atomicOr(bad, 1ull << node);
        *reinterpret_cast<uint4*>(c.piece(to, tok, y)) = make_uint4(f[0], f[1], f[2], f[3]);
    }
}

// Values of two blocks.  In a tile that reaches past the committed tokens (kEnds; `behind`: its first token's place behind them) values behind the context are 0, and those
// that are not finite are taken out.
// (A form of its own for the others: a branch at each token keeps loads and stores waiting, 1590 cycles a tile where it takes 1200;
// 64 requests of 8 nodes 214 us, 222 with one form; 32 of 64 nodes 524 and 529.)
template <int D, bool kEnds>
__device__ __forceinline__ void widen_values(const uint8_t* code_tile, uint8_t* to, int block0, int lane, int behind, int nodes,
                                             unsigned long long* bad)
{
    constexpr int W = ValueChunk<D>::W;
    const int other = (lane & 7) >> 2;
    bool odd = false;
#pragma unroll 2
    for (int it = 0; it < 4; ++it) {
        const ValueChunk<D> c(block0, it, lane);
        const uint8_t* at = c.codes(code_tile);
        uint32_t code[2 * W];
        if constexpr (W == 2) {
            const uint4 y = *reinterpret_cast<const uint4*>(at);
            // (lanes of the other half of the dimensions store their pieces the other way round: different banks)
            code[0] = other ? y.y : y.x; code[1] = other ? y.x : y.y;
            code[2] = other ? y.w : y.z; code[3] = other ? y.z : y.w;
        } else {
            const uint2 y = *reinterpret_cast<const uint2*>(at);
            code[0] = y.x; code[1] = y.y;
        }
        const uint32_t sc = c.scales(code_tile);
#pragma unroll
        for (int tok = 0; tok < 2; ++tok) {
            uint32_t s2 = __byte_perm(sc, 0, tok ? 0x3232 : 0x1010);
            const int node = behind + c.row(tok);
            if (kEnds && node >= 0) {
                if (node >= nodes) {
                    s2 = 0;
                } else if ((s2 & 0x7fffu) > 0x7154u) {  // (whatever the code, none below it gives an infinity)
                    odd = true;
                    s2 = 0;
                }
            }
#pragma unroll
            for (int y = 0; y < W; ++y) {
                uint32_t f[4];
                e2m1x8_to_f16x2(code[tok * W + y], f);
                *reinterpret_cast<uint4*>(c.piece(to, tok, W == 2 ? y ^ other : y)) =
                    make_uint4(hmul2(f[0], s2), hmul2(f[1], s2), hmul2(f[2], s2), hmul2(f[3], s2));
            }
        }
    }
    if (kEnds && odd) widen_odd_values<D>(code_tile, to, block0, lane, behind, nodes, bad);
}

// Eight warps widen a block of keys each, four two blocks of values.  (A tile's second operand of keys has one buffer: the next tile's wait
// for this one's product, by halves.  When the second operand was f16, short runs: 64 requests of 8 nodes 180 us, 32 of 64 nodes 461, with
// four warps for keys and whole tiles 224 and 568.)
template <int D, int P>
__device__ __forceinline__ void widen_role(Smem<D, true>& sm, const TreeArgs& a, Walk w, int warp, int lane)
{
    using C = Cfg<D, true>;
    static_assert(C::kKeyWarps == C::kBlocks && 2 * C::kValueWarps == C::kBlocks, "a block of keys or two of values");
    int* gave_up = &sm.gave_up;
    const bool values = warp >= C::kKeyWarps;
    const int block0 = values ? 2 * (warp - C::kKeyWarps) : warp, half = warp / (C::kKeyWarps / 2);  // (of keys)
    uint32_t tile = 0, n_unit = 0;
    do {
        for (int j = 0; j < w.tiles; ++j, ++tile) {
            const int behind = (w.tile0 + j) * kTile - w.committed();
            const uint32_t seq = 2 * tile + values, s = seq % C::kSlots, c = tile % C::kCodeSlots;
            if (!warp_wait(&sm.code_full[c], (tile / C::kCodeSlots) & 1, gave_up)) return;
            if (seq >= C::kSlots && !warp_wait(&sm.empty[s], ((seq / C::kSlots) - 1) & 1, gave_up)) return;
            if (!values && tile > 0 && !warp_wait(&sm.rest_empty[half], (tile - 1) & 1, gave_up)) return;
            const uint8_t* from = sm.code + c * C::kCodeBytes;
            if (!values) widen_keys<D>(from, sm.slot[s], sm.rest, block0, lane);
            else if (behind + kTile <= 0) widen_values<D, false>(from, sm.slot[s], block0, lane, behind, w.q.nodes, nullptr);
            else widen_values<D, true>(from, sm.slot[s], block0, lane, behind, w.q.nodes, &sm.bad[n_unit & 7]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(values ? &sm.full[s] : &sm.key_full[s][half]);
                mbar_arrive(&sm.code_empty[c]);
            }
        }
        ++n_unit;
    } while (w.next(a, sm.part));
}

template <int D, bool F4, int P>
__global__ void __launch_bounds__(Cfg<D, F4>::kThreads, 1)
tree_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const TreeArgs a)
{
    using C = Cfg<D, F4>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem<D, F4>& sm = *reinterpret_cast<Smem<D, F4>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    dependents_may_launch();
    if ((smem_u32(smem_raw) & 1023u) != 0) {  // (operand tiles lie on 1024-byte boundaries)
        if (tid == 0) atomicMin(a.kv.status, (int)MOSKA_ERR_CUDA);
        if (tid == 0 && a.cut != nullptr) a.cut[blockIdx.x] = CutUnit{};
        return;
    }
    if (tid < kFindThreads) {
        find_part<(P > 1 ? 1 : kMaxRowTiles)>(a, blockIdx.x, gridDim.x, sm.part);
    } else if (warp == C::kLoadWarp && lane == 0) {
        for (int s = 0; s < C::kSlots; ++s) {
            mbar_init(&sm.full[s], F4 ? C::kValueWarps : 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int x = 0; x < C::kCodeSlots; ++x) {
            mbar_init(&sm.code_full[x], 1);
            mbar_init(&sm.code_empty[x], C::kWidenWarps);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sm.q_full[x], kTileRows);
            mbar_init(&sm.stat_full[x], C::kGroups * kTileRows);
        }
        for (int x = 0; x < C::kGroups; ++x)
            for (int y = 0; y < 4; ++y) mbar_init(&sm.ref_full[x][y], 32);
        for (int x = 0; x < 4; ++x) {
            mbar_init(&sm.s_full[x], 1);
            mbar_init(&sm.p_full[x], kTileRows);
            mbar_init(&sm.pv_done[x], 1);
        }
        mbar_init(&sm.o_full, 1);
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sm.rest_empty[x], 1);
            for (int s = 0; s < C::kSlots; ++s) mbar_init(&sm.key_full[s][x], C::kKeyWarps / 2);
        }
        mbar_init(&sm.o_free, kTileRows);
        for (int x = 0; x < 8; ++x) sm.bad[x] = 0;
        sm.step = 0;
        sm.gave_up = 0;
        fence_mbar_init();
        fence_proxy_async_smem();
    } else if (warp == C::kScoreWarp) {
        tmem_alloc(&sm.tmem_base, 512);
        tmem_relinquish();
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sm.tmem_base;

    Walk w;
    const bool any = w.begin(a, sm.part);
    if (warp == C::kValueWarp + 1 && lane == 0 && a.cut != nullptr) {
        CutUnit u{};
        if (any && w.tile0 > 0) {
            u = {w.q.first + w.node0(a), w.h, w.rows(a), sm.part.cta0 + w.first_cta(sm.part), sm.part.cta0 + w.last_cta(sm.part), {}};
            if ((int)blockIdx.x != u.c0 + 1) u.rows = 0;
        }
        a.cut[blockIdx.x] = u;
    }
    if (any) {
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const int row = (warp & 3) * 32 + lane;
        if (warp < C::kRowWarp0) {
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
            softmax_role<D, F4, P>(sm, lanes, warp >> 2, warp, row);
        } else if (warp < C::kLoadWarp) {
            if constexpr (C::kRowRegs > C::kLaunchRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRowRegs));
            Rows<D, F4, P>{sm, a, lanes, row}.run(w);
        } else if (warp < C::kWidenWarp0) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kIssueRegs));
            if (warp == C::kLoadWarp) load_role<D, F4>(sm, tm_k, tm_v, a, w, lane);
            else if (warp == C::kScoreWarp) score_role<D, F4>(sm, tmem);
            else if (warp == C::kValueWarp) value_role<D, F4>(sm, tmem);
        } else {
            if constexpr (F4) {
                asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kWidenRegs));
                widen_role<D, P>(sm, a, w, warp - C::kWidenWarp0, lane);
            }
        }
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == C::kScoreWarp) tmem_dealloc(tmem, 512);
    if (tid == 0 && sm.gave_up) atomicMin(a.kv.status, (int)MOSKA_ERR_TIMEOUT);
}

// Joins the partial rows of a unit that cuts divide: kJoinCtas CTAs a cut, with 16 rows each, two a warp.  (Where a cut falls is
// written down: found anew here by all CTAs, each call took 2 to 10 us longer.)
constexpr int kJoinCtas = 8;
template <int D>
__global__ void __launch_bounds__(256) tree_join_kernel(const TreeArgs a)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wait_for_results();
    const CutUnit unit = a.cut[blockIdx.x / kJoinCtas + 1];  // (no unit's second part is the first CTA's)
    const int G = a.Hq / a.Hkv, rows = unit.rows, c0 = unit.c0, c1 = unit.c1;
    constexpr int W = D / 32;  // dimensions a lane
    using Vec = typename std::conditional<W == 4, float4, float2>::type;
    const int i0 = (blockIdx.x % kJoinCtas) * (kTileRows / kJoinCtas) + warp;  // and i0 + 8
    auto slot = [&](int c, int x) { return (int64_t)(2 * c + (c == c0 ? 1 : 0)) * kTileRows + i0 + 8 * x; };
    if (i0 >= rows) return;
    float top[2] = {-INFINITY, -INFINITY};
    for (int c = c0 + lane; c <= c1; c += 32)
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (i0 + 8 * x < rows) top[x] = max_or_nan(top[x], a.lse_cut[slot(c, x)]);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) top[x] = max_or_nan(top[x], __shfl_xor_sync(0xffffffffu, top[x], off));
    float total[2] = {}, acc[2][W] = {};
    constexpr int kAtOnce = 4;
    for (int c = c0; c <= c1; c += kAtOnce) {
        Vec o[kAtOnce][2];
        float weight[kAtOnce][2];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (c + u > c1 || i0 + 8 * x >= rows) continue;
                weight[u][x] = a.lse_cut[slot(c + u, x)];
                o[u][x] = *reinterpret_cast<const Vec*>(a.o_cut + slot(c + u, x) * D + W * lane);
            }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (c + u > c1 || i0 + 8 * x >= rows) continue;
                // (all parts empty: every weight is 0)
                const float y = __expf(weight[u][x] - (top[x] == -INFINITY ? 0.f : top[x]));
                total[x] += y;
#pragma unroll
                for (int e = 0; e < W; ++e) acc[x][e] = fmaf(y, reinterpret_cast<const float*>(&o[u][x])[e], acc[x][e]);
            }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int i = i0 + 8 * x;
        if (i >= rows) continue;
        const float inv = total[x] == 0.f ? 0.f : 1.f / total[x];
        const int64_t row = (int64_t)(unit.first + i / G) * a.Hq + unit.h * G + i % G;
#pragma unroll
        for (int e = 0; e < W; e += 2)
            *reinterpret_cast<uint32_t*>(a.out + row * D + W * lane + e) = bf16x2(acc[x][e] * inv, acc[x][e + 1] * inv);
        if (lane == 0 && a.lse_out != nullptr) a.lse_out[row] = top[x] == -INFINITY ? -INFINITY : top[x] + logf(total[x]);
    }
}

// ---- host side ------------------------------------------------------------------------------------
// Pages as [tokens][Hkv][D]: boxes of 64 dimensions of one head, a page's tokens or 128 of them.
int make_page_map(CUtensorMap* tm, const void* pool, const PagedView& kv, int Hkv, int D)
{
    EncodeTiledFn enc = nullptr;
    MOSKA_TRY_STATUS(tensor_map_encoder(&enc));
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

int default_tree_splits(int n_requests, int nodes, int G, int Hkv, int max_len)
{
    // slots for the parts that equal contexts are cut into: the CTAs that share a unit's tiles, and one more
    const long long row_tiles = (nodes + kTileRows / G - 1) / (kTileRows / G), units = (long long)n_requests * Hkv * row_tiles;
    const long long tiles = ((long long)max_len + kTile - 1) / kTile;
    long long s = (kMaxCtas + units - 1) / units + 1;
    if (s > tiles) s = tiles;
    return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

size_t tree_cut_bytes(int D)
{
    return kMaxCtas * (2 * kTileRows * (D + 1) * sizeof(float) + sizeof(CutUnit));
}

int launch_tree_attn(const uint16_t* q, const PagedView& kv, bool fp4, const TreeRows& tree, float* o_part, float* lse_part,
                     int slot0, int n_slots, uint16_t* out, float* lse_out, void* ws, float scale, const moska_shape* s,
                     cudaStream_t st)
{
    if (tree.n_rows == 0) return MOSKA_OK;
    const int G = s->Hq / s->Hkv, per_tile = kTileRows / G, row_tiles = (tree.max_nodes + per_tile - 1) / per_tile;
    if (((long long)kv.n_pages << kv.page_shift) > 0x7fffffffLL)
        return fail(MOSKA_ERR_UNSUPPORTED, "a pool of more than 2^31 tokens");
    if (tree.n_requests >= 1 << (62 - kUnitBit)) return fail(MOSKA_ERR_UNSUPPORTED, "%d requests", tree.n_requests);
    TreeArgs a{q, kv, tree, o_part, lse_part, out, lse_out, nullptr, nullptr, nullptr, scale, s->Hq, s->Hkv, s->n_unique_splits, slot0,
               n_slots, row_tiles, per_tile};
    if (ws != nullptr) {
        a.o_cut = static_cast<float*>(ws);
        a.lse_cut = a.o_cut + (size_t)kMaxCtas * 2 * kTileRows * s->D;
        a.cut = reinterpret_cast<CutUnit*>(a.lse_cut + kMaxCtas * 2 * kTileRows);
    }
    CUtensorMap tm_k{}, tm_v{};
    if (!fp4) {
        MOSKA_TRY_STATUS(make_page_map(&tm_k, kv.k, kv, s->Hkv, s->D));
        MOSKA_TRY_STATUS(make_page_map(&tm_v, kv.v, kv, s->Hkv, s->D));
    }
    int dev = 0, n_sms = 0;
    MOSKA_CUDA_TRY(cudaGetDevice(&dev));
    MOSKA_CUDA_TRY(cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev));
    // a multiple of the row tiles: trees of one size are cut alike in each
    const int ctas = (n_sms < kMaxCtas ? n_sms : kMaxCtas) / row_tiles * row_tiles;
    auto go = [&](auto kernel, int threads, int smem) {
        MOSKA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        kernel<<<(unsigned)ctas, threads, smem, st>>>(tm_k, tm_v, a);
        MOSKA_LAUNCH_CHECK("tree_attn_kernel");
        return (int)MOSKA_OK;
    };
    const int rows = tree.max_nodes * G;  // of the largest unit, if there is one row tile
    auto form = [&](auto d, auto f4) {
        constexpr int D = decltype(d)::value;
        constexpr bool F4 = decltype(f4)::value;
        auto kernel = tree_attn_kernel<D, F4, 1>;
        if constexpr (F4)
            kernel = rows <= Spread<4>::kRows ? tree_attn_kernel<D, F4, 4> : rows <= Spread<2>::kRows ? tree_attn_kernel<D, F4, 2> : kernel;
        return go(kernel, Cfg<D, F4>::kThreads, (int)sizeof(Smem<D, F4>));
    };
    const std::integral_constant<int, 128> d128;
    const std::integral_constant<int, 64> d64;
    if (s->D == 128) MOSKA_TRY_STATUS(fp4 ? form(d128, std::true_type{}) : form(d128, std::false_type{}));
    else MOSKA_TRY_STATUS(fp4 ? form(d64, std::true_type{}) : form(d64, std::false_type{}));
    if (out == nullptr || s->n_unique_splits == 1 || ctas < 2) return MOSKA_OK;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)(kJoinCtas * (ctas - 1)));
    config.blockDim = dim3(256);
    config.stream = st;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    MOSKA_CUDA_TRY(cudaLaunchKernelEx(&config, s->D == 128 ? tree_join_kernel<128> : tree_join_kernel<64>, a));
    return MOSKA_OK;
}

}  // namespace moska
