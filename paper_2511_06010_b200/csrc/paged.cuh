// The paged private store on the device: where a context token lives, and the byte layout of a
// 16-token block of the 4-bit format (include/moska.h has the definition).
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace moska {

constexpr int kBlockTokens = 16;        // tokens of a 4-bit block, and of a streaming tile
constexpr float kFp4MaxScale = 10912.f; // largest f16 whose sixfold is finite in f16

// moska_paged_kv as the kernels take it (page_size is a power of two: 1 << page_shift).
struct PagedView {
    uint8_t* k;
    uint8_t* v;
    const int32_t* page_table;
    const int32_t* kv_len;
    int32_t n_pages;
    int32_t max_pages;
    int32_t page_shift;
    int* status;  // the device status word
};

__host__ __device__ constexpr int fp4_block_bytes(int D) { return 18 * D; }

// Byte offsets inside a 4-bit block.
template <int D>
struct Fp4Block {
    static_assert(D == 64 || D == 128, "head dimension");
    static constexpr int kBytes = fp4_block_bytes(D);
    static constexpr int kGroups = D / 32;  // scales of a token row
    static constexpr int kV = 8 * D, kKScale = 16 * D, kVScale = 17 * D;
    // position of value chunk x (D / 8 dimensions of both tokens of pair p) inside the pair's row
    static __host__ __device__ constexpr int v_swap(int p) { return D == 128 ? 2 * (p & 3) : 4 * ((p >> 1) & 1); }
    // first byte of dimensions d .. d + 7 (d a multiple of 8) of token t: four bytes
    static __host__ __device__ constexpr int k_byte(int t, int d)
    {
        return t * (D / 2) + ((d & 31) >> 3) * (D / 8) + (d >> 5) * 4;
    }
    static __host__ __device__ constexpr int v_byte(int t, int d)
    {
        return kV + (t >> 1) * D + ((d / (D / 8)) ^ v_swap(t >> 1)) * (D / 8) + (t & 1) * (D / 16) + (d % (D / 8)) / 2;
    }
    static __host__ __device__ constexpr int k_scale(int t, int group) { return kKScale + 2 * (t * kGroups + group); }
    static __host__ __device__ constexpr int v_scale(int t, int group) { return kVScale + 2 * (group * 16 + t); }
};

// A context length cut to what a page-table row can hold (reported where it was not inside).
__device__ __forceinline__ int checked_len(const PagedView& p, int len)
{
    const long long most = (long long)p.max_pages << p.page_shift;
    if (len < 0 || len > most) {
        atomicMin(p.status, MOSKA_ERR_INVALID_ARG);
        return len < 0 ? 0 : (int)most;
    }
    return len;
}

__device__ __forceinline__ int paged_len(const PagedView& p, int r) { return checked_len(p, __ldg(p.kv_len + r)); }

// Attention takes the requests longest context first, so that no CTA of a long one starts when the others
// are done (default splits: 4 bits, 64 requests of 1K to 32K 260 -> 242 us, 48 x 4 query tokens 82 -> 64 us; bf16, 64
// requests of 1K to 32K 703 -> 640 us).  More requests than threads are many CTAs to a place and stay in order.
constexpr int kMaxOrdered = 128;
struct OrderSmem {
    uint4 key[kMaxOrdered / 8];
    int request, len;
};

// The request that is `rank`-th (equal lengths: in order) and its length; for all kMaxOrdered threads of a
// CTA.  Every CTA ranks the lengths by itself, a request a thread: blocks of 16 tokens as 16-bit keys, two
// compared at once.
__device__ __forceinline__ int request_at(const PagedView& p, int n, int rank, OrderSmem& sm, int& len)
{
    const int i = threadIdx.x;
    const int first = __ldg(p.kv_len), mine = i < n ? __ldg(p.kv_len + i) : first;
    const int key = i < n ? min(max(mine >> 4, 0), 0x7ffd) : -1;
    reinterpret_cast<int16_t*>(sm.key)[i] = (int16_t)key;
    if (__syncthreads_and(mine == first)) {
        len = checked_len(p, first);
        return rank;
    }
    const uint32_t equal_behind = (uint32_t)(-key & 0xffff) * 0x10001u;        // x - key > 0: larger
    const uint32_t equal_before = (uint32_t)((1 - key) & 0xffff) * 0x10001u;   // x - key + 1 > 0: or equal
    const uint32_t mixed = (equal_behind & 0xffff0000u) | (equal_before & 0xffffu);
    uint32_t before = 0;  // two counts of requests that come before this one
    for (int j = 0; j < n; j += 8) {
        const uint4 x = sm.key[j / 8];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = j + 2 * u;
            before += __viaddmin_s16x2_relu(w[u], at + 1 < i ? equal_before : at < i ? mixed : equal_behind, 0x00010001u);
        }
    }
    if (i < n && (int)((before & 0xffff) + (before >> 16)) == rank) {
        sm.request = i;
        sm.len = mine;
    }
    __syncthreads();
    len = checked_len(p, sm.len);
    return sm.request;
}

// Whether that is worth it: more than a CTA per SM.  (A kernel of its own: ranking in the same one costs one
// context of 8191 tokens 0.8 of 10.4 us.)
inline bool longest_first(long long n_requests, long long grid) { return n_requests > 1 && n_requests <= kMaxOrdered && grid > 148; }

// Page `i` of a page-table row for a read: an index outside the pool is reported and becomes page 0.
__device__ __forceinline__ int paged_page(const PagedView& p, const int32_t* row, int i)
{
    const int page = __ldg(row + i);
    if (static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages)) return page;
    atomicMin(p.status, MOSKA_ERR_INVALID_ARG);
    return 0;
}

// The merge behind an attention kernel is launched while that one runs (programmatic dependent launch):
// its own launch is hidden, and it waits for the results itself.
__device__ __forceinline__ void dependents_may_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_results() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Two E2M1 codes a byte -> two f16 values, exact; the four bytes of w give o[0..3].
__device__ __forceinline__ void e2m1x8_to_f16x2(uint32_t w, uint32_t (&o)[4])
{
    asm("{\n"
        ".reg .b8 b0, b1, b2, b3;\n"
        "mov.b32 {b0, b1, b2, b3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n"
        "}\n"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
        : "r"(w));
}

}  // namespace moska
