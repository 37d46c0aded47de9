// Trees of drafted tokens on the device: a request's rows, and which nodes a node sees (include/moska.h has
// the definition).
#pragma once

#include "paged.cuh"

namespace moska {

static_assert(MOSKA_TREE_MAX_NODES == 64, "a node's ancestors are the bits of a 64-bit word");

// First row and number of nodes of request r (rows outside the batch or more nodes than there may be are reported, and
// make *sound false).
__device__ __forceinline__ int2 tree_rows(const TreeRows& t, int r, int* status, bool* sound = nullptr)
{
    if (sound != nullptr) *sound = true;
    if (t.row_start == nullptr) return make_int2(r * t.max_nodes, t.max_nodes);
    const int a = __ldg(t.row_start + r), b = __ldg(t.row_start + r + 1);
    if (a < 0 || b < a || b > t.n_rows || b - a > t.max_nodes) {
        atomicMin(status, MOSKA_ERR_INVALID_ARG);
        if (sound != nullptr) *sound = false;
        if (a < 0 || b < a || b > t.n_rows) return make_int2(0, 0);
        return make_int2(a, t.max_nodes);
    }
    return make_int2(a, b - a);
}

// Parent of node i (< n) of the request whose rows begin at `first`; one that does not come before it is
// reported and counts as none.
__device__ __forceinline__ int tree_parent(const TreeRows& t, int first, int i, int* status)
{
    if (t.parents == nullptr) return i - 1;
    const int p = __ldg(t.parents + first + i);
    if (p >= -1 && p < i) return p;
    atomicMin(status, MOSKA_ERR_INVALID_ARG);
    return -1;
}

// For the first two warps of a CTA together (thread i: node i; all 64 call it, between two barriers of the
// CTA that the caller sees to): bits of the nodes that node i sees.  Ancestors double each round: after k of
// them a node has its 2^k nearest, itself among them.
struct TreeSmem {
    unsigned long long bits[MOSKA_TREE_MAX_NODES];
    int up[MOSKA_TREE_MAX_NODES];
};

template <class Sync>
__device__ __forceinline__ void tree_ancestors(TreeSmem& sm, int i, int parent, Sync sync)
{
    unsigned long long mine = 1ull << i;
    int up = parent;
#pragma unroll 1
    for (int round = 0; round < 6; ++round) {
        sm.bits[i] = mine;
        sm.up[i] = up;
        sync();
        if (up >= 0) {
            mine |= sm.bits[up];
            up = sm.up[up];
        }
        sync();
    }
    sm.bits[i] = mine;
}

}  // namespace moska
