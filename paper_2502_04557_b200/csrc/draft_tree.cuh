// The nodes that one pass of the target model works on: a chain of drafted tokens, or a tree.
//
// Sequence b has T nodes, of which the first count are used.  parents[b*T + i] is the node that node i follows, or
// negative where it follows the cached prefix; a parent comes before its children.  No parents: a chain, node i
// follows node i - 1.  Node i lies in slot lens[b] + i of the sequence and at position lens[b] + depth(i).
#pragma once

#include "common.cuh"

namespace spr {

constexpr int kMaxTreeNodes = 256;       // nodes of a tree (chains may be longer where nothing looks at paths)

struct DraftNodes {
    const int32_t *lens;      // [B] tokens in the cache before this pass; negative: the sequence is not used
    const int32_t *counts;    // [B] or null: T
    const int32_t *parents;   // [B,T] or null: a chain
    int T;
};

#ifdef __CUDACC__

__device__ __forceinline__ int node_count(const DraftNodes &n, int b)
{
    return n.counts ? min(max(__ldg(n.counts + b), 0), n.T) : n.T;
}

// Parent of node i as it counts: one that does not come before its child is an error, and the child then follows
// the prefix.  Any walk along parents ends, whatever they hold.
__device__ __forceinline__ int checked_parent(int p, int i, int *status)
{
    if (p < i) return p < 0 ? -1 : p;
    raise_status(status, SPR_ERR_BAD_TREE);
    return -1;
}

#endif

}  // namespace spr
