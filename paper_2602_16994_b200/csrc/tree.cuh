// Draft trees on chip: validation, depths and paths from the array of parents (shared by the operators around a verification).
#pragma once
#include "common.cuh"

namespace specv {

// What the operators read of a request's tree: its nodes (n_nodes[b], or N) and parents.
struct TreeArgs {
    int N;
    const int *lengths, *n_nodes, *parent;
    long long topo_seq_stride;
};
// number of nodes; -1 where n_nodes is out of range
__device__ __forceinline__ int tree_nodes(const TreeArgs &t, int b)
{
    if (!t.n_nodes) return t.N;
    const int n = __ldg(t.n_nodes + b);
    return n < 0 || n > t.N ? -1 : n;
}

// A node's word: the ancestor it has got to in the upper half (NO_NODE: it has passed the root), the steps to it in the lower.
constexpr uint32_t NO_NODE = 0xFFFFu;
// Depths by pointer doubling, words in shared memory, by `threads` threads that `sync` joins: every pass doubles the distance that a word
// spans, so a chain of 1024 nodes takes ten passes and a draft tree of depth 8 three.  A word is read and written whole, so it holds a
// valid pair whatever the order of the updates.  Returns false (to all) for a bad tree; depth of node i: words[i].
template <typename Any>
__device__ __forceinline__ bool tree_depths(const int *parent, int n, volatile uint32_t *words, int tid, int threads, Any any)
{
    bool bad = false;
    for (int i = tid; i < n; i += threads) {
        const int p = __ldg(parent + i);
        bad |= i == 0 ? p != -1 : p < 0 || p >= i;
        words[i] = i == 0 ? NO_NODE << 16 : ((uint32_t)p << 16) | 1u;
    }
    if (any(bad)) return false;
    for (;;) {
        bool more = false;
        for (int i = tid; i < n; i += threads) {
            const uint32_t w = words[i], a = w >> 16;
            if (a == NO_NODE) continue;
            const uint32_t up = words[a];
            words[i] = (up & 0xFFFF0000u) | ((w & 0xFFFFu) + (up & 0xFFFFu));
            more |= (up >> 16) != NO_NODE;
        }
        if (!any(more)) break;
    }
    for (int i = tid; i < n; i += threads) words[i] = words[i] & 0xFFFFu;
    any(false);
    return true;
}
// the join of a warp: every thread gets whether any of them says so, and sees what the others stored
struct AnyInWarp {
    __device__ bool operator()(bool x) const { __syncwarp(); return __any_sync(0xffffffffu, x); }
};

}  // namespace specv
