// The accepted path's entries of the cache move behind the committed tokens (spec_cache_commit).
#pragma once
#include "tree.cuh"

namespace specv {
namespace commit {

constexpr int NT = 256;

struct Params {
    TreeArgs tree;
    int B, caches, num_blocks, block, width, per;      // per: caches that a CTA goes through
    unsigned char *cache;
    long long stride[3];
    unsigned words;                                    // of type W in a row
    const int *table;
    long long table_stride;
    const int *accepted;
    int *lengths_out, *status;
};

// A CTA per request and `per` caches; a thread moves the words of one place of a row along the whole path.  Path nodes have rising indices
// with node(d) >= d, so entry len + d, written at depth d, may be read at depths up to d only: a thread that reads ahead of its
// writes in rising order is right without a second buffer, and no other thread touches its words.  8 requests, 64 caches of 2 KB rows
// (7 MB): 5.0 us; 128 requests, 24 caches of 1 KB rows (26 MB): 5.9, with divisions of 64 bits 6.7 (floors 1.1 and 3.9); the path has to be
// found before the first byte moves.
template <typename W>
__global__ void __launch_bounds__(NT) spec_commit_kernel(const Params P)
{
    grid_dependency_wait();
    __shared__ int parent[SPEC_MAX_NODES];
    __shared__ long long from[SPEC_MAX_NODES], to[SPEC_MAX_NODES];
    __shared__ int s_moves, s_depth;
    const int tid = threadIdx.x, b = blockIdx.y;
    const int len = __ldg(P.tree.lengths + b), acc = __ldg(P.accepted + b), n = len < 0 ? 0 : tree_nodes(P.tree, b);
    bool bad = n < 0;
    const int *row = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
    for (int i = tid; i < n; i += NT) {
        const int p = __ldg(row + i);
        bad |= i == 0 ? p != -1 : p < 0 || p >= i;
        parent[i] = p;
    }
    const bool idle = len < 0 || acc == -1;
    if (!idle) bad |= acc < 0 || acc >= n;
    bad = __syncthreads_or(bad) != 0;
    const bool out = blockIdx.x == 0 && tid == 0;
    if (idle || bad) {
        if (out) {
            P.lengths_out[b] = len;
            P.status[b] = len >= 0 && bad ? SPEC_DEV_TOPOLOGY : SPEC_DEV_OK;
        }
        return;
    }
    // the path upwards, then its nodes that move, downwards: from[] and to[] hold them as node and depth first
    if (tid == 0) {
        int depth = 0;
        for (int i = acc; i > 0; i = parent[i]) ++depth;
        int moves = 0, d = depth;
        for (int i = acc; i > 0 && i != d; i = parent[i], --d) { from[moves] = i; to[moves] = d; ++moves; }
        s_depth = depth; s_moves = moves;              // (above a node that stays, i = d, all stay: an ancestor's index is below, its depth one less)
    }
    __syncthreads();
    const int moves = s_moves;
    const int *table = P.table + (long long)b * P.table_stride;
    const auto offset = [&](long long at) -> long long {
        if (at > 0x7FFFFFFFll) return -1;              // (32 bits from here: a division of 64 costs more than the load)
        const unsigned col = (unsigned)at / (unsigned)P.block, in = (unsigned)at - col * (unsigned)P.block;
        const int id = col < (unsigned)P.width ? __ldg(table + col) : -1;
        return id < 0 || id >= P.num_blocks ? -1 : id * P.stride[1] + in * P.stride[2];
    };
    // the path's entries, those that stay in place too, have to have blocks, or a length would count what the cache cannot hold
    bool page = (long long)len + s_depth >= 0x7FFFFFFFll;
    for (int i = tid; i <= s_depth; i += NT) {         // (fewer move than the path has)
        const bool moved = i < moves;
        const long long at = offset((long long)len + i);
        const long long x = offset(len + (moved ? from[i] : i)), y = offset(len + (moved ? to[i] : i));
        page |= at < 0 || x < 0 || y < 0;
        if (moved) { from[i] = x; to[i] = y; }
    }
    page = __syncthreads_or(page) != 0;
    if (out) {
        P.lengths_out[b] = page ? len : len + s_depth + 1;
        P.status[b] = page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
    }
    if (page) return;
    const int c0 = blockIdx.x * P.per, c1 = min(P.caches, c0 + P.per);
    const unsigned all = (unsigned)(c1 - c0) * P.words;
    constexpr int AHEAD = 8;
    for (unsigned w = tid; w < all; w += NT) {
        const unsigned cache = w / P.words, word = w - cache * P.words;
        unsigned char *base = P.cache + (long long)(c0 + (int)cache) * P.stride[0] + (long long)word * (long long)sizeof(W);
        for (int m = moves; m > 0; m -= AHEAD) {       // (stored downwards: the last is the path's first)
            W x[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) if (k < m) x[k] = *(const W *)(base + from[m - 1 - k]);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) if (k < m) *(W *)(base + to[m - 1 - k]) = x[k];
        }
    }
}

}  // namespace commit
}  // namespace specv
