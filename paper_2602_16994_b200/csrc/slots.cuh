// Blocks, slots and positions of a step (spec_cache_slots).
#pragma once
#include "tree.cuh"

namespace specv {
namespace slots {

// A warp per request.  What a request is given depends on what the ones before it lack: every CTA adds that up by itself, from two or three
// words per request, instead of waiting for the others (2048 requests: up to 8 requests per thread, all in L2 after the first CTA), and one more CTA
// adds up all of them for what is left of the ring.  The call is bound by the latency of its launch and of two dependent loads
// (lengths, then table or ring): 5.7 us for 8 requests, 7.8 for 2048 (9.1 with divisions of 64 bits; 7.7 and 13.4 with the totals behind a CTA's
// requests).
constexpr int WARPS = 8, NT = WARPS * 32;

struct Params {
    TreeArgs tree;
    int B, block, width, free_size;
    int *table;
    long long table_stride;
    const int *owned, *ring, *range;
    int *slots, *positions, *owned_out, *range_out, *status;
};

// Blocks that request b lacks; *fit: its row of the table has room for all its columns.
__device__ __forceinline__ int lacks(const Params &P, int b, bool *fit)
{
    const int len = __ldg(P.tree.lengths + b), own = __ldg(P.owned + b);
    const int n = max(0, tree_nodes(P.tree, b));
    // (in 32 bits: len and n are below 2^31, and a division of 64 costs several of 32)
    const unsigned end = len < 0 ? 0u : (unsigned)len + (unsigned)n, cols = end == 0u ? 0u : (end - 1u) / (unsigned)P.block + 1u;
    *fit = len < 0 || (own >= 0 && own <= P.width && cols <= (unsigned)P.width && end <= 0x7FFFFFFFu);
    return len < 0 || !*fit ? 0 : max(0, (int)cols - own);
}

__device__ __forceinline__ long long block_sum(long long v, long long *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    long long s = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += part[w];
    __syncthreads();
    return s;
}

__global__ void __launch_bounds__(NT) spec_slots_kernel(const Params P)
{
    grid_dependency_wait();
    __shared__ long long part[WARPS];
    __shared__ int mine[WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b0 = blockIdx.x * WARPS, b = b0 + warp;
    int begin = P.free_size ? __ldg(P.range) : 0, count = P.free_size ? __ldg(P.range + 1) : 0;
    if (begin < 0 || begin >= P.free_size || count < 0 || count > P.free_size) begin = count = 0;
    bool fit;
    if (blockIdx.x == gridDim.x - 1) {
        // one CTA more: blocks taken by all, the largest running sum that the ring has; a run of requests per thread
        const int per = (P.B + NT - 1) / NT, i0 = min(P.B, tid * per), i1 = min(P.B, i0 + per);
        long long run = 0;
#pragma unroll 4
        for (int i = i0; i < i1; ++i) run += lacks(P, i, &fit);
        long long incl = run;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        __syncthreads();
        if (lane == 31) part[warp] = incl;
        __syncthreads();
        long long at = incl - run, best = 0;
        for (int w = 0; w < warp; ++w) at += part[w];
#pragma unroll 4
        for (int i = i0; i < i1; ++i) {
            at += lacks(P, i, &fit);
            if (at <= count) best = at;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        __syncthreads();
        if (lane == 0) part[warp] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < WARPS; ++w) best = max(best, part[w]);
            P.range_out[0] = P.free_size ? (int)((begin + best) % P.free_size) : 0;
            P.range_out[1] = (int)(count - best);
        }
        return;
    }
    long long before = 0;
#pragma unroll 4
    for (int i = tid; i < b0; i += NT) before += lacks(P, i, &fit);
    before = block_sum(before, part);
    const int lack = b < P.B ? lacks(P, b, &fit) : 0;
    if (lane == 0) mine[warp] = lack;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += mine[w];
    if (b < P.B) {
        const int len = __ldg(P.tree.lengths + b), n_or_bad = tree_nodes(P.tree, b), n = max(0, n_or_bad);
        const bool enough = lack == 0 || before + lack <= count;
        const int own = __ldg(P.owned + b), got = enough ? lack : 0;
        int *row = P.table + (long long)b * P.table_stride;
        const auto fresh = [&](int i) {                          // (begin + before + i < 2 free_size: what is taken is there)
            const long long at = begin + before + i;
            return __ldg(P.ring + (at < P.free_size ? at : at - P.free_size));
        };
        for (int i = lane; i < got; i += 32) row[own + i] = fresh(i);
        const int *parent = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
        volatile uint32_t *depth = (volatile uint32_t *)dyn_smem + (long long)warp * P.tree.N;
        const bool live = len >= 0, placed = live && fit && enough;
        const bool sound = !live || tree_depths(parent, n, depth, lane, 32, AnyInWarp());
        bool page = false;
        for (int i = lane; i < P.tree.N; i += 32) {
            int slot = -1;
            if (placed && i < n) {
                const unsigned at = (unsigned)len + (unsigned)i;             // (below 2^31: the row fits)
                const int col = (int)(at / (unsigned)P.block);
                const int id = col < own ? row[col] : fresh(col - own);
                const long long s = (long long)id * P.block + (int)(at - (unsigned)col * (unsigned)P.block);
                if (id < 0 || s > 0x7FFFFFFFll) page = true;
                else slot = (int)s;
            }
            P.slots[(long long)b * P.tree.N + i] = slot;
            P.positions[(long long)b * P.tree.N + i] = placed && sound && i < n ? len + (int)depth[i] : -1;
        }
        page = __any_sync(0xffffffffu, page);
        if (lane == 0) {
            P.owned_out[b] = own + got;
            P.status[b] = !live ? SPEC_DEV_OK
                          : n_or_bad < 0 ? SPEC_DEV_TOPOLOGY
                          : !placed ? SPEC_DEV_BLOCKS : page ? SPEC_DEV_PAGE : sound ? SPEC_DEV_OK : SPEC_DEV_TOPOLOGY;
        }
    }
}

}  // namespace slots
}  // namespace specv
