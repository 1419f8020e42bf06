// Attention of the nodes of draft trees over a paged cache (spec_tree_attention).
//
// Mathematics.  A unit is a request, a key head and a block of up to 128 MT of the rows (node, query head of the group) that share this
// head's keys.  Over tiles of 128 keys, S = Q K^T, y = scale log2(e) S - ref, P = 2^y, l += sum P, O += P V, with one reference per row: the
// largest y of the row's first tile, replaced (l and O scaled) only when a later y exceeds it by more than 8, so P stays
// below 2^8 and a tile is gone through once.  Tiles run from the last to the first: the tree's tile comes first, where every row sees
// itself.  The result is O / l.
//
// What bounds it.  Per tile and key head 64 KB of keys and values (D = 128): 2740 cycles of an SM's share of the HBM rate.  128 rows
// take 1020 cycles of products and 1024 of exponentials, 256 rows twice that: up to about 250 rows the cache's bytes are the
// bound, so both products go to the tensor cores even for one row (which fills 1 of 128 lanes), and rows share a lane each: a thread owns a row,
// and maxima and sums need no exchange.
//
// Balance.  The tiles of all units, in order, are cut into one run per CTA (one CTA per SM), whatever the lengths: a unit that a
// run ends in leaves its O, l and reference in the workspace, and spec_join_kernel puts such parts together.  Every CTA finds its run from
// the lengths by itself; the host never sees them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tmem.cuh"
#include "tree.cuh"

namespace specv {
namespace attend {

constexpr int KT = 128;                        // keys of a tile
constexpr int PANEL = KT * 128;                // bytes of a panel: 128 rows of 64 entries
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

struct Params {
    TreeArgs tree;
    int B, Hq, Hkv, G, num_blocks, block, width, window, sinks;
    float scale;
    const void *q, *k, *v;
    long long q_stride[3], k_stride[3], v_stride[3];
    const int *table;
    long long table_stride;
    void *out;
    long long out_stride[3];
    float *lse;
    int *status;
    int ctas;
    float *part;                               // [ctas][2][D / 4][rows][4] unfinished O
    float2 *ml;                                // [ctas][2][rows] reference and l
    int *late;                                 // [ctas] a wait ran out
};

// ---- the schedule -------------------------------------------------------------------------------------------------------------
// Tiles of a block of rows: [0, sink) and [from, end) of the tiles of its keys.
struct Tiles {
    int sink, from, end;
    __device__ __forceinline__ int count() const { return sink + end - from; }
    __device__ __forceinline__ int tile(int i) const { return i < sink ? i : from + i - sink; }
};
struct Request {
    int len, n, rows;                          // (n = 0 for idle requests)
};
__device__ __forceinline__ Request request_of(const Params &P, int b)
{
    Request r;
    r.len = __ldg(P.tree.lengths + b);
    r.n = r.len < 0 ? 0 : max(0, tree_nodes(P.tree, b));
    r.rows = r.n * P.G;
    return r;
}
__device__ __forceinline__ Tiles tiles_of(const Params &P, const Request &r, int m, int block_rows)
{
    const int last = (min(r.rows, (m + 1) * block_rows) - 1) / P.G;          // the block's last node
    Tiles t;
    t.end = (int)(((long long)r.len + last + KT) / KT);
    t.sink = t.from = 0;
    if (P.window) {
        t.sink = min(t.end, (int)(((long long)min(P.sinks, r.len) + KT - 1) / KT));
        t.from = max(0, r.len - P.window + 1) / KT;
        if (t.from < t.sink) t.from = t.sink;
    }
    return t;
}
__device__ __forceinline__ long long tiles_of_request(const Params &P, int b, int block_rows)
{
    const Request r = request_of(P, b);
    long long s = 0;
    for (int m = 0; m * block_rows < r.rows; ++m) s += tiles_of(P, r, m, block_rows).count();
    return s * P.Hkv;
}
__device__ __forceinline__ long long run_start(long long all, int c, int ctas) { return all * c / ctas; }

// A place in the order of all tiles: request, block of rows, key head, tile.
struct Place {
    int b, m, h, i;
};
// All threads of the CTA: the number of tiles; in found[], the request that the start of run `c` falls into and the tiles ahead of it.
__device__ __forceinline__ long long find_request(const Params &P, int block_rows, int c, long long *sums, long long *found, int tid, int threads)
{
    const int per = (P.B + threads - 1) / threads, b0 = min(P.B, tid * per), b1 = min(P.B, b0 + per);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles_of_request(P, b, block_rows);
    const int lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    long long ahead = incl - mine, all = 0;
    for (int w = 0; w < warps; ++w) {
        if (w < warp) ahead += sums[w];
        all += sums[w];
    }
    const long long target = run_start(all, c, P.ctas);
    if (target >= ahead && target < ahead + mine) {
        for (int b = b0; b < b1; ++b) {
            const long long t = tiles_of_request(P, b, block_rows);
            if (target < ahead + t) { found[0] = b; found[1] = ahead; break; }
            ahead += t;
        }
    }
    __syncthreads();
    return all;
}

// The unit that a CTA works on, tiles [begin, end) of it, the last first.
struct Segment {
    int b, m, h, begin, end;
    bool whole, head;                          // all of the unit; begins where the CTA's run does
    Request r;
    Tiles t;
    int rows;                                  // rows of the block
    __device__ __forceinline__ int tile(int step) const { return t.tile(end - 1 - step); }
    __device__ __forceinline__ int steps() const { return end - begin; }
};
struct Run {
    Place at;
    long long left;
    bool first;
    // the next segment of the run; false at its end
    __device__ __forceinline__ bool next(const Params &P, int block_rows, Segment &s)
    {
        if (left <= 0) return false;
        for (;;) {
            s.r = request_of(P, at.b);
            if (at.m * block_rows < s.r.rows) break;
            ++at.b; at.m = 0;
        }
        s.b = at.b; s.m = at.m; s.h = at.h;
        s.t = tiles_of(P, s.r, at.m, block_rows);
        const int count = s.t.count();
        s.begin = at.i;
        s.end = (int)min((long long)count, at.i + left);
        s.whole = s.begin == 0 && s.end == count;
        s.head = first;
        s.rows = min(s.r.rows - at.m * block_rows, block_rows);
        left -= s.end - s.begin;
        first = false;
        at.i = 0;
        if (++at.h == P.Hkv) { at.h = 0; ++at.m; }
        return true;
    }
};
// the place `skip` tiles into request b
__device__ __forceinline__ Place place_in(const Params &P, int b, long long skip, int block_rows)
{
    const Request r = request_of(P, b);
    Place p = {b, 0, 0, 0};
    for (;; ++p.m) {
        const int count = tiles_of(P, r, p.m, block_rows).count();
        if (skip < (long long)count * P.Hkv) {
            p.h = (int)(skip / count);
            p.i = (int)(skip % count);
            return p;
        }
        skip -= (long long)count * P.Hkv;
    }
}

// ---- what a row sees ----------------------------------------------------------------------------------------------------------
// bits of keys a .. a + 31 that lie in [lo, hi)
__device__ __forceinline__ uint32_t bits_of(long long a, long long lo, long long hi)
{
    const int x = (int)min(max(lo - a, 0ll), 32ll), y = (int)min(max(hi - a, 0ll), 32ll);
    if (x >= y) return 0;
    return (y == 32 ? 0xffffffffu : (1u << y) - 1u) & ~((1u << x) - 1u);
}
// Whether every row of any block sees all keys of a tile (a node's depth is at most its index).
__device__ __forceinline__ bool seen_by_all(const Params &P, const Request &r, int tile)
{
    const long long a = (long long)tile * KT, e = a + KT;
    return e <= r.len && (P.window == 0 || e <= P.sinks || a > (long long)r.len + r.n - 1 - P.window);
}
// A row's walk up the tree, as tiles are taken from the last to the first.
struct Walk {
    int node, depth;                           // next node to take, its depth less the row's (0, -1, ...)
};
// The keys of a tile that the row sees; `depth` its depth (used under a window only).
__device__ __forceinline__ void seen_words(const Params &P, const Request &r, int tile, int depth, const unsigned short *parent, Walk &walk,
                                           uint32_t (&words)[4])
{
    const long long a = (long long)tile * KT;
    const long long since = P.window ? (long long)r.len + depth - P.window + 1 : 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        words[w] = bits_of(a + 32 * w, max(since, 0ll), r.len);
        if (P.window) words[w] |= bits_of(a + 32 * w, 0, min(P.sinks, r.len));
    }
    while (walk.node >= 0) {
        const long long at = (long long)r.len + walk.node - a;
        if (at < 0) break;
        if (at < KT && (P.window == 0 || -walk.depth < P.window || (long long)r.len + depth + walk.depth < P.sinks)) {
            const uint32_t bit = 1u << (at & 31);
            const int w = (int)(at >> 5);
#pragma unroll
            for (int i = 0; i < 4; ++i) words[i] |= i == w ? bit : 0u;
        }
        const unsigned short up = parent[walk.node];
        walk.node = up == 0xFFFF ? -1 : up;
        --walk.depth;
    }
}
__device__ __forceinline__ int block_of(const Params &P, int b, long long key)
{
    const long long col = key / P.block;
    const int id = col < P.width ? __ldg(P.table + (long long)b * P.table_stride + col) : -1;
    return id < 0 || id >= P.num_blocks ? -1 : id;
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------
template <int D, int MT> struct Shape {
    static constexpr int PANELS = D / 64;
    static constexpr int ROWS = 128 * MT;
    static constexpr int SLOTS = D == 64 ? 10 : MT == 2 || D == 256 ? 9 : 11;     // panels of keys and values in flight
    static constexpr int LAG = D == 256 ? 1 : D == 128 ? 2 : 3;                    // copies of tiles that a thread has under way
    static constexpr int SOFT = 4 * MT, WARPS = SOFT + 1 + 4, NT = WARPS * 32;    // warps: rows, products, copies
    static constexpr int NP = 128;                                                // threads that copy
    static constexpr int O = 256;                                                 // column of the first O; S buffers at 0 and 128
    static constexpr int off_slots = ROWS * D * 2;
    static constexpr int off_parent = off_slots + SLOTS * PANEL;                  // one array of parents per row warpgroup
    static constexpr int off_rows = off_parent + MT * SPEC_MAX_NODES * 2;         // [2][128] sources of a tile's rows: keys, values
    static constexpr int off_bar = off_rows + 2 * KT * 16;
    static constexpr int total = off_bar + 1024;
    static_assert(total + 1024 <= 227 * 1024, "shared memory");
};
struct Bars {
    uint64_t full[16], empty[16];
    uint64_t q_full, q_empty, s_full[2], p_full[2], pv_done[2], o_empty[2];
    uint32_t tmem;
    int dead, poison;
    uint32_t hidden[8][4];                     // keys of a tile on bad blocks, by the tile's number in the CTA's run % 8
    long long found[2], sums[16];
};
static_assert(sizeof(Bars) <= 1024, "the area behind the buffers");

// A bounded wait; once one has run out all others return at once, and the kernel comes to its end.
__device__ __forceinline__ void wait(Bars *B, uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity)) {
        if (*(volatile int *)&B->dead) return;
        if (clock64() - t0 > WAIT_CYCLES) { *(volatile int *)&B->dead = 1; return; }
    }
}

__device__ __forceinline__ bool mbar_test(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(smem_u32(bar)), "r"(parity)
                 : "memory");
    return ok != 0;
}

template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static constexpr int TYPE = 1;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ bool finite(uint32_t w)                     // both of two entries
    {
        return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u;
    }
    static __device__ __forceinline__ float value(unsigned short x) { return __uint_as_float((uint32_t)x << 16); }
};
template <> struct Pair<__half> {
    static constexpr int TYPE = 0;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ bool finite(uint32_t w) { return (w & 0x7C00u) != 0x7C00u && (w & 0x7C000000u) != 0x7C000000u; }
    static __device__ __forceinline__ float value(unsigned short x) { return __half2float(__ushort_as_half(x)); }
};

// y of 32 columns and what comes of them
template <typename T, bool MASK>
__device__ __forceinline__ void weigh(const uint32_t (&s)[32], uint32_t word, unsigned long long c2, unsigned long long r2, float &top,
                                      unsigned long long &sum, uint32_t *pk)
{
#pragma unroll
    for (int k = 0; k < 32; k += 2) {
        const unsigned long long y2 = fma_f32x2(pack_f32x2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, r2);
        float y0, y1;
        unpack_f32x2(y2, y0, y1);
        if (MASK) {
            y0 = (word >> k) & 1u ? y0 : -CUDART_INF_F;
            y1 = (word >> (k + 1)) & 1u ? y1 : -CUDART_INF_F;
        }
        top = fmaxf(top, fmaxf(y0, y1));
        const float p0 = ex2_approx(y0), p1 = ex2_approx(y1);
        sum = add_f32x2(sum, pack_f32x2(p0, p1));
        pk[k / 2] = Pair<T>::pack(p0, p1);
    }
}
template <bool MASK> __device__ __forceinline__ void raise_top(const uint32_t (&s)[32], uint32_t word, float c, float &top)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        const float y = __uint_as_float(s[k]) * c;
        top = fmaxf(top, !MASK || ((word >> k) & 1u) ? y : -CUDART_INF_F);
    }
}
// A row's tile: largest y (against the reference), sum and packed weights.  128 columns in four loads, each under way while the one before
// is worked on.
template <typename T, bool MASK>
__device__ __forceinline__ float weigh_tile(uint32_t at, const uint32_t (&words)[4], float c, float ref, float &sum, uint32_t (&pk)[64])
{
    uint32_t a[32], b[32];
    float top = -CUDART_INF_F;
    unsigned long long s2 = 0ull;
    const unsigned long long c2 = pack_f32x2(c, c), r2 = pack_f32x2(-ref, -ref);
    tc::tmem_load(at, a);
    tc::wait_loads(a);
    tc::tmem_load(at + 32, b);
    weigh<T, MASK>(a, words[0], c2, r2, top, s2, pk);
    tc::wait_loads(b);
    tc::tmem_load(at + 64, a);
    weigh<T, MASK>(b, words[1], c2, r2, top, s2, pk + 16);
    tc::wait_loads(a);
    tc::tmem_load(at + 96, b);
    weigh<T, MASK>(a, words[2], c2, r2, top, s2, pk + 32);
    tc::wait_loads(b);
    weigh<T, MASK>(b, words[3], c2, r2, top, s2, pk + 48);
    float x, y;
    unpack_f32x2(s2, x, y);
    sum = x + y;
    return top;
}
template <bool MASK> __device__ __forceinline__ float top_of_tile(uint32_t at, const uint32_t (&words)[4], float c)
{
    uint32_t a[32];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        tc::tmem_load(at + 32 * w, a);
        tc::wait_loads(a);
        raise_top<MASK>(a, words[w], c, top);
    }
    return top;
}

template <typename T, int D, int MT>
__global__ void __launch_bounds__(Shape<D, MT>::NT, 1) spec_attend_kernel(const __grid_constant__ Params P)
{
    using S = Shape<D, MT>;
    unsigned char *base = dyn_smem + (-smem_u32(dyn_smem) & 1023u);
    Bars *B = (Bars *)(base + S::off_bar);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < S::SLOTS; ++i) { mbar_init(&B->full[i], S::NP); mbar_init(&B->empty[i], 1); }
        mbar_init(&B->q_full, S::NP);
        mbar_init(&B->q_empty, 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(&B->s_full[t], 1);
            mbar_init(&B->p_full[t], 4);
            mbar_init(&B->pv_done[t], 1);
            mbar_init(&B->o_empty[t], 4);
        }
        B->dead = 0;
        B->poison = 0;
        B->found[0] = -1;
        mbar_fence_init();
    }
    grid_dependency_wait();
    grid_launch_dependents();                  // (the joining kernel's CTAs may be placed as this one's leave; it waits by itself)
    __syncthreads();
    const int c = blockIdx.x;
    const long long all = find_request(P, S::ROWS, c, B->sums, B->found, tid, S::NT);
    Run run;
    run.left = run_start(all, c + 1, P.ctas) - run_start(all, c, P.ctas);
    run.first = true;
    if (run.left <= 0) {
        if (tid == 0) P.late[c] = 0;
        return;
    }
    run.at = place_in(P, (int)B->found[0], run_start(all, c, P.ctas) - B->found[1], S::ROWS);
    if (warp == S::SOFT) tc::tmem_alloc(&B->tmem, 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = B->tmem;
    Segment seg;
    if (warp < S::SOFT) {
        // ---------------------------------------------------------------- rows: a thread owns one
        const int t = warp >> 2, quad = warp & 3, row = t * 128 + quad * 32 + lane, gt = tid & 127;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16), o_at = lanes + S::O + t * D;
        unsigned short *parent = (unsigned short *)(base + S::off_parent) + t * SPEC_MAX_NODES;
        const float c = P.scale * LOG2E;
        uint32_t n_tile = 0, n_run = 0;        // tiles that this warpgroup has been through, tiles of the run that went by
        int tree_of = -1;
        while (run.next(P, S::ROWS, seg)) {
            if (t * 128 >= seg.rows) {
                n_run += seg.steps();
                continue;
            }
            const int r = seg.m * S::ROWS + row, node = min(r, seg.r.rows - 1) / P.G;
            const bool live = row < seg.rows, warp_live = t * 128 + quad * 32 < seg.rows;
            if (tree_of != seg.b && (tree_of < 0 || P.tree.topo_seq_stride || P.tree.n_nodes)) {
                bar_sync(1 + t, 128);
                const int *from = P.tree.parent + (long long)seg.b * P.tree.topo_seq_stride;
                for (int i = gt; i < seg.r.n; i += 128) {
                    const int p = __ldg(from + i);
                    parent[i] = p >= 0 && p < i ? (unsigned short)p : (unsigned short)0xFFFF;
                }
                tree_of = seg.b;
                bar_sync(1 + t, 128);
            }
            int depth = 0;
            if (P.window)
                for (unsigned short x = parent[node]; x != 0xFFFF; x = parent[x]) ++depth;
            Walk walk = {node, 0};
            float ref = 0.f, l = 0.f;
            bool any = false;                  // whether the row has a reference
            for (int step = 0; step < seg.steps(); ++step, ++n_tile, ++n_run) {
                const int buf = MT == 1 ? n_tile & 1 : t;
                const uint32_t parity = MT == 1 ? (n_tile >> 1) & 1 : n_tile & 1;
                const uint32_t s_at = lanes + buf * 128;
                wait(B, &B->s_full[buf], parity);
                tc::fence_after();
                if (warp_live) {
                    const int tile = seg.tile(step);
                    const volatile uint32_t *hidden = B->hidden[n_run & 7];
                    const uint32_t h0 = hidden[0], h1 = hidden[1], h2 = hidden[2], h3 = hidden[3];
                    const bool masked = !seen_by_all(P, seg.r, tile) || (h0 | h1 | h2 | h3) != 0;
                    uint32_t words[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu}, pk[64];
                    if (masked) {
                        seen_words(P, seg.r, tile, depth, parent, walk, words);
                        words[0] &= ~h0; words[1] &= ~h1; words[2] &= ~h2; words[3] &= ~h3;
                    }
                    if (step == 0) {
                        const float top = masked ? top_of_tile<true>(s_at, words, c) : top_of_tile<false>(s_at, words, c);
                        any = top > -CUDART_INF_F;
                        ref = any ? top : 0.f;
                    }
                    float sum;
                    const float top = masked ? weigh_tile<T, true>(s_at, words, c, ref, sum, pk) : weigh_tile<T, false>(s_at, words, c, ref, sum, pk);
                    const bool over = step > 0 && (any ? top > 8.f : top > -CUDART_INF_F);
                    if (__any_sync(0xffffffffu, over)) {
                        // a new reference: what has been summed is scaled, the tile gone through again
                        const float old = ref;
                        if (over) ref = ref + top;
                        const float f = over && any ? ex2_approx(old - ref) : 1.f;
                        any |= over;
                        l *= f;
                        wait(B, &B->pv_done[t], (n_tile - 1) & 1);
                        tc::fence_after();
#pragma unroll 1
                        for (int d = 0; d < D; d += 32) {
                            uint32_t o[32];
                            tc::tmem_load(o_at + d, o);
                            tc::wait_loads(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tc::tmem_store(o_at + d, o);
                        }
                        tc::wait_stores();
                        masked ? weigh_tile<T, true>(s_at, words, c, ref, sum, pk) : weigh_tile<T, false>(s_at, words, c, ref, sum, pk);
                    }
                    l += sum;
                    tc::tmem_store(s_at, pk);
                    tc::tmem_store(s_at + 32, pk + 32);
                    tc::wait_stores();
                    tc::fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&B->p_full[buf]);
            }
            // the segment's end
            wait(B, &B->pv_done[t], (n_tile - 1) & 1);
            tc::fence_after();
            if (warp_live) {
                const bool poison = *(volatile int *)&B->poison != 0;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const long long slot = (long long)blockIdx.x * 2 + (seg.head ? 0 : 1);
                const int head = seg.h * P.G + r % P.G;
                T *to = (T *)P.out + seg.b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2];
                float *part = P.part + slot * S::ROWS * D;
#pragma unroll 1
                for (int d = 0; d < D; d += 32) {
                    uint32_t o[32];
                    tc::tmem_load(o_at + d, o);
                    tc::wait_loads(o);
                    if (poison && live) {
                        // values that are not finite were taken out of tiles that not all rows see; those that this row sees come back
                        Walk w = {node, 0};
#pragma unroll 1
                        for (int step = 0; step < seg.steps(); ++step) {
                            const int tile = seg.tile(step);
                            if (seen_by_all(P, seg.r, tile)) continue;
                            uint32_t words[4];
                            seen_words(P, seg.r, tile, depth, parent, w, words);
#pragma unroll 1
                            for (int j = 0; j < KT; ++j) {
                                const uint32_t word = j < 32 ? words[0] : j < 64 ? words[1] : j < 96 ? words[2] : words[3];
                                if (!((word >> (j & 31)) & 1u)) continue;
                                const long long key = (long long)tile * KT + j;
                                const int id = block_of(P, seg.b, key);
                                if (id < 0) continue;
                                const unsigned short *v = (const unsigned short *)P.v + id * P.v_stride[0] + key % P.block * P.v_stride[1] +
                                                          seg.h * P.v_stride[2] + d;
#pragma unroll
                                for (int k = 0; k < 32; ++k) {
                                    const float x = Pair<T>::value(__ldg(v + k));
                                    if (!(fabsf(x) < CUDART_INF_F)) o[k] = __float_as_uint(__uint_as_float(o[k]) + x);
                                }
                            }
                        }
                    }
                    if (!live) continue;
                    if (seg.whole) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            uint4 w;
                            w.x = Pair<T>::pack(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv);
                            w.y = Pair<T>::pack(__uint_as_float(o[k + 2]) * inv, __uint_as_float(o[k + 3]) * inv);
                            w.z = Pair<T>::pack(__uint_as_float(o[k + 4]) * inv, __uint_as_float(o[k + 5]) * inv);
                            w.w = Pair<T>::pack(__uint_as_float(o[k + 6]) * inv, __uint_as_float(o[k + 7]) * inv);
                            *(uint4 *)(to + d + k) = w;
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *(uint4 *)(part + ((long long)((d + k) / 4) * S::ROWS + row) * 4) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    }
                }
                if (live) {
                    if (seg.whole) {
                        if (P.lse)
                            P.lse[((long long)seg.b * P.tree.N + node) * P.Hq + head] = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
                    } else {
                        P.ml[slot * S::ROWS + row] = make_float2(any ? ref : -CUDART_INF_F, l);
                    }
                }
                tc::fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&B->o_empty[t]);
        }
    } else if (warp == S::SOFT) {
        // ---------------------------------------------------------------- products: one thread issues, the warp waits
        constexpr uint32_t DS = tc::product_desc(Pair<T>::TYPE, KT, false), DO = tc::product_desc(Pair<T>::TYPE, 64, true);
        const uint32_t q_at = smem_u32(base), slots = smem_u32(base + S::off_slots);
        uint32_t n_slot = 0, n_seg = 0, n_tile = 0, n_p[2] = {0, 0}, n_o[2] = {0, 0};
        const auto slot_wait = [&](uint32_t n) { wait(B, &B->full[n % S::SLOTS], (n / S::SLOTS) & 1); };
        // S of row block t into buffer buf, from the keys in slots n ..
        const auto scores = [&](int t, int buf, uint32_t n, bool release) {
            if (lane == 0) {
#pragma unroll
                for (int p = 0; p < S::PANELS; ++p) {
                    const uint64_t qd = tc::panel_desc(q_at + (p * MT + t) * PANEL);
                    const uint64_t kd = tc::panel_desc(slots + (n + p) % S::SLOTS * PANEL);
#pragma unroll
                    for (int k = 0; k < 4; ++k) tc::mma_ss(tmem + buf * 128, qd + 2 * k, kd + 2 * k, DS, p > 0 || k > 0);
                    if (release) tc::commit(&B->empty[(n + p) % S::SLOTS]);
                }
                tc::commit(&B->s_full[buf]);
            }
            __syncwarp();
        };
        const auto sums = [&](int t, int buf, uint32_t n, bool add, bool release) {
            if (lane == 0) {
#pragma unroll
                for (int p = 0; p < S::PANELS; ++p) {
                    const uint64_t vd = tc::panel_desc(slots + (n + p) % S::SLOTS * PANEL);
#pragma unroll
                    for (int k = 0; k < KT / 16; ++k)
                        tc::mma_ts(tmem + S::O + t * D + p * 64, tmem + buf * 128 + k * 8, vd + k * (2048 >> 4), DO, add || k > 0);
                    if (release) tc::commit(&B->empty[(n + p) % S::SLOTS]);
                }
                tc::commit(&B->pv_done[t]);
            }
            __syncwarp();
        };
        while (run.next(P, S::ROWS, seg)) {
            const int steps = seg.steps(), tiles = MT == 1 || seg.rows <= 128 ? 1 : 2;
            const auto keys_in = [&](uint32_t n) { for (int p = 0; p < S::PANELS; ++p) slot_wait(n + p); tc::fence_after(); };
            wait(B, &B->q_full, n_seg & 1);
            if (MT == 1) {
                // order of the slots: K0, K1, V0, K2, V1, ...: scores one tile ahead
                uint32_t n = n_slot;
                keys_in(n);
                scores(0, n_tile & 1, n, true);
                n += S::PANELS;
                for (int i = 0; i < steps; ++i) {
                    if (i + 1 < steps) {
                        keys_in(n);
                        scores(0, (n_tile + i + 1) & 1, n, true);
                        n += S::PANELS;
                    }
                    if (i + 1 == max(1, steps - 1) && lane == 0) tc::commit(&B->q_empty);
                    keys_in(n);
                    const int buf = (n_tile + i) & 1;
                    wait(B, &B->p_full[buf], ((n_tile + i) >> 1) & 1);
                    if (i == 0) { if (n_o[0]) wait(B, &B->o_empty[0], (n_o[0] - 1) & 1); ++n_o[0]; }
                    tc::fence_after();
                    sums(0, buf, n, i > 0, true);
                    n += S::PANELS;
                }
                n_slot = n;
                n_tile += steps;
            } else {
                // order of the slots: K0, V0, K1, V1, ...: a row block's next scores right behind its sums
                uint32_t n = n_slot;
                keys_in(n);
                for (int t = 0; t < tiles; ++t) scores(t, t, n, t == tiles - 1);
                n += S::PANELS;
                if (steps == 1 && lane == 0) tc::commit(&B->q_empty);
                for (int i = 0; i < steps; ++i) {
                    keys_in(n);
                    for (int t = 0; t < tiles; ++t) {
                        wait(B, &B->p_full[t], n_p[t] & 1);
                        ++n_p[t];
                        if (i == 0) { if (n_o[t]) wait(B, &B->o_empty[t], (n_o[t] - 1) & 1); ++n_o[t]; }
                        tc::fence_after();
                        sums(t, t, n, i > 0, t == tiles - 1);
                        if (i + 1 < steps) {
                            if (t == 0) keys_in(n + S::PANELS);
                            scores(t, t, n + S::PANELS, t == tiles - 1);
                        }
                    }
                    if (i + 2 == steps && lane == 0) tc::commit(&B->q_empty);
                    n += 2 * S::PANELS;
                }
                n_slot = n - S::PANELS;
            }
            ++n_seg;
        }
    } else {
        // ---------------------------------------------------------------- copies: 128 threads, a row's 16-byte chunks over its lanes
        const int pt = tid - (S::SOFT + 1) * 32;
        constexpr int CH = D / 8, RPI = S::NP / CH;                   // chunks of a row; rows that the threads copy at a time
        const int ch = pt % CH, r0 = pt / CH;
        const uint32_t slots = smem_u32(base + S::off_slots), q_at = smem_u32(base);
        ulonglong2 *rows = (ulonglong2 *)(base + S::off_rows);
        uint32_t n_slot = 0, n_seg = 0, n_row = 0;
        uint32_t open[S::LAG + 1];                                    // the copies under way: slot, and whether values of a tile in part seen
        int under = 0;
        for (int i = 0; i <= S::LAG; ++i) open[i] = 0;
        // a copy's arrival: values that are not finite leave a tile that some rows do not see
        const auto arrive = [&](uint32_t o) {
            const uint32_t n = o >> 2;
            if (o & 2) {
#pragma unroll 1
                for (int i = r0; i < KT; i += RPI) {
                    unsigned char *at = base + S::off_slots + (n + ch / 8) % S::SLOTS * PANEL + i * 128 + (((ch & 7) ^ (i & 7)) << 4);
                    uint4 w = *(uint4 *)at;
                    uint32_t *x = (uint32_t *)&w;
                    bool bad = false;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (Pair<T>::finite(x[k])) continue;
                        bad = true;
                        const uint32_t lo = x[k] & 0xFFFFu, hi = x[k] & 0xFFFF0000u;
                        x[k] = (Pair<T>::finite(lo) ? lo : 0u) | (Pair<T>::finite(hi) ? hi : 0u);
                    }
                    if (bad) { *(uint4 *)at = w; *(volatile int *)&B->poison = 1; }
                }
            }
            tc::publish_shared();
            if (o & 1) mbar_arrive(&B->q_full);
            else for (int p = 0; p < S::PANELS; ++p) mbar_arrive(&B->full[(n + p) % S::SLOTS]);
        };
        // closes the copies issued last and lets the oldest arrive
        const auto turn = [&](uint32_t o) {
            tc::close_copies();
#pragma unroll
            for (int i = S::LAG; i > 0; --i) open[i] = open[i - 1];
            open[0] = o;
            if (under < S::LAG) { ++under; return; }
            tc::wait_copies<S::LAG>();
            arrive(open[S::LAG]);
        };
        // A wait for room.  Copies under way arrive first: what has been copied may be what the room is waiting for.
        const auto room = [&](uint64_t *bar, uint32_t parity) {
            if (mbar_test(bar, parity)) return;
            tc::wait_copies<0>();
            for (int i = under - 1; i >= 0; --i) {
#pragma unroll
                for (int j = 0; j < S::LAG; ++j) if (j == i) arrive(open[j]);
            }
            under = 0;
            wait(B, bar, parity);
        };
        // sources of a tile's rows, one per thread: null where no row of the request sees the key or its block is bad
        const auto sources = [&](const Segment &s, int tile) {
            const long long key = (long long)tile * KT + pt;
            const bool seen = key < (long long)s.r.len + s.r.n &&
                              (key >= s.r.len || P.window == 0 || key < P.sinks || key > (long long)s.r.len - P.window);
            const int id = seen ? block_of(P, s.b, key) : -1;
            ulonglong2 a = make_ulonglong2(0, 0);
            if (id >= 0) {
                const int in = (int)(key % P.block);
                a.x = (unsigned long long)((const T *)P.k + id * P.k_stride[0] + in * P.k_stride[1] + s.h * P.k_stride[2]);
                a.y = (unsigned long long)((const T *)P.v + id * P.v_stride[0] + in * P.v_stride[1] + s.h * P.v_stride[2]);
            }
            bar_sync(4, S::NP);                                       // (all are through with the tile before the last)
            rows[(n_row & 1) * KT + pt] = a;
            const uint32_t bad = __ballot_sync(0xffffffffu, seen && id < 0);
            if (lane == 0) B->hidden[n_row & 7][pt >> 5] = bad;
            bar_sync(4, S::NP);
            ++n_row;
        };
        const auto copy_tile = [&](uint32_t n, uint32_t which, bool values, bool part) {
            for (int p = 0; p < S::PANELS; ++p) {
                const uint32_t k = n + p;
                if (k >= S::SLOTS) room(&B->empty[k % S::SLOTS], (k / S::SLOTS - 1) & 1);
            }
            const ulonglong2 *from = rows + (which & 1) * KT;
#pragma unroll 8
            for (int i = r0; i < KT; i += RPI) {
                const unsigned long long a = values ? from[i].y : from[i].x;
                tc::copy16(slots + (n + ch / 8) % S::SLOTS * PANEL + i * 128 + (((ch & 7) ^ (i & 7)) << 4), a ? (const char *)a + ch * 16 : nullptr, P.k);
            }
            turn(n << 2 | (values && part ? 2u : 0u));
        };
        while (run.next(P, S::ROWS, seg)) {
            const int steps = seg.steps();
            const auto copy_q = [&]() {
                if (n_seg) room(&B->q_empty, (n_seg - 1) & 1);
                for (int i = r0; i < S::ROWS; i += RPI) {
                    const int r = seg.m * S::ROWS + i;
                    const T *from = nullptr;
                    if (i < seg.rows)
                        from = (const T *)P.q + seg.b * P.q_stride[0] + r / P.G * P.q_stride[1] + (seg.h * P.G + r % P.G) * P.q_stride[2] + ch * 8;
                    tc::copy16(q_at + ((ch / 8) * MT + i / 128) * PANEL + i % 128 * 128 + (((ch & 7) ^ (i & 7)) << 4), from, P.q);
                }
                turn(1u);
                ++n_seg;
            };
            uint32_t last_row = 0;
            bool last_part = false;
            for (int i = 0; i < steps; ++i) {
                const int tile = seg.tile(i);
                const bool part = !seen_by_all(P, seg.r, tile);
                sources(seg, tile);
                copy_tile(n_slot, n_row - 1, false, part);
                n_slot += S::PANELS;
                if (i == 0) copy_q();
                if (MT == 1) {
                    if (i > 0) { copy_tile(n_slot, last_row, true, last_part); n_slot += S::PANELS; }
                    last_row = n_row - 1;
                    last_part = part;
                } else {
                    copy_tile(n_slot, n_row - 1, true, part);
                    n_slot += S::PANELS;
                }
            }
            if (MT == 1) { copy_tile(n_slot, last_row, true, last_part); n_slot += S::PANELS; }
        }
        // the last arrivals
        tc::wait_copies<0>();
        for (int i = under - 1; i >= 0; --i) {
#pragma unroll
            for (int j = 0; j < S::LAG; ++j) if (j == i) arrive(open[j]);
        }
    }
    tc::fence_before();
    __syncthreads();
    if (warp == S::SOFT) {
        tc::fence_after();
        tc::tmem_free(tmem, 512);
        if (lane == 0) P.late[c] = B->dead;
    }
}

// ---- joining ------------------------------------------------------------------------------------------------------------------
// The first P.ctas * groups CTAs: (start of run j + 1, 32 rows).  Where that start lies inside a unit and is the first to, the unit's
// parts are put together: out = sum 2^(ref_c - ref) O_c / sum 2^(ref_c - ref) l_c.  The others: a request each, its status (while the
// attention still runs: that reads inputs alone) and zeros for a bad tree.
constexpr int JOIN_NT = 256, CTAS_MAX = 256;

template <typename T, int D, int MT> __global__ void __launch_bounds__(JOIN_NT) spec_join_kernel(const __grid_constant__ Params P)
{
    using S = Shape<D, MT>;
    constexpr int GROUPS = S::ROWS / 32, WARPS = JOIN_NT / 32;
    __shared__ float share[CTAS_MAX][32];
    __shared__ long long sums[WARPS], found[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int)blockIdx.x >= P.ctas * GROUPS) {
        const int b = blockIdx.x - P.ctas * GROUPS;
        const int len = __ldg(P.tree.lengths + b), nn = tree_nodes(P.tree, b), n = len < 0 ? 0 : max(nn, 0);
        const int *parent = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
        bool bad = false, page = false;
        for (int i = tid; i < n; i += JOIN_NT) {
            const int p = __ldg(parent + i);
            bad |= i == 0 ? p != -1 : p < 0 || p >= i;
        }
        // columns of the table that hold a key that some node sees
        const long long keys = n ? (long long)len + n : 0, since = P.window ? max(0ll, (long long)len - P.window + 1) : 0;
        const long long sinks = min((long long)P.sinks, (long long)len), cols = (keys + P.block - 1) / P.block;
        for (long long col = tid; col < cols; col += JOIN_NT) {
            const long long a = col * P.block, e = a + P.block;
            if (e > since || a < sinks) page |= block_of(P, b, a) < 0;
        }
        bad = __syncthreads_or(bad) != 0;
        page = __syncthreads_or(page) != 0;
        grid_dependency_wait();
        bool late = false;
        for (int i = tid; i < P.ctas; i += JOIN_NT) late |= *(volatile int *)(P.late + i) != 0;
        late = __syncthreads_or(late) != 0;
        if (tid == 0)
            P.status[b] = len < 0 ? SPEC_DEV_OK
                          : nn < 0 || bad ? SPEC_DEV_TOPOLOGY : late ? SPEC_DEV_TIMEOUT : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
        if (!bad) return;
        for (long long i = tid; i < (long long)n * P.Hq * (D / 8); i += JOIN_NT) {
            const int d = (int)(i % (D / 8)) * 8, h = (int)(i / (D / 8) % P.Hq), node = (int)(i / (D / 8) / P.Hq);
            *(uint4 *)((T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + h * P.out_stride[2] + d) = make_uint4(0, 0, 0, 0);
            if (P.lse && d == 0) P.lse[((long long)b * P.tree.N + node) * P.Hq + h] = -CUDART_INF_F;
        }
        return;
    }
    const int j = blockIdx.x / GROUPS, group = blockIdx.x % GROUPS;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    const long long all = find_request(P, S::ROWS, j + 1, sums, found, tid, JOIN_NT);
    const long long cut = run_start(all, j + 1, P.ctas);
    if (j + 1 < P.ctas && found[0] >= 0) {
        const int b = (int)found[0];
        const Place at = place_in(P, b, cut - found[1], S::ROWS);
        const Request r = request_of(P, b);
        const long long begin = cut - at.i, end = begin + tiles_of(P, r, at.m, S::ROWS).count();
        const int rows = min(r.rows - at.m * S::ROWS, S::ROWS), row = group * 32 + lane;
        if (at.i > 0 && run_start(all, j, P.ctas) <= begin && group * 32 < rows) {
            grid_dependency_wait();
            // CTA c's part: where its run starts is the unit's start or inside it; the first CTA's may start before
            int last = j;
            while (last + 1 < P.ctas && run_start(all, last + 1, P.ctas) < end) ++last;
            const auto slot = [&](int c) { return 2 * c + (run_start(all, c, P.ctas) < begin ? 1 : 0); };
            const auto has = [&](int c) { return run_start(all, c, P.ctas) < run_start(all, c + 1, P.ctas); };
            for (int c = j + warp; c <= last; c += WARPS)
                share[c][lane] = has(c) && row < rows ? __ldcg(&P.ml[(long long)slot(c) * S::ROWS + row].x) : -CUDART_INF_F;
            __syncthreads();
            float ref = -CUDART_INF_F, l = 0.f;
            for (int c = j; c <= last; ++c) ref = fmaxf(ref, share[c][lane]);
            __syncthreads();
            const float base = ref == -CUDART_INF_F ? 0.f : ref;
            for (int c = j + warp; c <= last; c += WARPS) {
                const float x = share[c][lane];
                // (a part whose reference is no number stays what it is: its sums are not either)
                share[c][lane] = x == -CUDART_INF_F ? 0.f : ex2_approx(x - base);
            }
            __syncthreads();
            if (row < rows) {
                for (int c = j; c <= last; ++c)
                    if (has(c)) l += share[c][lane] == 0.f ? 0.f : share[c][lane] * __ldcg(&P.ml[(long long)slot(c) * S::ROWS + row].y);
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const int q = at.m * S::ROWS + row, node = q / P.G, head = at.h * P.G + q % P.G;
                T *to = (T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2];
                for (int ch = warp; ch < D / 4; ch += WARPS) {
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int c = j; c <= last; ++c) {
                        const float w = share[c][lane];
                        if (w == 0.f) continue;
                        const float4 x = __ldcg((const float4 *)P.part + ((long long)slot(c) * (D / 4) + ch) * S::ROWS + row);
                        o.x = fmaf(w, x.x, o.x); o.y = fmaf(w, x.y, o.y); o.z = fmaf(w, x.z, o.z); o.w = fmaf(w, x.w, o.w);
                    }
                    *(uint2 *)(to + ch * 4) = make_uint2(Pair<T>::pack(o.x * inv, o.y * inv), Pair<T>::pack(o.z * inv, o.w * inv));
                }
                if (P.lse && warp == 0)
                    P.lse[((long long)b * P.tree.N + node) * P.Hq + head] = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
            }
            return;
        }
    }
    grid_dependency_wait();
}

}  // namespace attend
}  // namespace specv
