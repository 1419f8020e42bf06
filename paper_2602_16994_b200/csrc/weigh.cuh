// Attention weight that entries of a paged cache get (spec_cache_weights).
//
// Mathematics.  w_j += sum over rows (node i that sees j, query head) of 2^(c k_j . q_r - lse_r log2 e), c = scale log2 e.  The product is taken with the
// keys as the tensor cores' rows: S = K Q^T, 128 keys by up to 128 rows of a key head, so a thread owns a key and adds up along its own
// columns; over the rows, blocks of rows and key heads its sum never leaves its register, and no two CTAs add to the same entry: the order
// of every sum is fixed.
//
// What bounds it.  With many rows the exponentials: 16 a cycle and SM, of which this reaches 0.52 (2 stretches of 512 nodes, 32 heads to 8, behind up to 16384 tokens: 184 us; 96
// of exponentials alone, 64 of products): a warp loads 32 columns, waits for them and takes their exponentials, and four such warps to a scheduler do not cover the
// loads.  Taking one to three of eight by a polynomial instead made that 1 to 5 % longer.  With few rows latency: the keys'
// bytes of 8 requests of 19 nodes over 1500 to 4096 keys would take 7.5 us, the call takes 25, of one token over 4096 keys 1.3 and 12: a CTA knows its run
// after 2.7 us and has its first sums after 6, then a tile and head take 1300 to 2200 cycles.
//
// Balance.  Two tiles that lie wholly among the committed tokens go together (a block of queries that is on chip serves both), the others by themselves; a
// unit is such a group and a key head, its length its tiles.  The units of all requests, groups in order, heads within, are cut into one run per CTA (one
// CTA per SM).  A group whose heads are in several runs leaves their sums in the workspace, and spec_weigh_join_kernel adds them up in order.
// Four warps copy keys (by tensor map where all 32 of a warp's keys are there and blocks are multiples of 8 slots, else 16 bytes at a time), two
// queries (by tensor map where a block of them is whole nodes: 179 us for the stretches of 512 nodes, 292 by 16-byte copies; keys 25.0 and 25.2 for 8 requests), two issue the products, sixteen take the exponentials, a product a
// warpgroup in turn (128 columns: 1800 cycles of an SM where all warps had 32 columns each of every product, and its barriers).
//
// What is not a number adds nothing: the maximum that bounds exponents from below takes NaN for its bound.  So it does not matter what
// rows without a finite lse, columns beyond the rows, or keys that are not there hold.
#pragma once
#include "attend.cuh"

namespace specv {
namespace weigh {

constexpr int KT = 128, PANEL = 128 * 128;
constexpr float LOG2E = 1.4426950408889634f;

struct Params {
    CUtensorMap k_map;                         // the cache as [block][slot][head][entry], boxes of `box` slots by 64 entries
    CUtensorMap q_map;                         // the queries as [request][node][head][entry], boxes of the rows of `q_nodes` nodes by 64 entries
    int q_nodes;                               // 0: where a block of queries is no whole number of nodes
    int box;                                   // a power of two up to 32 that divides the block; 0: blocks of no multiple of 8 slots
    TreeArgs tree;
    int B, Hq, Hkv, G, num_blocks, block, width, fresh;
    unsigned block_mul, group_mul;             // divisions by block and G, as in the attention
    int block_shift, group_shift;
    float c;
    const void *q, *k;
    long long q_stride[3], k_stride[3];
    const float *lse;
    const int *table;
    long long table_stride;
    const int *protect;
    float *weights;
    int *status;
    int ctas;
    float *part;                               // [ctas][2][2][128] sums of a run's first and last group, where others have heads of them too
    int4 *joint;                               // [ctas] the group whose first heads this CTA has: request, tile, tiles; parts and slot
    int *late;                                 // [ctas] a wait ran out
};

struct Request {
    int len, n, from, end;                     // nodes (0: idle or a bad number of them); entries [from, end) count
    __device__ __forceinline__ int first() const { return from / KT; }
    __device__ __forceinline__ int tiles() const { return n == 0 || end <= from ? 0 : (int)(((unsigned)end + KT - 1) / KT) - from / KT; }
    __device__ __forceinline__ int pairs() const { return max(0, min(len / KT - from / KT, tiles())) / 2; }
};
__device__ __forceinline__ Request request_of(const Params &P, int b)
{
    Request r;
    r.len = __ldg(P.tree.lengths + b);
    r.n = r.len < 0 ? 0 : max(0, tree_nodes(P.tree, b));
    // (entries behind the table's end have no block)
    const long long held = min((long long)P.width * P.block, 0x7FFFFFFFll);
    r.end = r.len < 0 ? 0 : (int)min((long long)r.len + r.n, held);
    r.from = P.protect ? max(0, __ldg(P.protect + b)) : 0;
    return r;
}
__device__ __forceinline__ int column_of(const Params &P, int key) { return (int)((__umulhi(P.block_mul, (unsigned)key) + (unsigned)key) >> P.block_shift); }
__device__ __forceinline__ int node_of(const Params &P, int row) { return (int)((__umulhi(P.group_mul, (unsigned)row) + (unsigned)row) >> P.group_shift); }

// A unit's length: two tiles that go together take some 1.5 times as long as one (8 requests of 19 nodes: 3500 cycles a head to 2200; stretches of 512 nodes:
// 49000 to 31000).
__device__ __forceinline__ int length_of(int count) { return count == 2 ? 3 : 2; }
__device__ __forceinline__ int length_of(const Request &r) { return 2 * r.tiles() - r.pairs(); }         // of all a request's groups, for a head
// What a CTA has next: heads of a group; every role counts for itself.
struct Run {
    int b, t, h, left, next_at;                // the next unit: request, tiles of it gone by, head; length of the run from there on, and its place
    Request r;
    int tile, count, h0, h1, at;               // this step's group, and the heads of it, and its place among all units
    __device__ __forceinline__ bool next(const Params &P)
    {
        if (left <= 0) return false;
        while (t >= r.tiles()) {
            if (++b >= P.B) return false;
            r = request_of(P, b);
            t = 0;
        }
        tile = r.first() + t;
        count = t < 2 * r.pairs() ? 2 : 1;
        h0 = h;
        const int each = length_of(count);
        h1 = min(P.Hkv, h0 + (int)((unsigned)(left + each - 1) / (unsigned)each));
        at = next_at;
        left -= (h1 - h0) * each;
        next_at += (h1 - h0) * each;
        h = h1;
        if (h == P.Hkv) { h = 0; t += count; }
        return true;
    }
};

constexpr int SR = 8;                          // blocks of queries whose references are on chip: their products read them, the sums' warps these
template <int D_> struct Shape {
    static constexpr int D = D_, PANELS = D / 64, QB = D == 256 ? 64 : 128;       // rows of a block of queries
    static constexpr int K_SLOT = KT * D * 2, Q_SLOT = QB * D * 2;
    static constexpr int SK = D == 64 ? 6 : D == 128 ? 3 : 2, SQ = D == 64 ? 4 : D == 128 ? 3 : 2;
    static constexpr int off_q = SK * K_SLOT, off_mask = off_q + SQ * Q_SLOT;
    static constexpr int off_ref = off_mask + SPEC_MAX_NODES * 16;                // [SR][128] -lse log2 e
    static constexpr int off_node = off_ref + SR * 128 * 4;                       // [SR][128] nodes of the columns
    static constexpr int off_parent = off_node + SR * 128 * 2;
    static constexpr int off_part = off_parent + SPEC_MAX_NODES * 2;              // [2][4][2][128] the warpgroups' sums
    static constexpr int off_bar = off_part + 8192;
    static constexpr int total = off_bar + 512;
    static_assert(total + 1024 <= 227 * 1024, "shared memory");
};
constexpr int SUM_WARPS = 16, WG = SUM_WARPS / 4, SUMS = SUM_WARPS * 32, PRODUCTS = SUM_WARPS, KEYS = PRODUCTS + 2, QUERIES = KEYS + 4, NT = (QUERIES + 2) * 32;      // the roles' first warps
struct Bars {
    uint64_t k_full[6], k_empty[6], q_full[4], q_empty[4], s_full[4], s_empty[4], r_full[SR], r_empty[SR];
    uint32_t tmem;
    int dead, found[2];
    int sums[NT / 32];                         // an entry for every warp of the CTA
    Request request;                           // the one that the run begins in
};
static_assert(sizeof(Bars) <= 512, "the area behind the buffers");

__device__ __forceinline__ void wait(Bars *B, uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return;
    const long long t0 = clock64();
    do {
        if (*(volatile int *)&B->dead) return;
        if (clock64() - t0 > WAIT_CYCLES) { *(volatile int *)&B->dead = 1; return; }
    } while (!mbar_try_wait(bar, parity));
}
// one answer for the whole (converged) warp
__device__ __forceinline__ bool stopped(Bars *B) { return __any_sync(0xffffffffu, *(volatile int *)&B->dead) != 0; }

struct Cuts {                                  // runs of equal length, the first `more` of them longer by one
    int all, each, more;
    __device__ __forceinline__ int start(int c) const { return each * c + min(c, more); }
};
// The run of CTA c: all threads.  Between the two barriers every warp reads all of `sums`, and the one thread that finds the run's start writes `found` and
// `request`, which no other reads there: sums has an entry for every warp and ends ahead of both, so nothing that is written is read before the second barrier.
__device__ __forceinline__ void find_run(const Params &P, int c, Bars *S, Run *run, Cuts *cuts, int tid)
{
    const int lane = tid & 31, warp = tid >> 5;
    const int per = (P.B + NT - 1) / NT, b0 = min(P.B, tid * per), b1 = min(P.B, b0 + per);
    int mine = 0;
    Request only = {};                         // (at most one request to a thread: it is looked up once)
    for (int b = b0; b < b1; ++b) { only = request_of(P, b); mine += length_of(only) * P.Hkv; }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    if (lane == 31) S->sums[warp] = incl;
    if (tid == 0) { S->found[0] = P.B; S->found[1] = 0; }
    __syncthreads();
    static_assert(sizeof(S->sums) / sizeof(int) == NT / 32 && NT / 32 <= 32, "an entry of sums, and a lane, for every warp");
    int warps = lane < NT / 32 ? S->sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, warps, o);
        if (lane >= o) warps += t;
    }
    const int before = __shfl_sync(0xffffffffu, warps, max(warp - 1, 0)), all = __shfl_sync(0xffffffffu, warps, 31);
    int ahead = incl - mine + (warp ? before : 0);
    const int each = (int)((unsigned)all / (unsigned)P.ctas), more = all - each * P.ctas, start = each * c + min(c, more);
    if (start >= ahead && start < ahead + mine) {
        for (int b = b0; b < b1; ++b) {
            if (per > 1) only = request_of(P, b);
            const int t = length_of(only) * P.Hkv;
            if (start < ahead + t) { S->found[0] = b; S->found[1] = start - ahead; S->request = only; break; }
            ahead += t;
        }
    }
    __syncthreads();
    run->b = S->found[0];
    run->r = S->request;
    run->left = run->b < P.B ? each + (c < more) : 0;
    // the place in the request: the first unit that begins there or behind
    run->next_at = start;
    int at = S->found[1];
    const int n_pairs = run->b < P.B ? run->r.pairs() : 0, paired = n_pairs * length_of(2) * P.Hkv, in_pairs = at < paired, each_unit = length_of(in_pairs ? 2 : 1);
    at -= in_pairs ? 0 : paired;
    const int units = (int)((unsigned)(at + each_unit - 1) / (unsigned)each_unit), g = (int)((unsigned)units / (unsigned)P.Hkv), past = units * each_unit - at;
    run->left -= past;
    run->next_at += past;
    run->t = in_pairs ? 2 * g : 2 * n_pairs + g;
    run->h = units - g * P.Hkv;
    cuts->all = all; cuts->each = each; cuts->more = more;
}

// What a key gets of 16 columns of scores: sum 2^(c s + ref), ref -lse log2 e or -inf.  BOUND: what is no number adds nothing.
template <bool BOUND> __device__ __forceinline__ float sixteen(const uint32_t *s, unsigned long long c2, const float *ref)
{
    unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
        const float4 r4 = *(const float4 *)(ref + k);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x, y;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[k + 2 * i]), __uint_as_float(s[k + 2 * i + 1])), c2,
                                   i ? pack_f32x2(r4.z, r4.w) : pack_f32x2(r4.x, r4.y)), x, y);
            sum[i] = add_f32x2(sum[i], BOUND ? pack_f32x2(ex2_approx(fmaxf(x, -200.f)), ex2_approx(fmaxf(y, -200.f))) : pack_f32x2(ex2_approx(x), ex2_approx(y)));
        }
    }
    float x, y;
    unpack_f32x2(add_f32x2(sum[0], sum[1]), x, y);
    return x + y;
}
// The same of 32 columns, the first `columns` of which are rows' (more than 16 or not).  The exponentials are what the rest waits for (16 a cycle on an SM); the
// bound that takes NaN out is one instruction more for each, so it is applied where the sum came to NaN only.
__device__ __forceinline__ float weights_of(uint32_t (&s)[32], unsigned long long c2, const float *ref, int columns, bool masked, const uint4 *mask,
                                            const unsigned short *nodes, int quad, int lane)
{
    if (masked) {
        // a lane for a column: what its node sees of the warp's 32 keys.  All of them for most columns of a stretch of a prompt, or none.
        const uint32_t word = lane < columns ? ((const uint32_t *)(mask + nodes[lane]))[quad] : 0xFFFFFFFFu;
        if (__all_sync(0xffffffffu, word == 0u || lane >= columns)) return 0.f;
        if (!__all_sync(0xffffffffu, word == 0xFFFFFFFFu)) {
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                const uint32_t w = __shfl_sync(0xffffffffu, word, k);
                if (!((w >> lane) & 1u)) s[k] = 0xFF800000u;
            }
        }
    }
    float got = sixteen<false>(s, c2, ref);
    if (columns > 16) got += sixteen<false>(s + 16, c2, ref + 16);
    if (__any_sync(0xffffffffu, got != got)) {
        got = sixteen<true>(s, c2, ref);
        if (columns > 16) got += sixteen<true>(s + 16, c2, ref + 16);
    }
    return got;
}

template <typename T, typename S> __global__ void __launch_bounds__(NT, 1) spec_weigh_kernel(const __grid_constant__ Params P)
{
    constexpr int D = S::D;
    unsigned char *base = dyn_smem + (-smem_u32(dyn_smem) & 1023u);
    Bars *B = (Bars *)(base + S::off_bar);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (warp == PRODUCTS) tc::tmem_alloc(&B->tmem, 512);
    if (tid == NT - 1) {
        if (P.box) tc::prefetch_map(&P.k_map);
        if (P.q_nodes) tc::prefetch_map(&P.q_map);
    }
    if (tid == 0) {
        for (int i = 0; i < S::SK; ++i) { mbar_init(&B->k_full[i], 128); mbar_init(&B->k_empty[i], 2); }
        for (int i = 0; i < S::SQ; ++i) { mbar_init(&B->q_full[i], 128); mbar_init(&B->q_empty[i], 2); }
        for (int i = 0; i < SR; ++i) { mbar_init(&B->r_full[i], 64); mbar_init(&B->r_empty[i], 8); }
        for (int i = 0; i < 4; ++i) { mbar_init(&B->s_full[i], 1); mbar_init(&B->s_empty[i], 4); }
        B->dead = 0;
        mbar_fence_init();
    }
    grid_dependency_wait();
    Run run;
    Cuts cuts;
    find_run(P, blockIdx.x, B, &run, &cuts, tid);
    grid_launch_dependents();                  // (the joining kernel waits by itself)
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = B->tmem;
    if (warp < SUM_WARPS) {
        // ---------------------------------------------------------------- sums: a thread owns a key
        const int w = warp >> 2, quad = warp & 3, mine = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        unsigned short *parent = (unsigned short *)(base + S::off_parent);
        uint4 *mask = (uint4 *)(base + S::off_mask);
        float *part = (float *)(base + S::off_part);
        const unsigned long long c2 = pack_f32x2(P.c, P.c);
        uint32_t n_q = 0, n_s = 0, n_step = 0;
        int tree_of = -1;
        bool sound = true;
        int4 joint = make_int4(0, 0, 0, 0);
        for (; run.next(P); ++n_step) {
            const Request r = run.r;
            const bool whole = run.h0 == 0 && run.h1 == P.Hkv;
            const int rows = r.n * P.G, blocks = (rows + S::QB - 1) / S::QB;
            // the thread's entry of the tile that it finishes, and what it holds
            const int entry = (run.tile + (run.count == 2 ? w : 0)) * KT + mine;
            long long slot = -1;
            float old = 0.f;
            if (whole && entry >= r.from && entry < r.end && w < run.count) {
                const int col = column_of(P, entry), id = __ldg(P.table + (long long)run.b * P.table_stride + col);
                if (id >= 0 && id < P.num_blocks) {
                    slot = (long long)id * P.block + (entry - col * P.block);
                    if (!(P.fresh && entry >= r.len)) old = __ldcg(P.weights + slot);
                }
            }
            if (tree_of != run.b) {
                bool bad = false;
                const int *row = P.tree.parent + (long long)run.b * P.tree.topo_seq_stride;
                bar_sync(1, SUMS);
                for (int i = tid; i < r.n; i += SUMS) {
                    const int p = __ldg(row + i);
                    const bool wrong = i == 0 ? p != -1 : p < 0 || p >= i;
                    parent[i] = wrong || i == 0 ? (unsigned short)0xFFFF : (unsigned short)p;
                    bad |= wrong;
                }
                part[tid] = __int_as_float(bad ? 1 : 0);
                bar_sync(1, SUMS);
                int x = 0;
                for (int i = lane; i < SUMS; i += 32) x |= __float_as_int(part[i]);
                sound = __any_sync(0xffffffffu, x) == 0;
                tree_of = run.b;
                bar_sync(1, SUMS);
            }
            const bool masked = (long long)(run.tile + 1) * KT > r.len;            // (then the tile goes by itself)
            if (masked) {
                // what each node sees of the tile: itself and its ancestors, by doubling, and all committed tokens
                const long long a = (long long)run.tile * KT;
                constexpr int MINE = SPEC_MAX_NODES / SUMS;
                int up[MINE];
                uint4 m[MINE];
#pragma unroll
                for (int x = 0; x < MINE; ++x) {
                    const int i = x * SUMS + tid;
                    m[x] = make_uint4(0, 0, 0, 0);
                    up[x] = 0xFFFF;
                    if (i >= r.n) continue;
                    // (32 steps up by itself: all the way in a draft tree)
                    uint32_t bits[4] = {0u, 0u, 0u, 0u};
                    int node = i;
                    for (int step = 0; step <= 32 && node != 0xFFFF; ++step) {
                        const long long at = (long long)r.len + node - a;
                        if (at < 0) { node = 0xFFFF; break; }
#pragma unroll
                        for (int k = 0; k < 4; ++k) bits[k] |= at >> 5 == k ? 1u << (at & 31) : 0u;
                        node = parent[node];
                    }
                    up[x] = node;
                    m[x] = make_uint4(bits[0], bits[1], bits[2], bits[3]);
                    mask[i] = m[x];
                }
                unsigned short *above = parent;
                bar_sync(1, SUMS);
                if (r.n > 33) {
#pragma unroll
                    for (int x = 0; x < MINE; ++x)
                        if (x * SUMS + tid < r.n) above[x * SUMS + tid] = (unsigned short)up[x];
                    bar_sync(1, SUMS);
                }
                for (int span = 33; span < r.n; span <<= 1) {
                    uint4 more[MINE];
                    int further[MINE];
#pragma unroll
                    for (int x = 0; x < MINE; ++x) {
                        more[x] = make_uint4(0, 0, 0, 0);
                        further[x] = up[x];
                        if (up[x] != 0xFFFF) { more[x] = mask[up[x]]; further[x] = above[up[x]]; }
                    }
                    bar_sync(1, SUMS);
#pragma unroll
                    for (int x = 0; x < MINE; ++x) {
                        const int i = x * SUMS + tid;
                        if (i >= r.n) continue;
                        m[x].x |= more[x].x; m[x].y |= more[x].y; m[x].z |= more[x].z; m[x].w |= more[x].w;
                        up[x] = further[x];
                        mask[i] = m[x];
                        above[i] = (unsigned short)up[x];
                    }
                    bar_sync(1, SUMS);
                }
                if (r.n > 33) tree_of = -1;                          // (the parents have been used up)
                uint32_t all[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) all[k] = attend::bits_of(a + 32 * k, 0, r.len);
#pragma unroll
                for (int x = 0; x < MINE; ++x) {
                    const int i = x * SUMS + tid;
                    if (i < r.n) mask[i] = make_uint4(m[x].x | all[0], m[x].y | all[1], m[x].z | all[2], m[x].w | all[3]);
                }
                bar_sync(1, SUMS);
            }
            float acc0 = 0.f, acc1 = 0.f;
            for (int h = run.h0; h < run.h1; ++h)
                for (int qb = 0; qb < blocks; ++qb, ++n_q)
                    for (int ti = 0; ti < run.count; ++ti, ++n_s) {
                        if ((int)(n_s % WG) != w) continue;
                        const uint32_t rs = n_q % SR;
                        wait(B, &B->s_full[w], n_s / WG & 1);
                        tc::fence_after();
                        // (the references are there, as the product is; a barrier that this warp does not see every filling of is not waited for ahead of that)
                        wait(B, &B->r_full[rs], n_q / SR & 1);
                        const float *ref = (const float *)(base + S::off_ref) + rs * 128;
                        const unsigned short *nodes = (const unsigned short *)(base + S::off_node) + rs * 128;
                        const int columns = min(S::QB, rows - qb * S::QB);
                        float got = 0.f;
#pragma unroll 1
                        for (int g = 0; g < columns; g += 32) {
                            uint32_t x[32];
                            tc::tmem_load(lanes + w * 128 + g, x);
                            tc::wait_loads(x);
                            if (g + 32 >= columns) {                                       // (the next product may come while these are at work)
                                tc::fence_before();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&B->s_empty[w]);
                            }
                            got += weights_of(x, c2, ref + g, columns - g, masked, mask, nodes + g, quad, lane);
                        }
                        if (ti == 0) acc0 += got; else acc1 += got;
                        __syncwarp();
                        if (lane == 0) tc::arrive_many(&B->r_empty[rs], 3 - run.count);    // (two products to a block of queries: a warp arrives once for each)
                    }
            // the first warpgroups finish a tile each, with what the others have of it
            float *mail = part + (n_step & 1) * (WG * 256);
            mail[w * 256 + mine] = acc0;
            mail[w * 256 + 128 + mine] = acc1;
            bar_sync(1, SUMS);
            float got = 0.f;
            if (w < run.count)
#pragma unroll
                for (int k = 0; k < WG; ++k) got += mail[k * 256 + w * 128 + mine];
            if (slot >= 0 && sound && *(volatile int *)&B->dead == 0) __stcg(P.weights + slot, old + got);
            if (!whole) {
                const int c = blockIdx.x, place = n_step == 0 ? 0 : 1;
                if (w < 2) __stcg(P.part + ((c * 2 + place) * 2 + w) * 128 + mine, got);
                if (run.h0 == 0 && sound) {
                    // the CTA that has a group's first heads tells what there is to join: runs that begin ahead of the group's last unit's end have one
                    // of its units (or are shorter than that and have none at all)
                    const int last = run.at + (P.Hkv - 1) * length_of(run.count);
                    int parts = 1;
                    while (c + parts < P.ctas && cuts.start(c + parts) <= last) ++parts;
                    joint = make_int4(run.b, run.tile, run.count, parts << 1 | place);
                }
            }
        }
        // (a run without a unit: its part of whatever group is 0)
        if (n_step == 0) __stcg(P.part + blockIdx.x * 512 + tid, 0.f);
        static_assert(SUMS == 512, "a thread for an entry of the CTA's parts");
        if (tid == 0) P.joint[blockIdx.x] = joint;
    } else if (warp < KEYS) {
        // ---------------------------------------------------------------- products: two warps in turn, one thread of each issues (a product's 8 instructions,
        // its barriers and the loop around them take some 900 cycles of a warp).  Each waits for every filling of keys and queries, and has a part in
        // letting go of it, whether it has a product with it or not: a barrier's phase tells even fillings from odd ones only.
        const int mine = warp - PRODUCTS;
        const uint32_t k_at = smem_u32(base), q_at = smem_u32(base + S::off_q);
        uint32_t n_k = 0, n_q = 0, n_s = 0;
        const auto gone = [&] { return *(volatile int *)&B->dead != 0; };
        while (run.next(P)) {
            const int rows = run.r.n * P.G, blocks = (rows + S::QB - 1) / S::QB;
            for (int h = run.h0; h < run.h1; ++h, n_k += run.count) {
                for (int qb = 0; qb < blocks; ++qb, ++n_q) {
                    const uint32_t qs = n_q % S::SQ;
                    const int columns = (min(S::QB, rows - qb * S::QB) + 15) / 16 * 16;
                    const uint32_t desc = tc::product_desc(attend::Pair<T>::TYPE, columns, false);
                    wait(B, &B->q_full[qs], n_q / S::SQ & 1);
                    const bool has = run.count == 2 || (int)(n_s & 1) == mine;
                    if (!has && lane == 0) mbar_arrive(&B->q_empty[qs]);
                    for (int ti = 0; ti < run.count; ++ti, ++n_s) {
                        const uint32_t ks = (n_k + ti) % S::SK, buf = n_s & 3;
                        if (qb == 0) wait(B, &B->k_full[ks], (n_k + ti) / S::SK & 1);
                        if ((int)(n_s & 1) != mine) continue;
                        if (n_s >= 4) wait(B, &B->s_empty[buf], (n_s / 4 - 1) & 1);
                        tc::publish_shared();
                        tc::fence_after();
                        if (tc::elected() && !gone()) {
#pragma unroll
                            for (int p = 0; p < S::PANELS; ++p) {
                                const uint64_t kd = tc::panel_desc(k_at + ks * S::K_SLOT + p * PANEL);
                                const uint64_t qd = tc::panel_desc(q_at + qs * S::Q_SLOT + p * S::QB * 128);
#pragma unroll
                                for (int i = 0; i < 4; ++i) tc::mma_ss(tmem + buf * 128, kd + 2 * i, qd + 2 * i, desc, p > 0 || i > 0);
                            }
                            tc::commit(&B->s_full[buf]);
                            tc::commit(&B->q_empty[qs]);
                        }
                        __syncwarp();
                    }
                }
                // (an arrival when this warp's products so far are done; both warps': the keys are free)
                if (tc::elected() && !gone())
                    for (int ti = 0; ti < run.count; ++ti) tc::commit(&B->k_empty[(n_k + ti) % S::SK]);
                __syncwarp();
            }
        }
    } else if (warp < QUERIES) {
        // ---------------------------------------------------------------- keys: a warp for 32 of every tile
        const int which = warp - KEYS;
        constexpr int CH = D / 8;                                     // 16-byte chunks of a row
        const uint32_t k_at = smem_u32(base);
        uint32_t n_k = 0;
        while (run.next(P)) {
            const Request r = run.r;
            int id[2], in[2];
            bool whole[2];
#pragma unroll
            for (int ti = 0; ti < 2; ++ti) {
                const long long key = (long long)(run.tile + ti) * KT + which * 32 + lane;
                id[ti] = -1; in[ti] = 0;
                if (ti < run.count && key >= r.from && key < r.end) {
                    const int col = column_of(P, (int)key);
                    in[ti] = (int)key - col * P.block;
                    id[ti] = __ldg(P.table + (long long)run.b * P.table_stride + col);
                    if (id[ti] >= P.num_blocks) id[ti] = -1;
                }
                whole[ti] = P.box && __all_sync(0xffffffffu, id[ti] >= 0);
            }
            for (int h = run.h0; h < run.h1; ++h)
                for (int ti = 0; ti < run.count; ++ti, ++n_k) {
                    const uint32_t slot = n_k % S::SK;
                    if (n_k >= S::SK) wait(B, &B->k_empty[slot], (n_k / S::SK - 1) & 1);
                    __syncwarp();
                    if (stopped(B)) continue;
                    const uint32_t to = k_at + slot * S::K_SLOT;
                    if (whole[ti]) {
                        // (by one thread, in a loop that the whole warp goes through: boxes from several threads at once go out one by one, far apart)
                        if (tc::elected()) {
                            tc::expect_bytes(&B->k_full[slot], 32 * D * 2);
                            tc::arrive_many(&B->k_full[slot], 32);
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int g = 0; g < 32; g += P.box) {
                            const int block = __shfl_sync(0xffffffffu, id[ti], g), at = __shfl_sync(0xffffffffu, in[ti], g);
                            if (tc::elected()) {
#pragma unroll
                                for (int p = 0; p < S::PANELS; ++p)
                                    tc::box_load(to + p * PANEL + (which * 32 + g) * 128, &P.k_map, p * 64, h, at, block, &B->k_full[slot]);
                            }
                            __syncwarp();
                        }
                    } else {
                        const unsigned long long from = id[ti] >= 0 ? (unsigned long long)((const T *)P.k + id[ti] * P.k_stride[0] + in[ti] * P.k_stride[1] +
                                                                                           h * P.k_stride[2])
                                                                    : (unsigned long long)P.k | 1;           // (odd: zeros)
#pragma unroll 4
                        for (int i = 0; i < CH; ++i) {
                            const int y = i * 32 + lane, row = y / CH, ch = y % CH, at = which * 32 + row;
                            const unsigned long long f = __shfl_sync(0xffffffffu, from, row);
                            tc::copy16(to + ch / 8 * PANEL + at * 128 + (((ch & 7) ^ (at & 7)) << 4), (f & ~1ull) + (f & 1 ? 0 : ch * 16), f & 1 ? 0 : 16);
                        }
                        tc::arrive_with_copies(&B->k_full[slot]);
                    }
                }
        }
        tc::close_copies();
        tc::wait_copies<0>();
    } else {
        // ---------------------------------------------------------------- queries: a warp for 64 rows of every block of them
        const int which = warp - QUERIES;
        constexpr int CH = D / 8;
        const uint32_t q_at = smem_u32(base + S::off_q);
        float *refs = (float *)(base + S::off_ref);
        unsigned short *nodes = (unsigned short *)(base + S::off_node);
        uint32_t n_q = 0;
        while (run.next(P)) {
            const Request r = run.r;
            const int rows = r.n * P.G, blocks = (rows + S::QB - 1) / S::QB;
            // the references of the lane's two rows, asked for a block ahead of their use
            const auto reference = [&](int h, int qb, int x) {
                const int in = which * 64 + x * 32 + lane, row = qb * S::QB + in;
                if (h >= run.h1 || in >= S::QB || row >= rows) return -CUDART_INF_F;
                const int node = node_of(P, row);
                const float l = __ldg(P.lse + ((long long)run.b * P.tree.N + node) * P.Hq + h * P.G + row - node * P.G);
                return fabsf(l) < CUDART_INF_F ? -l * LOG2E : -CUDART_INF_F;
            };
            float ahead[2] = {reference(run.h0, 0, 0), reference(run.h0, 0, 1)};
            for (int h = run.h0; h < run.h1; ++h)
                for (int qb = 0; qb < blocks; ++qb, ++n_q) {
                    const uint32_t slot = n_q % S::SQ;
                    const float ref[2] = {ahead[0], ahead[1]};
#pragma unroll
                    for (int x = 0; x < 2; ++x) ahead[x] = qb + 1 < blocks ? reference(h, qb + 1, x) : reference(h + 1, 0, x);
                    const uint32_t rs = n_q % SR;
                    if (n_q >= SR) wait(B, &B->r_empty[rs], (n_q / SR - 1) & 1);
                    __syncwarp();
                    if (stopped(B)) continue;
                    if (c_hold_slot >= 0 && c_hold_slot / P.tree.N == run.b) continue;       // (a test may ask for a request's queries to stay away)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int in = which * 64 + x * 32 + lane;
                        refs[rs * 128 + in] = ref[x];
                        nodes[rs * 128 + in] = (unsigned short)node_of(P, min(qb * S::QB + in, rows - 1));
                    }
                    mbar_arrive(&B->r_full[rs]);
                    if (n_q >= S::SQ) wait(B, &B->q_empty[slot], (n_q / S::SQ - 1) & 1);
                    __syncwarp();
                    if (stopped(B)) continue;
                    const int columns = min(S::QB, rows - qb * S::QB);
                    if (P.q_nodes && which == 0) {
                        // (rows behind the tree's come as zeros, those behind the box as they are: columns that nobody counts)
                        if (tc::elected()) {
                            tc::expect_bytes(&B->q_full[slot], P.q_nodes * P.G * D * 2);
#pragma unroll
                            for (int p = 0; p < S::PANELS; ++p)
                                tc::box_load(q_at + slot * S::Q_SLOT + p * S::QB * 128, &P.q_map, p * 64, h * P.G, node_of(P, qb * S::QB), run.b,
                                             &B->q_full[slot]);
                        }
                        __syncwarp();
                    }
                    for (int x = 0; x < 2 && !P.q_nodes; ++x) {
                        const int first = which * 64 + x * 32, mine = min(qb * S::QB + first + lane, rows - 1), node = node_of(P, mine);
                        if (first < (columns + 15) / 16 * 16) {
                            const T *q = (const T *)P.q + run.b * P.q_stride[0] + (long long)h * P.G * P.q_stride[2];
                            const uint32_t to = q_at + slot * S::Q_SLOT;
                            const unsigned long long from = (unsigned long long)(q + node * P.q_stride[1] + (mine - node * P.G) * P.q_stride[2]);
#pragma unroll 4
                            for (int i = 0; i < CH; ++i) {
                                const int y = i * 32 + lane, row = y / CH, ch = y % CH, at = first + row;
                                const unsigned long long f = __shfl_sync(0xffffffffu, from, row);
                                tc::copy16(to + ch / 8 * (S::QB * 128) + at * 128 + (((ch & 7) ^ (at & 7)) << 4), f + ch * 16, at < columns ? 16 : 0);
                            }
                        }
                    }
                    tc::arrive_with_copies(&B->q_full[slot]);
                    mbar_arrive(&B->q_full[slot]);
                }
        }
        tc::close_copies();
        tc::wait_copies<0>();
    }
    if (*(volatile int *)&B->dead) {
        // a wait ran out, and nobody waits any more: copies and products under way, which depend on nothing else, get a millisecond to end
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) __nanosleep(1000);
    }
    tc::fence_before();
    __syncthreads();
    if (warp == PRODUCTS) {
        tc::fence_after();
        tc::tmem_free(tmem, 512);
        if (lane == 0) P.late[blockIdx.x] = B->dead;
    }
}

// ---- joining ------------------------------------------------------------------------------------------------------------------
// The first P.ctas CTAs: where that one had a group's first heads and not all of them, the group's sums are added up, in order.  The others: a request
// each, its status (from inputs alone, while the sums are still made).
constexpr int JOIN_NT = 256;

__global__ void __launch_bounds__(JOIN_NT) spec_weigh_join_kernel(const __grid_constant__ Params P)
{
    const int tid = threadIdx.x;
    grid_launch_dependents();                  // (the next kernel waits for this one by itself, and this one for the sums)
    if ((int)blockIdx.x >= P.ctas) {
        const int b = blockIdx.x - P.ctas;
        const int len = __ldg(P.tree.lengths + b), nn = tree_nodes(P.tree, b), n = len < 0 ? 0 : max(nn, 0);
        const int *row = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
        bool bad = false, page = false, late = false;
        for (int i = tid; i < n; i += JOIN_NT) {
            const int p = __ldg(row + i);
            bad |= i == 0 ? p != -1 : p < 0 || p >= i;
        }
        const long long keys = n ? (long long)len + n : 0;
        const int from = P.protect ? max(0, __ldg(P.protect + b)) : 0;
        if (n && from < keys) {
            page = keys > (long long)P.width * P.block;
            const int last = (int)min((keys + P.block - 1) / P.block, (long long)P.width);
            for (int col = from / P.block + tid; col < last; col += JOIN_NT) {
                const int id = __ldg(P.table + (long long)b * P.table_stride + col);
                page |= id < 0 || id >= P.num_blocks;
            }
        }
        bad = __syncthreads_or(bad) != 0;
        page = __syncthreads_or(page) != 0;
        grid_dependency_wait();
        for (int i = tid; i < P.ctas; i += JOIN_NT) late |= *(volatile int *)(P.late + i) != 0;
        late = __syncthreads_or(late) != 0;
        if (tid == 0)
            P.status[b] = len < 0 ? SPEC_DEV_OK
                          : nn < 0 || bad ? SPEC_DEV_TOPOLOGY : late ? SPEC_DEV_TIMEOUT : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
        return;
    }
    grid_dependency_wait();
    const int4 joint = __ldcg(P.joint + blockIdx.x);
    const int w = tid >> 7, mine = tid & 127, parts = joint.w >> 1;
    if (w >= joint.z) return;
    const Request r = request_of(P, joint.x);
    const int entry = (joint.y + w) * KT + mine;
    if (entry < r.from || entry >= r.end) return;
    const int col = column_of(P, entry), id = __ldg(P.table + (long long)joint.x * P.table_stride + col);
    float got = 0.f;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) got += __ldcg(P.part + (((blockIdx.x + k) * 2 + (k ? 0 : joint.w & 1)) * 2 + w) * 128 + mine);
    if (id < 0 || id >= P.num_blocks) return;
    float *to = P.weights + (long long)id * P.block + (entry - col * P.block);
    __stcg(to, (P.fresh && entry >= r.len ? 0.f : __ldcg(to)) + got);
}

}  // namespace weigh
}  // namespace specv
