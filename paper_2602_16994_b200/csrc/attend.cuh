// Attention of the nodes of draft trees over a paged cache (spec_tree_attention).
//
// Mathematics.  A unit is a request, a key head and a block of up to 128 MT of the rows (node, query head of the group) that share this
// head's keys.  Over tiles of 128 keys, S = Q K^T, y = scale log2(e) S - ref, P = 2^y, l += sum P, O += P V, with one reference per row: the
// largest y of what the row saw first, raised (l and O scaled) only when a later y exceeds it by more than 8, so P stays
// below 2^8.  Tiles run from the last to the first: the tree's tile comes first, where every row sees itself.  The result is O / l.
//
// What bounds it.  Per tile and key head 64 KB of keys and values (D = 128): 2740 cycles of an SM's share of the HBM rate at 1.9 GHz.  128
// rows take 1040 cycles of products and about 1100 of arithmetic per scheduler, 256 rows twice that, so up to about 250 rows the cache's
// bytes are the floor, and both products go to the tensor cores even for one row (which fills 1 of 128 lanes).  A thread owns a row, and maxima and
// sums need no exchange.  Measured (one B200): a tile takes 3100 cycles with up to 128 rows (8 requests, 19 nodes, 4 query heads to a key
// head, contexts to 4096: 37 us, floor 15) and 4500 with 204 (128 requests of 51 nodes: 427 to 435 us in a short row of calls, 517 to 524 in a long one, which
// runs into the power limit at 1.64 GHz; floor 226): there a row block's weights wait for its products and these for their turn on the tensor cores.
// Small calls are bound by latency: one token over 8192 keys takes 22 us (floor 5), of which 5 pass until the first scores are there, 1.2 a
// tile, and 6 from the last tile to the joined result.
//
// Precision.  Scores, references, sums and O are fp32.  P is rounded to the type of the values: the product takes two operands of one type, and the rest
// of P as a second operand would cost the products with V again, and their arithmetic.  The rounding is half a step (2^-8 of a weight in bf16,
// 2^-11 in fp16), by itself for every weight, so a row is off by 2^-8 sum p |v| at most; measured against 64 bits, 0.0021 to 0.0023 of the result's norm
// where rounding it once leaves 0.0017 (fp16: 0.00029, 0.00021).  l sums the weights before they are rounded.
//
// Balance.  The tiles of all units, in order, are cut into one run per CTA (one CTA per SM), whatever the lengths: a unit that a
// run ends in leaves its O, l and reference in the workspace, and spec_join_kernel puts such parts together.  Every CTA finds its run from
// the lengths by itself; the host never sees them.
#pragma once
#include <cuda.h>
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
    CUtensorMap k_map, v_map;                  // the caches as [block][slot][head][entry], boxes of `box` slots by 64 entries
    CUtensorMap q_map;                         // the queries as [request][node][head][entry], boxes of 128 rows by 64 entries
    bool q_boxes;                              // (where 128 rows are whole nodes)
    int box;                                   // a power of two up to 32 that divides the block; 0: blocks of no multiple of 8 slots
    TreeArgs tree;
    int B, Hq, Hkv, G, num_blocks, block, width, window, sinks;
    unsigned block_mul;                        // key / block = (umulhi(block_mul, key) + key) >> block_shift for keys below 2^31
    int block_shift;
    unsigned group_mul;                        // row / G likewise
    int group_shift;
    float scale;
    const void *q, *k, *v;
    long long q_stride[3], k_stride[3], v_stride[3];
    const int *table;
    long long table_stride;
    void *out;
    long long out_stride[3];
    float *lse;
    int *status;
    int ctas, groups;                          // CTAs with a run each; groups of JOIN_ROWS rows that a block of rows has at most
    float *part;                               // [ctas][2][D / 4][rows][4] unfinished O
    float2 *ml;                                // [ctas][2][rows] reference and l; reference -inf: none, and l is 1 where keys were seen
    int *late;                                 // [ctas] a wait ran out
    int4 *joint;                               // [ctas] the unit whose first part this is: request, block, head; parts, slot and rows
    // shared prefixes (prefix.cuh)
    int n_groups, n_members, prefix_width;
    const int *group, *members, *first, *place, *shared, *prefix_table;
    long long prefix_stride;
    unsigned nodes_mul;                        // division by N
    int nodes_shift;
    float *whole[2];                           // O of units that were not cut, by row: of requests, of prefixes
    float2 *whole_ml[2];
    int2 *unit[2];                             // where a unit's parts are: first CTA's slot (-1: in whole), number of them
    int unit_blocks;                           // blocks of rows of a request
    int merge_rows;                            // rows of a CTA of the joining kernel
};

// ---- the schedule -------------------------------------------------------------------------------------------------------------
// A unit's length, in tiles, is its tiles and START: what its first segment costs beside them (queries, the tree's tile, results).  A cut in those first
// START goes to the unit's beginning: no run ends with the first tile or two of a unit.
constexpr int START = 2;
// Tiles of a block of rows: [0, sink) and [from, end) of the tiles of its keys.
struct Tiles {
    int sink, from, end;
    __device__ __forceinline__ int count() const { return sink + end - from; }
    __device__ __forceinline__ int tile(int i) const { return i < sink ? i : from + i - sink; }
};
struct Request {
    int len, n, rows;                          // (n = 0 for idle requests)
    int skip;                                  // tokens of its prefix, which other units see to (shared prefixes)
};
// With shared prefixes (SH) the requests' units have those of the groups' prefixes ahead of them: an entry e < n_groups is a prefix, whose rows are those of
// all of the group's members (no tree, the prefix as its committed tokens), entry n_groups + b request b with what lies behind its prefix.
template <bool SH> __device__ __forceinline__ int entries(const Params &P) { return SH ? P.n_groups + P.B : P.B; }
template <bool SH> __device__ __forceinline__ bool is_prefix(const Params &P, int e) { return SH && e < P.n_groups; }
// a group's members are members[x .. y)
__device__ __forceinline__ int2 members_of(const Params &P, int g)
{
    const int x = min(max(__ldg(P.first + g), 0), P.n_members);
    return make_int2(x, min(max(__ldg(P.first + g + 1), x), P.n_members));
}
__device__ __forceinline__ int prefix_len(const Params &P, int g)
{
    return (int)min((long long)min(max(__ldg(P.shared + g), 0), P.prefix_width) * P.block, 0x7FFFFFFFll / P.block * P.block);
}
// tokens of a request's prefix
__device__ __forceinline__ int skip_of(const Params &P, int b)
{
    const int g = __ldg(P.group + b);
    return g < 0 || g >= P.n_groups ? 0 : prefix_len(P, g);
}
template <bool SH> __device__ __forceinline__ Request request_of(const Params &P, int b)
{
    Request r;
    r.skip = 0;
    if (SH) {
        if (b < P.n_groups) {
            const int2 m = members_of(P, b);
            r.len = prefix_len(P, b);
            r.n = 0;
            r.rows = r.len ? (m.y - m.x) * P.tree.N * P.G : 0;
            return r;
        }
        b -= P.n_groups;
        r.skip = skip_of(P, b);
        r.len = __ldg(P.tree.lengths + b);
        r.n = r.len < r.skip ? 0 : max(0, tree_nodes(P.tree, b));
        r.len -= r.skip;
        r.rows = r.n * P.G;
        return r;
    }
    r.len = __ldg(P.tree.lengths + b);
    r.n = r.len < 0 ? 0 : max(0, tree_nodes(P.tree, b));
    r.rows = r.n * P.G;
    return r;
}
__device__ __forceinline__ int node_of(const Params &P, int row)
{
    return (int)((__umulhi(P.group_mul, (unsigned)row) + (unsigned)row) >> P.group_shift);
}
template <bool SH> __device__ __forceinline__ Tiles tiles_of(const Params &P, const Request &r, int m, int block_rows)
{
    if (SH && r.n == 0) return Tiles{0, 0, (int)(((unsigned)r.len + KT - 1) / KT)};                          // a prefix, within its table
    const int last = (m + 1) * block_rows >= r.rows ? r.n - 1 : node_of(P, (m + 1) * block_rows - 1);        // the block's last node
    // (keys behind the table's end have no block: a tile at least, for the rows to come out as those of rows that see nothing)
    const long long held = max(min((long long)P.width * P.block, 0x7FFFFFFFll) - r.skip, 1ll);
    Tiles t;
    t.end = (int)((min((unsigned)r.len + (unsigned)last + 1, (unsigned)held) + KT - 1) / KT);
    t.sink = t.from = 0;
    if (P.window) {
        t.sink = min(t.end, (int)(((unsigned)min(P.sinks, r.len) + KT - 1) / KT));
        t.from = max(min(max(0, r.len - P.window + 1) / KT, t.end - 1), t.sink);
    }
    return t;
}
template <bool SH> __device__ __forceinline__ int tiles_of_request(const Params &P, int b, int block_rows)
{
    const Request r = request_of<SH>(P, b);
    if (is_prefix<SH>(P, b)) return (r.rows + block_rows - 1) / block_rows * (tiles_of<SH>(P, r, 0, block_rows).count() + START) * P.Hkv;
    int s = 0;
    for (int m = 0; m * block_rows < r.rows; ++m) s += tiles_of<SH>(P, r, m, block_rows).count() + START;
    return s * P.Hkv;
}
struct Cuts {                                  // runs of equal length, the first `more` of them longer by one
    int all, each, more;
    __device__ __forceinline__ Cuts(int all_, int ctas) : all(all_), each((int)((unsigned)all_ / (unsigned)ctas)) { more = all - each * ctas; }
    __device__ __forceinline__ int start(int c) const { return each * c + min(c, more); }
};

// A place in the order of all units: request, block of rows, key head, and the way into the unit (START, then its tiles).
struct Place {
    int b, m, h, i;
    __device__ __forceinline__ int tile() const { return max(0, i - START); }
};
// Whether the groups that this thread looks at lie one behind the other among the members.
__device__ __forceinline__ bool groups_in_order(const Params &P, int tid, int threads)
{
    bool good = true;
    for (int g = tid; g < P.n_groups; g += threads) {
        const int x = __ldg(P.first + g), y = __ldg(P.first + g + 1);
        good &= x >= 0 && x <= y && y <= P.n_members;
    }
    return good;
}
// All threads of the CTA: the cuts; in found[], the request that the start of run `c` falls into and the length of all ahead of it.
template <bool SH> __device__ __forceinline__ Cuts find_request(const Params &P, int block_rows, int c, int *sums, int *found, int tid, int threads)
{
    const int n = entries<SH>(P), per = (n + threads - 1) / threads, b0 = min(n, tid * per), b1 = min(n, b0 + per);
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles_of_request<SH>(P, b, block_rows);
    // (groups that overlap could add up to more than the launch was checked for: nothing is done then, and the joining kernel says so)
    if (SH && __syncthreads_or(!groups_in_order(P, tid, threads))) mine = 0;
    const int lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    int upto = lane < warps ? sums[lane] : 0;                      // (at most 32 warps)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
    }
    const int before = __shfl_sync(0xffffffffu, upto, max(warp - 1, 0)), all = __shfl_sync(0xffffffffu, upto, 31);
    int ahead = incl - mine + (warp ? before : 0);
    const Cuts cuts(all, P.ctas);
    const int target = cuts.start(c);
    if (target >= ahead && target < ahead + mine) {
        for (int b = b0; b < b1; ++b) {
            const int t = per == 1 ? mine : tiles_of_request<SH>(P, b, block_rows);
            if (target < ahead + t) { found[0] = b; found[1] = ahead; break; }
            ahead += t;
        }
    }
    __syncthreads();
    return cuts;
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
    int left;
    bool first;
};
// The next segment of a run; false at its end.  (Once in the code: every role of the kernel takes its segments here, and what runs once
// per segment costs its instructions' fetching.)
template <bool SH> static __device__ __noinline__ bool next_segment(const Params &P, int block_rows, Run *run, Segment *s)
{
    if (run->left <= 0) return false;
    Place at = run->at;
    Request r;
    for (;;) {
        if (at.b >= entries<SH>(P)) return false;
        r = request_of<SH>(P, at.b);
        if (at.m * block_rows < r.rows) break;
        ++at.b; at.m = 0;
    }
    const Tiles t = tiles_of<SH>(P, r, at.m, block_rows);
    const int count = t.count(), upto = min(count + START, at.i + run->left), end = max(0, upto - START);
    run->left -= upto - at.i;
    if (end == 0) return false;                // (the run ends before the unit's first tile)
    s->b = at.b; s->m = at.m; s->h = at.h; s->begin = at.tile(); s->end = end;
    s->whole = s->begin == 0 && end == count;
    s->head = run->first;
    s->r = r;
    s->t = t;
    s->rows = min(r.rows - at.m * block_rows, block_rows);
    run->first = false;
    at.i = 0;
    if (++at.h == P.Hkv) { at.h = 0; ++at.m; }
    run->at = at;
    return true;
}
// a warp's run and the segments it has in hand
struct __align__(16) Hand {
    Run run;
    Segment seg[2];
    int more, segments;                        // (segments: how many there were)
    // all lanes of the warp; seg[i] is the next segment
    template <bool SH> __device__ __forceinline__ bool next(const Params &P, int block_rows, int i)
    {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            more = next_segment<SH>(P, block_rows, &run, &seg[i]);
            segments += more;
        }
        __syncwarp();
        return more != 0;
    }
};
// the place `skip` into request b
template <bool SH> __device__ __forceinline__ Place place_in(const Params &P, int b, int skip, int block_rows)
{
    const Request r = request_of<SH>(P, b);
    Place p = {b, 0, 0, 0};
    if (is_prefix<SH>(P, b)) {                 // (its blocks of rows are equally long)
        const int whole = (tiles_of<SH>(P, r, 0, block_rows).count() + START) * P.Hkv;
        p.m = (int)((unsigned)skip / (unsigned)whole);
        skip -= p.m * whole;
    }
    for (; p.m * block_rows < r.rows; ++p.m) {
        const int length = tiles_of<SH>(P, r, p.m, block_rows).count() + START;
        if (skip < length * P.Hkv) {
            p.h = (int)((unsigned)skip / (unsigned)length);
            p.i = skip - p.h * length;
            return p;
        }
        skip -= length * P.Hkv;
    }
    return p;                                  // (not reached: the request has that many tiles)
}

// ---- what a row sees ----------------------------------------------------------------------------------------------------------
// bits of keys a .. a + 31 that lie in [lo, hi)
__device__ __forceinline__ uint32_t bits_of(long long a, long long lo, long long hi)
{
    const int x = (int)min(max(lo - a, 0ll), 32ll), y = (int)min(max(hi - a, 0ll), 32ll);
    if (x >= y) return 0;
    return (y == 32 ? 0xffffffffu : (1u << y) - 1u) & ~((1u << x) - 1u);
}
// Whether every row of any block sees keys a .. a + count - 1 (a node's depth is at most its index).
__device__ __forceinline__ bool seen_by_all(const Params &P, const Request &r, long long a, int count)
{
    const long long e = a + count;
    return e <= r.len && (P.window == 0 || e <= P.sinks || a > (long long)r.len + r.n - 1 - P.window);
}
__device__ __forceinline__ bool seen_by_all(const Params &P, const Request &r, int tile) { return seen_by_all(P, r, (long long)tile * KT, KT); }
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
__device__ __forceinline__ int column_of(const Params &P, int key)
{
    return (int)((__umulhi(P.block_mul, (unsigned)key) + (unsigned)key) >> P.block_shift);
}
// the table's entry of a column, the first being that of the entry's first key; -1 behind the row's end
template <bool SH> __device__ __forceinline__ int id_in(const Params &P, int b, int skip, int col)
{
    if (SH) {
        if (b < P.n_groups) return col < P.prefix_width ? __ldg(P.prefix_table + (long long)b * P.prefix_stride + col) : -1;
        b -= P.n_groups;
        col += skip / P.block;
    }
    return col < P.width ? __ldg(P.table + (long long)b * P.table_stride + col) : -1;
}
// the block of a column; -1 where there is none in the cache
template <bool SH> __device__ __forceinline__ int block_in(const Params &P, int b, int skip, int col)
{
    const int id = id_in<SH>(P, b, skip, col);
    return id < 0 || id >= P.num_blocks ? -1 : id;
}
// A row of a unit (node and head of the group, or member, node and head): whose it is.  b = -1: nobody's (a plan that names no request).
struct RowOf {
    int b, node, head;
};
template <bool SH> __device__ __forceinline__ RowOf row_of(const Params &P, int e, int h, int r)
{
    int node = node_of(P, r);
    const int head = h * P.G + r - node * P.G;
    if (!SH) return RowOf{e, node, head};
    if (e >= P.n_groups) return RowOf{e - P.n_groups, node, head};
    const int i = (int)((__umulhi(P.nodes_mul, (unsigned)node) + (unsigned)node) >> P.nodes_shift);
    const int b = __ldg(P.members + min(members_of(P, e).x + i, P.n_members - 1));
    return RowOf{b < 0 || b >= P.B ? -1 : b, node - i * P.tree.N, head};
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------
// MT = 2: 256 rows, a warpgroup per 128.  MT = 1, WG = 2: 128 rows, the warpgroups take tiles in turn, each with its own O, reference and l,
// put together at the segment's end: one warpgroup's tile takes some 2400 cycles of arithmetic and 1040 of products one after the other, and the
// cache delivers one every 2740.  WG = 1: one warpgroup (D = 256: tensor memory has room for one O).
template <int D_, int MT_, int WG_, bool SH_ = false> struct Shape {
    static constexpr int D = D_, MT = MT_, WG = WG_;
    static constexpr bool SH = SH_;                                               // prefixes are shared
    static constexpr bool TURNS = MT == 1 && WG == 2;
    static constexpr int PARTS = MT == 2 ? 2 : 1, W = KT / PARTS;                 // a tile's columns in parts: see the products
    static constexpr int PANELS = D / 64;
    static constexpr int ROWS = 128 * MT;
    static constexpr int WIDE = PANELS < 2 ? 1 : 2;                               // panels of a slot: up to 128 entries of a tile's rows
    static constexpr int SLOT = WIDE * PANEL, STEP = PANELS / WIDE;               // bytes of a slot; slots of a tile's keys or values
    static constexpr int SLOTS = D == 64 ? 10 : MT == 2 || D == 256 ? 4 : 5;      // slots in flight
    static constexpr int SOFT = 4 * WG, WARPS = SOFT + WG + 4, NT = WARPS * 32;   // warps: rows, products (one per row warpgroup), copies
    static constexpr int NP = 128;                                                // threads that copy
    static constexpr int FILLED = NP + 4;                                         // arrivals that fill a slot: theirs, and one more per warp, see filled()
    static constexpr int O = 256;                                                 // column of the first O; S buffers at 0 and 128
    static constexpr int off_slots = ROWS * D * 2;
    static constexpr int off_parent = off_slots + SLOTS * SLOT;                  // one array of parents per row warpgroup
    static constexpr int off_halves = off_parent + WG * SPEC_MAX_NODES * 2;       // [2][2][128] references and sums of the two turns
    static constexpr int off_hand = off_halves + (TURNS ? 4096 : 0);
    static constexpr int off_bar = off_hand + WARPS * (int)sizeof(Hand);
    static constexpr int total = off_bar + 1024;
    static_assert(off_bar % 16 == 0 && total + 1024 <= 227 * 1024, "shared memory");
};
struct Bars {
    uint64_t full[16], empty[16];
    uint64_t q_full, q_empty, s_full[4], p_full[4], o_empty[2];
    uint64_t pv_done[2][2];                    // per O, even and odd parts: see the rows' wait
    uint32_t tmem;
    int dead, poison, bad_tree;                // (bad_tree: of the request that the rows' parents were read for last)
    uint32_t hidden[8][4];                     // keys of a tile on bad blocks, by the tile's number in the CTA's run % 8
    uint32_t plain[8];                         // a byte per warp that copies: whether it stored (part of) the tile by itself
    int found[2], sums[16];
};
static_assert(sizeof(Bars) <= 1024, "the area behind the buffers");

// ---- where the parts of units lie (shared prefixes) -----------------------------------------------------------------------------
// the row of a unit that was not cut, in whole[]
__device__ __forceinline__ long long whole_row_of(const Params &P, int e, int h, int r)
{
    const long long rows = (long long)P.tree.N * P.G;
    return e < P.n_groups ? ((long long)h * P.n_members + members_of(P, e).x) * rows + r : ((long long)h * P.B + e - P.n_groups) * rows + r;
}
// A unit's place in unit[]: of requests their blocks of rows in order; a group's blocks begin where its rows would, and one further for each group ahead, so
// that no two groups' overlap.
__device__ __forceinline__ long long unit_of(const Params &P, int e, int m, int h, int block_rows)
{
    if (e >= P.n_groups) return ((long long)(e - P.n_groups) * P.unit_blocks + m) * P.Hkv + h;
    return ((long long)members_of(P, e).x * P.tree.N * P.G / block_rows + e + m) * P.Hkv + h;
}
// What the joining kernel is told of a unit, by the CTA that has its first part.
__device__ __forceinline__ void tell_unit(const Params &P, const Segment &seg, const Cuts &cuts, int c, int block_rows)
{
    if (seg.begin != 0) return;
    int last = c;
    if (!seg.whole) {                          // (cut: the run's last segment; the unit's end, from what of it lies in this run)
        const int end = cuts.start(c + 1) + seg.t.count() - seg.end;
        last = c + 1;
        while (cuts.start(last + 1) < end) ++last;
    }
    P.unit[seg.b < P.n_groups][unit_of(P, seg.b, seg.m, seg.h, block_rows)] =
        make_int2(seg.whole ? -1 : 2 * c + (seg.head ? 0 : 1), last + 1 - c);
}

// A bounded wait; once one has run out all others return at once, no copies or products are issued any more, and the kernel comes to its end.
__device__ __forceinline__ void wait(Bars *B, uint64_t *bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return;
    const long long t0 = clock64();
    do {
        if (*(volatile int *)&B->dead) return;
        if (clock64() - t0 > WAIT_CYCLES) { *(volatile int *)&B->dead = 1; return; }
    } while (!mbar_try_wait(bar, parity));
}

// Whether a wait has run out, one answer for the whole (converged) warp: what follows is done by all of its threads or by none.
__device__ __forceinline__ bool stopped(Bars *B) { return __any_sync(0xffffffffu, *(volatile int *)&B->dead) != 0; }

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

// the largest of three, NaN where one of them is
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 2^y of a pair without the special function unit, which does 16 a cycle on an SM and is what the arithmetic of a tile waits for: y = n + f,
// n the nearest integer (adding 1.5 2^23 leaves it in the low bits), 2^f by a polynomial, n added to the exponent.  Exactly 0 for y <= -127.
// The polynomial 1 + f (c_0 + c_1 f + ...) of degree 5 has the smallest largest relative error on [-1/2, 1/2] (minimax under the constant 1, so that 2^0
// is 1; found by linear programming over a grid): 9.2e-8, 1.1e-7 with coefficients in fp32, 1.7e-7 with the arithmetic as well.
__device__ __forceinline__ unsigned long long exp2_pair(unsigned long long y2)
{
    constexpr float EXP2_FIT[5] = {0.69314698f, 0.24022242f, 0.055507337f, 0.0096715126f, 0.0013264727f};
    const auto both = [](float v) { return pack_f32x2(v, v); };
    float y0, y1;
    unpack_f32x2(y2, y0, y1);
    y2 = pack_f32x2(fmaxf(y0, -127.f), fmaxf(y1, -127.f));
    const unsigned long long t = add_f32x2(y2, both(12582912.f)), n = add_f32x2(t, both(-12582912.f)), f = fma_f32x2(n, both(-1.f), y2);
    unsigned long long p = fma_f32x2(f, both(EXP2_FIT[4]), both(EXP2_FIT[3]));
    p = fma_f32x2(p, f, both(EXP2_FIT[2]));
    p = fma_f32x2(p, f, both(EXP2_FIT[1]));
    p = fma_f32x2(p, f, both(EXP2_FIT[0]));
    p = fma_f32x2(p, f, both(1.f));
    float t0, t1, p0, p1;
    unpack_f32x2(t, t0, t1);
    unpack_f32x2(p, p0, p1);
    return pack_f32x2(__int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23)), __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23)));
}
// 32 columns of scores: weights, their sum, and the weights rounded to the values' type, two to a register.  One pair of eight goes without the
// special function unit.  By itself the loop is fastest with three of eight (128 columns of two warps of a scheduler: 1826 cycles, none: 2381), in the
// kernel, whose schedulers have the other roles' instructions to issue as well, with one (128 requests of 51 nodes, short rows of calls: 445 us, three of
// eight: 456, half: 471).
template <typename T>
__device__ __forceinline__ void weigh(const uint32_t (&s)[32], unsigned long long c2, unsigned long long r2, unsigned long long &sum, uint32_t (&pk)[16])
{
#pragma unroll
    for (int k = 0; k < 32; k += 2) {
        const unsigned long long y2 = fma_f32x2(pack_f32x2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, r2);
        unsigned long long p2;
        float x, y;
        if (k % 16 == 14) {
            p2 = exp2_pair(y2);
        } else {
            unpack_f32x2(y2, x, y);
            p2 = pack_f32x2(ex2_approx(x), ex2_approx(y));
        }
        sum = add_f32x2(sum, p2);
        unpack_f32x2(p2, x, y);
        pk[k / 2] = Pair<T>::pack(x, y);
    }
}
// the largest of 32 scores, NaN where one of them is
__device__ __forceinline__ float top_of(const uint32_t (&s)[32])
{
    float top = __uint_as_float(s[0]), other = __uint_as_float(s[1]);         // (two chains)
#pragma unroll
    for (int k = 2; k < 30; k += 4) {
        top = max3(top, __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
        other = max3(other, __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
    }
    return max3(max3(top, other, other), __uint_as_float(s[30]), __uint_as_float(s[31]));
}
// Scores that the row does not see become -inf.
template <int W> __device__ __forceinline__ void hide(uint32_t at, const uint32_t (&words)[4], int first)
{
#pragma unroll 1
    for (int w = 0; w < W / 32; ++w) {
        uint32_t a[32];
        tc::tmem_load(at + 32 * w, a);
        tc::wait_loads(a);
        const int x = first + w;
        const uint32_t word = x == 0 ? words[0] : x == 1 ? words[1] : x == 2 ? words[2] : words[3];
#pragma unroll
        for (int k = 0; k < 32; ++k) a[k] = (word >> k) & 1u ? a[k] : 0xFF800000u;
        tc::tmem_store(at + 32 * w, a);
    }
    tc::wait_stores();
}
// A row's state: reference (any: there is one) and the sum of its weights.
struct Row {
    float ref, l;
    bool any;
};
static __device__ __noinline__ void scale_sums(uint32_t at, int columns, float f)
{
    for (int d = 0; d < columns; d += 32) {
        uint32_t o[32];
        tc::tmem_load(at + d, o);
        tc::wait_loads(o);
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
        tc::tmem_store(at + d, o);
    }
    tc::wait_stores();
}
// The largest of W scores.
template <int W> __device__ __forceinline__ float tile_top(uint32_t at)
{
    float top = -CUDART_INF_F;
#pragma unroll 1
    for (int w = 0; w < W; w += 64) {
        uint32_t a[32], b[32];
        tc::tmem_load(at + w, a);
        tc::tmem_load(at + w + 32, b);
        tc::wait_loads(a);
        tc::wait_loads(b);
        top = max3(top, top_of(a), top_of(b));
    }
    return top;
}
// W weights, put in the place of the scores (16 columns for 32: never beyond the scores that are loaded).  A loop, not copies: the schedulers'
// instruction caches hold the loops of all roles, and fetching what does not fit took longer than the arithmetic (unrolled: 3700
// cycles for a tile of 256 rows, rolled: 1700).
template <typename T, int W> __device__ __forceinline__ float tile_weights(uint32_t at, float c, float ref)
{
    unsigned long long s2 = 0ull;
    const unsigned long long c2 = pack_f32x2(c, c), r2 = pack_f32x2(-ref, -ref);
#pragma unroll 1
    for (int w = 0; w < W / 32; ++w) {
        uint32_t a[32], pk[16];
        tc::tmem_load(at + 32 * w, a);
        tc::wait_loads(a);
        weigh<T>(a, c2, r2, s2, pk);
        tc::tmem_store16(at + 16 * w, pk);
    }
    float x, y;
    unpack_f32x2(s2, x, y);
    return x + y;
}
// Values that are not finite were taken out of tiles that not all rows see; those that this row sees come back, into columns d .. d + 31.
template <typename T, bool SH>
__device__ __noinline__ void put_back(const Params &P, const Segment &seg, int node, int depth, const unsigned short *parent, int d, float *o)
{
    Walk walk = {node, 0};
    for (int step = 0; step < seg.steps(); ++step) {
        const int tile = seg.tile(step);
        if (seen_by_all(P, seg.r, tile)) continue;
        uint32_t words[4];
        seen_words(P, seg.r, tile, depth, parent, walk, words);
        for (int j = 0; j < KT; ++j) {
            const uint32_t word = j < 32 ? words[0] : j < 64 ? words[1] : j < 96 ? words[2] : words[3];
            if (!((word >> (j & 31)) & 1u)) continue;
            const int key = tile * KT + j, col = column_of(P, key), id = block_in<SH>(P, seg.b, seg.r.skip, col);
            if (id < 0) continue;
            const unsigned short *v = (const unsigned short *)P.v + id * P.v_stride[0] + (key - col * P.block) * P.v_stride[1] + seg.h * P.v_stride[2] + d;
            for (int k = 0; k < 32; ++k) {
                const float x = Pair<T>::value(__ldg(v + k));
                if (!(fabsf(x) < CUDART_INF_F)) o[k] += x;
            }
        }
    }
}

// Whether a row sees any key of a segment: asked for rows whose weights came to nothing, which are 0 where they see nothing, and no number where all that
// they see has a score of -inf (0 / 0).
template <bool SH> static __device__ __noinline__ bool sees_any(const Params &P, const Segment &seg, int node, int depth, const unsigned short *parent)
{
    Walk walk = {node, 0};
    for (int step = 0; step < seg.steps(); ++step) {
        const int tile = seg.tile(step);
        uint32_t words[4];
        seen_words(P, seg.r, tile, depth, parent, walk, words);
        for (int j = 0; j < KT; ++j) {
            const uint32_t word = j < 32 ? words[0] : j < 64 ? words[1] : j < 96 ? words[2] : words[3];
            if (((word >> (j & 31)) & 1u) && block_in<SH>(P, seg.b, seg.r.skip, column_of(P, tile * KT + j)) >= 0) return true;
        }
    }
    return false;
}

template <typename T, typename S> __global__ void __launch_bounds__(S::NT, 1) spec_attend_kernel(const __grid_constant__ Params P)
{
    constexpr int D = S::D, MT = S::MT;
    unsigned char *base = dyn_smem + (-smem_u32(dyn_smem) & 1023u);
    Bars *B = (Bars *)(base + S::off_bar);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
    Hand *hand = (Hand *)(base + S::off_hand) + warp;
    // what needs no input comes ahead of the wait for the kernel before
    if (warp == S::SOFT) tc::tmem_alloc(&B->tmem, 512);
    if (tid == S::NT - 1 && P.box) { tc::prefetch_map(&P.k_map); tc::prefetch_map(&P.v_map); }
    if (tid == 0) {
        for (int i = 0; i < S::SLOTS; ++i) { mbar_init(&B->full[i], S::FILLED); mbar_init(&B->empty[i], MT); }
        mbar_init(&B->q_full, S::NP);
        mbar_init(&B->q_empty, S::WG);
        for (int t = 0; t < 4; ++t) { mbar_init(&B->s_full[t], 1); mbar_init(&B->p_full[t], 4); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&B->pv_done[t][0], 1);
            mbar_init(&B->pv_done[t][1], 1);
            mbar_init(&B->o_empty[t], S::TURNS ? 8 : 4);
        }
        B->dead = 0;
        B->poison = 0;
        B->bad_tree = 0;
        mbar_fence_init();
    }
    grid_dependency_wait();
    grid_launch_dependents();                  // (the joining kernel's CTAs may be placed beside this one's; they wait by themselves)
    static_assert(S::NT / 32 <= (int)(sizeof(B->sums) / sizeof(int)), "an entry of sums for every warp");
    const Cuts cuts = find_request<S::SH>(P, S::ROWS, c, B->sums, B->found, tid, S::NT);
    if (lane == 0) {
        hand->run.left = cuts.start(c + 1) - cuts.start(c);
        hand->run.first = true;
        hand->segments = 0;
        if (hand->run.left > 0) hand->run.at = place_in<S::SH>(P, B->found[0], cuts.start(c) - B->found[1], S::ROWS);
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = B->tmem;
    if (warp < S::SOFT) {
        // ---------------------------------------------------------------- rows: a thread owns one
        const int w = warp >> 2, quad = warp & 3, t = MT == 2 ? w : 0, row = t * 128 + quad * 32 + lane, gt = tid & 127;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16), o_at = lanes + S::O + w * D;
        unsigned short *parent = (unsigned short *)(base + S::off_parent) + w * SPEC_MAX_NODES;
        float2 *halves = (float2 *)(base + S::off_halves);
        const float c = P.scale * LOG2E;
        uint32_t n_part = 0, n_run = 0, n_seg = 0;     // parts of tiles that this warpgroup has been through, tiles of the run, segments
        int tree_of = -1;
        // The wait for the product of part n with the values.  Scores run up to two parts ahead of these products, and a barrier's phase tells even numbers
        // from odd ones only: with one barrier for all parts, waiting for the last but one did not end where the last had already come as well, and
        // without waiting for it the last could not be told from the one two before.  So even and odd parts have a barrier each, and part n + 2 waits
        // for this warp.
        const auto products = [&](uint32_t n) { wait(B, &B->pv_done[w][n & 1], n >> 1 & 1); };
        Segment &seg = hand->seg[0];
        for (; hand->template next<S::SH>(P, S::ROWS, 0); ++n_seg) {
            const int steps = seg.steps();
            if (t * 128 >= seg.rows) {
                n_run += steps;
                continue;
            }
            const int r = seg.m * S::ROWS + row;
            const RowOf of_row = row_of<S::SH>(P, seg.b, seg.h, min(r, seg.r.rows - 1));
            const bool prefix = is_prefix<S::SH>(P, seg.b);
            const int node = prefix ? -1 : of_row.node;                        // (no row of a prefix is in a tree)
            const bool live = row < seg.rows, warp_live = t * 128 + quad * 32 < seg.rows;
            if (!prefix && tree_of != seg.b && (tree_of < 0 || P.tree.topo_seq_stride || P.tree.n_nodes)) {
                if (tid == 0) B->bad_tree = 0;
                bar_sync(1 + w, 128);
                const int *from = P.tree.parent + (long long)of_row.b * P.tree.topo_seq_stride;
                for (int i = gt; i < seg.r.n; i += 128) {
                    const int p = __ldg(from + i);
                    parent[i] = p >= 0 && p < i ? (unsigned short)p : (unsigned short)0xFFFF;
                    if (w == 0 && (i == 0 ? p != -1 : p < 0 || p >= i)) *(volatile int *)&B->bad_tree = 1;
                }
                tree_of = seg.b;
                bar_sync(1 + w, 128);
            }
            int depth = 0;
            if (!S::SH && P.window)
                for (unsigned short x = parent[node]; x != 0xFFFF; x = parent[x]) ++depth;
            Walk walk = {node, 0};
            Row of = {0.f, 0.f, false};
            bool begun = false;                        // whether there has been a tile
            for (int step = 0; step < steps; ++step, ++n_run) {
                if (S::TURNS && (int)(n_run & 1) != w) continue;
                uint32_t words[4] = {0u, 0u, 0u, 0u};
                bool masked = false;
#pragma unroll 1
                for (int h = 0; h < S::PARTS; ++h, ++n_part) {
                    const int buf = MT == 2 ? t * S::PARTS + h : n_run & 1;
                    const uint32_t s_at = lanes + buf * S::W;
                    wait(B, &B->s_full[buf], (MT == 2 ? n_part / S::PARTS : n_run >> 1) & 1);
                    tc::fence_after();
                    if (warp_live) {
                        if (h == 0) {
                            const int tile = seg.tile(step);
                            const volatile uint32_t *hidden = B->hidden[n_run & 7];
                            const uint32_t h0 = hidden[0], h1 = hidden[1], h2 = hidden[2], h3 = hidden[3];
                            masked = !seen_by_all(P, seg.r, tile) || (h0 | h1 | h2 | h3) != 0;
                            if (masked) {
                                seen_words(P, seg.r, tile, depth, parent, walk, words);
                                words[0] &= ~h0; words[1] &= ~h1; words[2] &= ~h2; words[3] &= ~h3;
                            }
                        }
                        if (masked) hide<S::W>(s_at, words, h * (S::W / 32));
                        const float top = tile_top<S::W>(s_at) * c;                // (c > 0)
                        const bool over = of.any ? !(top <= of.ref + 8.f) : !(top <= -CUDART_INF_F);
                        if (__any_sync(0xffffffffu, over)) {
                            // a new reference: what has been summed is scaled
                            float f = 1.f;
                            if (over) {
                                // (the first one is the largest score, which gets the weight 1; later ones lie whole numbers above it, so that what is
                                // scaled keeps its digits; a score that is no number, or infinite, leaves the row no number either, for good)
                                const float up = of.any ? ceilf(top - of.ref) : 0.f;
                                if (of.any) f = ex2_approx(-up);
                                of.ref = top < CUDART_INF_F && of.ref == of.ref ? (of.any ? of.ref + up : top) : CUDART_NAN_F;
                                of.any = true;
                            }
                            of.l *= f;
                            if (begun && __any_sync(0xffffffffu, f != 1.f)) {
                                products(n_part - 1);
                                tc::fence_after();
                                scale_sums(o_at, D, f);
                            }
                        }
                        of.l += tile_weights<T, S::W>(s_at, c, of.ref);
                        tc::wait_stores();
                        tc::fence_before();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&B->p_full[buf]);
                    begun = true;
                }
            }
            // the segment's end (products come to their end in order: the last is the last of all)
            if (begun) products(n_part - 1);
            tc::fence_after();
            float ref = of.ref, l = of.l, f0 = 1.f, f1 = 0.f;
            bool any = of.any;
            if (S::TURNS) {
                // both turns' references and sums, then both O: this warpgroup gives out half of the columns
                float2 *mine = halves + (n_seg & 1) * 256;
                mine[w * 128 + gt] = make_float2(any ? ref : -CUDART_INF_F, l);
                tc::fence_before();
                bar_sync(3, 256);
                tc::fence_after();
                const float2 x = mine[gt], y = mine[128 + gt];
                ref = x.x >= y.x || x.x != x.x ? x.x : y.x;                  // (NaN if one is)
                f0 = x.x == -CUDART_INF_F ? 0.f : ex2_approx(x.x - ref);
                f1 = y.x == -CUDART_INF_F ? 0.f : ex2_approx(y.x - ref);
                any = f0 != 0.f || f1 != 0.f;
                l = (f0 == 0.f ? 0.f : f0 * x.y) + (f1 == 0.f ? 0.f : f1 * y.y);
            }
            if (warp_live) {
                const bool poison = *(volatile int *)&B->poison != 0;
                const bool only = live && l == 0.f && sees_any<S::SH>(P, seg, node, depth, parent);         // sees keys, all with a score of -inf
                const float inv = l == 0.f ? only ? CUDART_NAN_F : 0.f : 1.f / l;
                const long long slot = (long long)blockIdx.x * 2 + (seg.head ? 0 : 1);
                const int head = of_row.head;
                // (a row that has a prefix elsewhere is put together with it)
                const bool direct = seg.whole && (!S::SH || (!prefix && seg.r.skip == 0));
                T *to = (T *)P.out + max(of_row.b, 0) * P.out_stride[0] + of_row.node * P.out_stride[1] + head * P.out_stride[2];
                float *part = P.part + slot * S::ROWS * D;
                const long long whole_row = S::SH ? whole_row_of(P, seg.b, seg.h, r) : 0;
                const int d0 = S::TURNS ? w * (D / 2) : 0, d1 = S::TURNS ? d0 + D / 2 : D;
#pragma unroll 1
                for (int d = d0; d < d1; d += 32) {
                    uint32_t o[32];
                    tc::tmem_load((S::TURNS ? lanes + S::O : o_at) + d, o);
                    tc::wait_loads(o);
                    if (S::TURNS) {
                        uint32_t o1[32];
                        tc::tmem_load(lanes + S::O + D + d, o1);
                        tc::wait_loads(o1);
#pragma unroll
                        for (int k = 0; k < 32; ++k)                          // (a turn without a tile has no O)
                            o[k] = __float_as_uint((f0 == 0.f ? 0.f : f0 * __uint_as_float(o[k])) + (f1 == 0.f ? 0.f : f1 * __uint_as_float(o1[k])));
                    }
                    if (poison && live) {
                        float x[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = __uint_as_float(o[k]);
                        put_back<T, S::SH>(P, seg, node, depth, parent, d, x);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(x[k]);
                    }
                    if (!live) continue;
                    if (direct) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            uint4 x;
                            x.x = Pair<T>::pack(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv);
                            x.y = Pair<T>::pack(__uint_as_float(o[k + 2]) * inv, __uint_as_float(o[k + 3]) * inv);
                            x.z = Pair<T>::pack(__uint_as_float(o[k + 4]) * inv, __uint_as_float(o[k + 5]) * inv);
                            x.w = Pair<T>::pack(__uint_as_float(o[k + 6]) * inv, __uint_as_float(o[k + 7]) * inv);
                            *(uint4 *)(to + d + k) = x;
                        }
                    } else if (S::SH && seg.whole) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *(uint4 *)(P.whole[prefix] + ((whole_row >> 5) * (D / 4) + (d + k) / 4) * 128 + (whole_row & 31) * 4) =
                                make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *(uint4 *)(part + ((long long)((d + k) / 4) * S::ROWS + row) * 4) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    }
                }
                if (live && d0 == 0) {
                    if (direct) {
                        if (P.lse)
                            P.lse[((long long)of_row.b * P.tree.N + of_row.node) * P.Hq + head] = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
                    } else if (S::SH && seg.whole) {
                        P.whole_ml[prefix][whole_row] = make_float2(any ? ref : -CUDART_INF_F, only ? 1.f : l);
                    } else {
                        P.ml[slot * S::ROWS + row] = make_float2(any ? ref : -CUDART_INF_F, only ? 1.f : l);
                    }
                }
                tc::fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&B->o_empty[t]);
        }
    } else if (warp < S::SOFT + S::WG) {
        // ---------------------------------------------------------------- products: one thread issues, the warp waits.  A warp per row warpgroup: what
        // one spends on barriers (some 800 cycles a tile) passes while the tensor cores work for the other.
        const int m = warp - S::SOFT;
        constexpr uint32_t DS = tc::product_desc(Pair<T>::TYPE, S::W, false), DO = tc::product_desc(Pair<T>::TYPE, 64 * S::WIDE, true);
        const uint32_t q_at = smem_u32(base), slots = smem_u32(base + S::off_slots);
        uint32_t n = 0, n_seg = 0, n_tile = 0, n_mine = 0, n_o = 0;    // next slot; segments and tiles of the run; own tiles, own segments
        // the copies to slots k .., of the run's tile i, are there; what threads stored, seen through the barrier, is put before the tensor cores.
        // In turns a slot's last contents may have been the other warp's: a phase tells even fillings from odd ones only, so that one is first seen let
        // go of, or its not yet having come would look like the next one's being there.
        const auto copied = [&](uint32_t k, uint32_t i) {
            for (int p = 0; p < S::STEP; ++p) {
                const uint32_t slot = (k + p) % S::SLOTS, filling = (k + p) / S::SLOTS;
                if (S::TURNS && filling > 0) wait(B, &B->empty[slot], (filling - 1) & 1);
                wait(B, &B->full[slot], filling & 1);
            }
            if (*(volatile uint32_t *)&B->plain[i & 7]) tc::publish_shared();
            tc::fence_after();
        };
        // (asked by the one thread that issues, behind the choice of it, which takes the whole warp)
        const auto gone = [&] { return *(volatile int *)&B->dead != 0; };
        // S of row block t for part h of a tile into columns `to`, from the keys in slots k ..; `bar`: where that is told
        const auto scores = [&](int t, int h, int to, uint32_t k, uint64_t *bar, bool release) {
            if (tc::elected() && !gone()) {
#pragma unroll
                for (int p = 0; p < S::STEP; ++p) {
                    const uint32_t slot = (k + p) % S::SLOTS;
#pragma unroll
                    for (int x = 0; x < S::WIDE; ++x) {
                        const uint64_t qd = tc::panel_desc(q_at + ((p * S::WIDE + x) * MT + t) * PANEL);
                        const uint64_t kd = tc::panel_desc(slots + slot * S::SLOT + x * PANEL + h * S::W * 128);
#pragma unroll
                        for (int i = 0; i < 4; ++i) tc::mma_ss(tmem + to, qd + 2 * i, kd + 2 * i, DS, p > 0 || x > 0 || i > 0);
                    }
                    if (release) tc::commit(&B->empty[slot]);
                }
                tc::commit(bar);
            }
            __syncwarp();
        };
        // O number o (+)= P (in columns `from`) V for part h of a tile, the part'th of this O's parts, from the values in slots k ..
        const auto sums = [&](int o, int h, uint32_t part, int from, uint32_t k, bool add, bool release) {
            if (tc::elected() && !gone()) {
#pragma unroll
                for (int p = 0; p < S::STEP; ++p) {
                    const uint32_t slot = (k + p) % S::SLOTS;
                    const uint64_t vd = tc::panel_desc(slots + slot * S::SLOT + h * S::W * 128);
#pragma unroll
                    for (int i = 0; i < S::W / 16; ++i)
                        tc::mma_ts(tmem + S::O + o * D + p * 128, tmem + from + i * 8, vd + i * (2048 >> 4), DO, add || i > 0);
                    if (release) tc::commit(&B->empty[slot]);
                }
                tc::commit(&B->pv_done[o][part & 1]);
            }
            __syncwarp();
        };
        const auto let_go = [&](uint64_t *bar) {
            if (tc::elected() && !gone()) tc::commit(bar);
            __syncwarp();
        };
        // (the slots' order: K0, V0, K1, V1, ...)
        const auto keys_of = [&](int i) { return n + 2 * S::STEP * i; };
        const auto values_of = [&](int i) { return n + 2 * S::STEP * i + S::STEP; };
        for (; hand->template next<S::SH>(P, S::ROWS, 0); ++n_seg) {
            if (S::SH && warp == S::SOFT && lane == 0) tell_unit(P, hand->seg[0], cuts, c, S::ROWS);
            const int steps = hand->seg[0].steps();
            const bool mine = MT == 1 || m * 128 < hand->seg[0].rows;
            wait(B, &B->q_full, n_seg & 1);
            if (!P.q_boxes) tc::publish_shared();
            if (MT == 2 && !mine) {
                for (int i = 0; i < steps; ++i) {
                    copied(keys_of(i), n_tile + i);
                    for (int p = 0; p < S::STEP; ++p) let_go(&B->empty[(keys_of(i) + p) % S::SLOTS]);
                    copied(values_of(i), n_tile + i);
                    for (int p = 0; p < S::STEP; ++p) let_go(&B->empty[(values_of(i) + p) % S::SLOTS]);
                }
                let_go(&B->q_empty);
            } else if (MT == 2) {
                // A tile in two parts of 64 keys: while the weights of one part are at work the other has its products, and its next scores right behind
                // them.  (Products of a part: 8 with N = 64 for S, which take as long as 6 of full width, 4 with N = 128 for O.  128 requests of 51 nodes, when
                // this was chosen: 457 us; scores of a whole tile at once, which are ready later: 498; weights of a whole tile at once as well: 505.)
                copied(n, n_tile);
                for (int h = 0; h < S::PARTS; ++h) scores(m, h, (m * S::PARTS + h) * S::W, n, &B->s_full[m * S::PARTS + h], h == S::PARTS - 1);
                if (steps == 1) let_go(&B->q_empty);
#pragma unroll 1
                for (int i = 0; i < steps; ++i, ++n_mine) {
                    const bool more = i + 1 < steps;
                    copied(values_of(i), n_tile + i);
#pragma unroll 1
                    for (int h = 0; h < S::PARTS; ++h) {
                        const int buf = m * S::PARTS + h;
                        const bool last = h == S::PARTS - 1;
                        wait(B, &B->p_full[buf], n_mine & 1);
                        if (i == 0 && h == 0 && n_o) wait(B, &B->o_empty[m], (n_o - 1) & 1);
                        tc::fence_after();
                        sums(m, h, n_mine * S::PARTS + h, buf * S::W, values_of(i), i > 0 || h > 0, last);
                        if (!more) continue;
                        if (h == 0) copied(keys_of(i + 1), n_tile + i + 1);
                        scores(m, h, buf * S::W, keys_of(i + 1), &B->s_full[buf], last);
                    }
                    if (i + 2 == steps) let_go(&B->q_empty);
                }
                ++n_o;
            } else if (S::TURNS) {
                const int first = (int)((m - n_tile) & 1);
                if (first >= steps) let_go(&B->q_empty);
#pragma unroll 1
                for (int i = first; i < steps; i += 2, ++n_mine) {
                    copied(keys_of(i), n_tile + i);
                    scores(0, 0, m * 128, keys_of(i), &B->s_full[m], true);
                    if (i + 2 >= steps) let_go(&B->q_empty);
                    copied(values_of(i), n_tile + i);
                    wait(B, &B->p_full[m], n_mine & 1);
                    if (i == first && n_seg) wait(B, &B->o_empty[0], (n_seg - 1) & 1);
                    tc::fence_after();
                    sums(m, 0, n_mine, m * 128, values_of(i), i > first, true);
                }
            } else {
                // scores a tile ahead
                copied(n, n_tile);
                scores(0, 0, (n_tile & 1) * 128, n, &B->s_full[n_tile & 1], true);
                if (steps == 1) let_go(&B->q_empty);
#pragma unroll 1
                for (int i = 0; i < steps; ++i) {
                    const uint32_t at = n_tile + i;
                    if (i + 1 < steps) {
                        copied(keys_of(i + 1), at + 1);
                        scores(0, 0, (at + 1 & 1) * 128, keys_of(i + 1), &B->s_full[at + 1 & 1], true);
                        if (i + 2 == steps) let_go(&B->q_empty);
                    }
                    copied(values_of(i), at);
                    wait(B, &B->p_full[at & 1], (at >> 1) & 1);
                    if (i == 0 && n_seg) wait(B, &B->o_empty[0], (n_seg - 1) & 1);
                    tc::fence_after();
                    sums(0, 0, at, (at & 1) * 128, values_of(i), i > 0, true);
                }
            }
            n_tile += steps;
            n += 2 * S::STEP * steps;
        }
    } else {
        // ---------------------------------------------------------------- copies: a warp for 32 rows of every tile, each for itself
        const int part = warp - S::SOFT - S::WG;
        constexpr int CH = D / 8;                                     // 16-byte chunks of a row
        const uint32_t slots = smem_u32(base + S::off_slots), q_at = smem_u32(base);
        uint32_t n = 0, n_seg = 0, n_tile = 0;                        // n: the next slot to fill
        // Blocks of boxes of at least 8 slots go by the tensor map, a box per thread and panel.  Where not all rows see all of the warp's keys, or a
        // block is bad, the warp's threads copy: keys that no row sees, or on bad blocks, as zeros, nothing of them is read.  Such copies arrive
        // on their barrier by themselves, but for values: entries that are not finite leave those first, as 0 times them would reach rows that do
        // not see them.  That waits until the next copies are under way, or until there is no room for them.
        bool late_values = false;
        uint32_t late_slot = 0;
        const auto place = [&](uint32_t slot, int row, int chunk) {
            return (slot + chunk / (8 * S::WIDE)) % S::SLOTS * S::SLOT + chunk / 8 % S::WIDE * PANEL + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
        };
        // The warp's own arrival, by the thread that wrote the tile's `hidden` and `plain`: an arrival that copies make when they are done says nothing
        // of what their thread stored beside them.
        const auto filled = [&](uint64_t *bar) { if (lane == 0) mbar_arrive(bar); };
        const auto clean = [&]() {
#pragma unroll 1
            for (int i = 0; i < CH; ++i) {
                const int x = i * 32 + lane;
                unsigned char *at = base + S::off_slots + place(late_slot, part * 32 + x / CH, x % CH);
                uint4 v = *(uint4 *)at;
                uint32_t *e = (uint32_t *)&v;
                bool bad = false;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (Pair<T>::finite(e[k])) continue;
                    bad = true;
                    const uint32_t lo = e[k] & 0xFFFFu, hi = e[k] & 0xFFFF0000u;
                    e[k] = (Pair<T>::finite(lo) ? lo : 0u) | (Pair<T>::finite(hi) ? hi : 0u);
                }
                if (bad) { *(uint4 *)at = v; *(volatile int *)&B->poison = 1; }
            }
            tc::publish_shared();
            for (int p = 0; p < S::STEP; ++p) {
                uint64_t *bar = &B->full[(late_slot + p) % S::SLOTS];
                mbar_arrive(bar);
                filled(bar);
            }
            late_values = false;
        };
        // a wait for room: values that are held back may be what the room is waiting for
        const auto room = [&](uint64_t *bar, uint32_t parity) {
            if (late_values && !__all_sync(0xffffffffu, mbar_test(bar, parity))) { tc::wait_copies<0>(); clean(); }
            wait(B, bar, parity);
            __syncwarp();
        };
        // Block and slot of the lane's key of a tile, asked for a tile ahead of its use.  whole: all rows see all of the warp's keys.
        struct Source { int id, in, h, b; bool seen, whole; };
        const auto source = [&](const Segment &s, int tile) {
            const long long first = (long long)tile * KT + part * 32, key = first + lane;
            Source x = {-1, 0, s.h, s.b,
                        key < (long long)s.r.len + s.r.n &&
                            (key >= s.r.len || P.window == 0 || key < P.sinks || key > (long long)s.r.len - P.window),
                        seen_by_all(P, s.r, first, 32)};
            if (x.seen) {
                const int col = column_of(P, (int)key);
                x.in = (int)key - col * P.block;
                x.id = id_in<S::SH>(P, s.b, s.r.skip, col);
            }
            return x;
        };
        const auto copy_rows = [&](const Source &x, bool by_map, bool values) {
            for (int p = 0; p < S::STEP; ++p) {
                const uint32_t k = n + p;
                if (k >= S::SLOTS) room(&B->empty[k % S::SLOTS], (k / S::SLOTS - 1) & 1);
            }
            if (stopped(B)) { n += S::STEP; return; }
            bool hold = false;
            if (by_map) {
                // (by one thread, in a loop that the whole warp goes through: from several threads at once they went out one by one all the same, but 290
                // cycles apart)
                if (tc::elected()) {
                    for (int p = 0; p < S::STEP; ++p) {
                        uint64_t *bar = &B->full[(n + p) % S::SLOTS];
                        tc::expect_bytes(bar, 32 * 128 * S::WIDE);
                        tc::arrive_many(bar, S::FILLED / 4);
                    }
                }
                __syncwarp();
                const CUtensorMap *map = values ? &P.v_map : &P.k_map;
#pragma unroll 1
                for (int g = 0; g < 32; g += P.box) {
                    const int id = __shfl_sync(0xffffffffu, x.id, g), in = __shfl_sync(0xffffffffu, x.in, g);
                    if (tc::elected()) {
#pragma unroll
                        for (int k = 0; k < S::PANELS; ++k)
                            tc::box_load(slots + place(n, part * 32 + g, k * 8), map, k * 64, x.h, in, id, &B->full[(n + k / S::WIDE) % S::SLOTS]);
                    }
                    __syncwarp();
                }
            } else {
                const long long *st = values ? P.v_stride : P.k_stride;
                const T *from = (const T *)(values ? P.v : P.k);
                const bool good = x.seen && x.id >= 0 && x.id < P.num_blocks;
                // (odd: zeros)
                const unsigned long long a = good ? (unsigned long long)(from + x.id * st[0] + x.in * st[1] + x.h * st[2]) : (unsigned long long)from | 1;
#pragma unroll 4
                for (int i = 0; i < CH; ++i) {
                    const int y = i * 32 + lane, row = y / CH;
                    const unsigned long long f = __shfl_sync(0xffffffffu, a, row);
                    tc::copy16(slots + place(n, part * 32 + row, y % CH), (f & ~1ull) + (y % CH) * 16, f & 1 ? 0 : 16);
                }
                hold = values && !x.whole;
                if (!hold)
                    for (int p = 0; p < S::STEP; ++p) {
                        uint64_t *bar = &B->full[(n + p) % S::SLOTS];
                        tc::arrive_with_copies(bar);
                        filled(bar);
                    }
            }
            tc::close_copies();
            if (late_values) { tc::wait_copies<1>(); clean(); }
            if (hold) { late_values = true; late_slot = n; }
            n += S::STEP;
        };
        // (A warp waits only for room that it fills itself: where a unit has one tile, the products let go of its queries as soon as the keys are there,
        // and a warp that comes to ask after that, and has no part in the next queries, would find a phase that is not told from the one before.)
        const auto copy_q = [&](const Segment &s) {
            if (P.q_boxes && part != 0) return;
            if (n_seg) room(&B->q_empty, (n_seg - 1) & 1);
            ++n_seg;
            if (stopped(B)) return;
            if (c_hold_slot >= 0 && c_hold_slot / P.tree.N == (S::SH ? s.b - P.n_groups : s.b)) return;       // (a test may ask for a request's queries to stay away)
            if (P.q_boxes) {
                // (nodes beyond N come as zeros)
                if (lane == 0) {
                    tc::expect_bytes(&B->q_full, S::ROWS * D * 2);
                    tc::arrive_many(&B->q_full, S::NP);
                }
                __syncwarp();
                if (lane < S::PANELS * MT)
                    tc::box_load(q_at + lane * PANEL, &P.q_map, lane / MT * 64, s.h * P.G, node_of(P, s.m * S::ROWS + lane % MT * 128), s.b, &B->q_full);
                return;
            }
            if (S::SH) {
                // (rows of several requests: a lane finds a row's place for all)
#pragma unroll 1
                for (int x = 0; x < MT; ++x) {
                    const int first = part * (32 * MT) + x * 32, mine = s.m * S::ROWS + first + lane;
                    const RowOf at = row_of<S::SH>(P, s.b, s.h, min(mine, s.r.rows - 1));
                    const bool in = first + lane < s.rows && at.b >= 0;
                    const unsigned long long a =
                        in ? (unsigned long long)((const T *)P.q + at.b * P.q_stride[0] + at.node * P.q_stride[1] + at.head * P.q_stride[2])
                           : (unsigned long long)P.q | 1;                        // (odd: zeros)
#pragma unroll 4
                    for (int i = 0; i < CH; ++i) {
                        const int y = i * 32 + lane, row = first + y / CH, ch = y % CH;
                        const unsigned long long f = __shfl_sync(0xffffffffu, a, y / CH);
                        tc::copy16(q_at + ((ch / 8) * MT + row / 128) * PANEL + row % 128 * 128 + (((ch & 7) ^ (row & 7)) << 4),
                                   (f & ~1ull) + (f & 1 ? 0 : ch * 16), f & 1 ? 0 : 16);
                    }
                }
                tc::arrive_with_copies(&B->q_full);
                tc::close_copies();
                return;
            }
            const T *q = (const T *)P.q + s.b * P.q_stride[0] + s.h * P.G * P.q_stride[2];
#pragma unroll 4
            for (int i = 0; i < MT * CH; ++i) {
                const int y = i * 32 + lane, row = part * (32 * MT) + y / CH, c = y % CH, r = s.m * S::ROWS + row, node = node_of(P, r);
                const bool in = row < s.rows;
                tc::copy16(q_at + ((c / 8) * MT + row / 128) * PANEL + row % 128 * 128 + (((c & 7) ^ (row & 7)) << 4),
                           (unsigned long long)(in ? q + node * P.q_stride[1] + (r - node * P.G) * P.q_stride[2] + c * 8 : (const T *)P.q), in ? 16 : 0);
            }
            tc::arrive_with_copies(&B->q_full);
            tc::close_copies();
        };
        if (hand->template next<S::SH>(P, S::ROWS, 0)) {
            bool more = true;
            int step = 0, in = 0;                                     // in: which of the segments in hand is gone through
            Source ahead = source(hand->seg[0], hand->seg[0].tile(0));
            while (more) {
                const Segment &now = hand->seg[in];
                const int at = step;
                const Source here = ahead;
                const bool last = ++step == now.steps();
                if (last) { more = hand->template next<S::SH>(P, S::ROWS, in ^= 1); step = 0; }
                if (more) ahead = source(hand->seg[in], hand->seg[in].tile(step));
                const uint32_t bad = __ballot_sync(0xffffffffu, here.seen && (here.id < 0 || here.id >= P.num_blocks));
                const bool by_map = P.box && here.whole && bad == 0;
                if (lane == 0) {
                    B->hidden[n_tile & 7][part] = bad;
                    ((volatile unsigned char *)&B->plain[n_tile & 7])[part] = !by_map;
                }
                ++n_tile;
                copy_rows(here, by_map, false);
                if (at == 0) copy_q(now);
                copy_rows(here, by_map, true);
            }
        }
        tc::wait_copies<0>();
        if (late_values) clean();
    }
    if (*(volatile int *)&B->dead) {
        // a wait ran out, and nobody waits any more: copies and products under way, which depend on nothing else, get a millisecond to end
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) __nanosleep(1000);
    }
    tc::fence_before();
    __syncthreads();
    if (warp == S::SOFT) {
        tc::fence_after();
        tc::tmem_free(tmem, 512);
        if (lane == 0) {
            P.late[c] = B->dead;
            // The first of a unit's parts tells what there is to join, unless the tree is bad: zeros for its rows come from the request's CTA of the
            // joining kernel, and nothing else of that kernel may write them.  (The unit is this run's last, so its tree is the one read last.)
            const Segment &seg = hand->seg[0];
            if (S::SH) return;
            int4 joint = make_int4(0, 0, 0, 0);
            if (hand->segments && seg.begin == 0 && !seg.whole && !B->bad_tree) {
                // (the unit's end, from what of it lies in this run)
                const int end = cuts.start(c + 1) + seg.t.count() - seg.end;
                int last = c + 1;
                while (cuts.start(last + 1) < end) ++last;
                joint = make_int4(seg.b, seg.m, seg.h, last + 1 - c | (seg.head ? 0 : 1 << 15) | seg.rows << 16);
            }
            P.joint[c] = joint;
        }
    }
}

// ---- joining ------------------------------------------------------------------------------------------------------------------
// The first P.ctas * groups CTAs: (CTA of the attention, JOIN_ROWS rows).  Where that one had the first of a unit's parts, they are put together, in
// order: out = sum 2^(ref_c - ref) O_c / sum 2^(ref_c - ref) l_c.  The others: a request each, its status (from inputs alone, while the
// attention still runs) and zeros for a bad tree.
constexpr int JOIN_NT = 128, JOIN_ROWS = 8;

template <typename T, typename S> __global__ void __launch_bounds__(JOIN_NT, 8) spec_join_kernel(const __grid_constant__ Params P)
{
    constexpr int D = S::D;
    const int tid = threadIdx.x, groups = P.groups;
    grid_launch_dependents();                  // (the next kernel waits for this one by itself, and this one for the attention)
    if ((int)blockIdx.x >= P.ctas * groups) {
        const int b = blockIdx.x - P.ctas * groups;
        const int len = __ldg(P.tree.lengths + b), nn = tree_nodes(P.tree, b), n = len < 0 ? 0 : max(nn, 0);
        const int *parent = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
        bool bad = false, page = false;
        for (int i = tid; i < n; i += JOIN_NT) {
            const int p = __ldg(parent + i);
            bad |= i == 0 ? p != -1 : p < 0 || p >= i;
        }
        // columns of the table that hold a key that some node sees
        const long long keys = n ? (long long)len + n : 0, since = P.window ? max(0ll, (long long)len - P.window + 1) : 0;
        const long long sinks = min((long long)P.sinks, (long long)len);
        const int cols = (int)min((keys + P.block - 1) / P.block, (long long)P.width);
        page = keys > (long long)P.width * P.block;
        for (int col = tid; col < cols; col += JOIN_NT) {
            const long long a = (long long)col * P.block, e = a + P.block;
            if (e > since || a < sinks) page |= block_in<false>(P, b, 0, col) < 0;
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
    const int j = blockIdx.x / groups, row0 = blockIdx.x % groups * JOIN_ROWS;
    grid_dependency_wait();
    const int4 joint = __ldcg(P.joint + j);
    const int b = joint.x, parts = joint.w & 0x7FFF, first = joint.w >> 15 & 1, rows = min((joint.w >> 16) - row0, JOIN_ROWS);
    if (parts == 0 || rows <= 0) return;
    const int last = j + parts - 1;
    // a thread per four entries of a row, eight parts' loads under way
    for (int i = tid; i < rows * (D / 4); i += JOIN_NT) {
        const int row = row0 + i % rows, ch = i / rows;
        float ref = -CUDART_INF_F, l = 0.f;
        bool only = false;                     // (some part saw keys, all with a score of -inf)
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c0 = j; c0 <= last; c0 += 8) {
            float4 x[8];
            float2 m[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = min(c0 + k, last), slot = 2 * c + (c == j ? first : 0);
                m[k] = __ldcg(&P.ml[slot * S::ROWS + row]);
                x[k] = __ldcg((const float4 *)P.part + (slot * (D / 4) + ch) * S::ROWS + row);
            }
            float top = ref;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                top = fmaxf(top, m[k].x);
                only |= m[k].x == -CUDART_INF_F && m[k].y != 0.f;
            }
            const float f = ref == -CUDART_INF_F ? 0.f : ex2_approx(ref - top);
            ref = top;
            l *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // (a part that saw nothing counts for nothing, whatever the others' reference)
                const float w = c0 + k > last || m[k].x == -CUDART_INF_F ? 0.f : ex2_approx(m[k].x - ref);
                if (w != 0.f) {
                    l = fmaf(w, m[k].y, l);
                    o.x = fmaf(w, x[k].x, o.x); o.y = fmaf(w, x[k].y, o.y); o.z = fmaf(w, x[k].z, o.z); o.w = fmaf(w, x[k].w, o.w);
                }
            }
        }
        const int q = joint.y * S::ROWS + row, node = node_of(P, q), head = joint.z * P.G + q - node * P.G;
        const float inv = l == 0.f ? only ? CUDART_NAN_F : 0.f : 1.f / l;
        T *to = (T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2] + ch * 4;
        *(uint2 *)to = make_uint2(Pair<T>::pack(o.x * inv, o.y * inv), Pair<T>::pack(o.z * inv, o.w * inv));
        if (P.lse && ch == 0) P.lse[((long long)b * P.tree.N + node) * P.Hq + head] = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
    }
}

}  // namespace attend
}  // namespace specv
