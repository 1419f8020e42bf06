// Attention over a paged cache for requests that share prefixes (spec_prefix_attention): what joins the parts.
//
// The kernel is the tree attention's, over more units: a group's prefix is seen by all rows of all of its members, so its units are (group, key head, up to
// 128 or 256 rows of member, node and query head), and its keys and values are read once for all of them instead of once a member.  The requests' own
// units begin behind their prefix.  All units' tiles are cut into one run per CTA, as there; every row of a member then has the parts of two
// units, each cut or not, and this kernel puts them together.
//
// What bounds it.  Products where trees share (64 requests of 19 nodes, 32 heads to 8, one prefix of 8192 keys: 255 us in a short row of calls, 267 to 276 in a long one; floor of
// products 104, 25 are this kernel): tiles of 256 rows take 3700 to 4000 cycles, the tensor cores' share is 2760.  Bytes where tokens do (128 requests, 4 groups: 265 us in a short
// row, 278 to 291 in a long one, floor 170): a request's own unit of 4 rows costs two tiles' time beside its own 5 to 16.  Few requests: latency, as in the tree attention (4 tokens
// over 2048 shared keys 23 us: the parts that were timed, 5 until the first scores and 6 for the join, are not all of it).
//
// Precision.  As in the tree attention: P is rounded to the values' type.  Against 64 bits the error is 1.1 to 1.4 times that of weights kept in 32 bits and rounded once
// (bf16 0.0018 to 0.0016 and 0.0023 to 0.0017 of the result's norm, fp16 0.00029 to 0.00021); putting the parts together, in fp32, adds nothing that shows.
#pragma once
#include "attend.cuh"

namespace specv {
namespace attend {

constexpr int MERGE_NT = 128, MERGE_ROWS = 32;

// A CTA per request, key head and up to MERGE_ROWS rows of that head (in the order of nodes, then heads of the group); a thread has eight entries of a row.  Its
// rows belong to two units of the request's own and two of the prefix at most.  Where that makes few CTAs they have fewer rows, down to one for a thread: a row
// of a unit that is cut into many parts takes a load's latency for every three of them (3 requests of 18 nodes, D = 256: 89 us with 32 rows).
template <typename T, typename S> __global__ void __launch_bounds__(MERGE_NT, 8) spec_prefix_join_kernel(const __grid_constant__ Params P)
{
    constexpr int D = S::D;
    static_assert(MERGE_ROWS <= S::ROWS, "two units at most");
    __shared__ int2 s_unit[2][2];
    const int tid = threadIdx.x, rows = P.tree.N * P.G;
    const int b = (int)(blockIdx.x / (unsigned)P.groups), in = (int)blockIdx.x - b * P.groups, chunks = P.groups / P.Hkv;
    const int h = (int)((unsigned)in / (unsigned)chunks), row0 = (in - h * chunks) * P.merge_rows;
    grid_launch_dependents();                  // (the next kernel waits for this one by itself, and this one for the attention)
    // ---- what the inputs alone tell, while the attention still runs
    const int len = __ldg(P.tree.lengths + b), g_or_none = __ldg(P.group + b), place = P.n_groups ? __ldg(P.place + b) : 0, nn = tree_nodes(P.tree, b);
    const int n = len < 0 ? 0 : max(nn, 0);
    const int *parent = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
    bool bad = nn < 0 || g_or_none >= P.n_groups || !groups_in_order(P, tid, MERGE_NT);
    for (int i = tid; i < n; i += MERGE_NT) {
        const int p = __ldg(parent + i);
        bad |= i == 0 ? p != -1 : p < 0 || p >= i;
    }
    const int g = g_or_none < 0 || g_or_none >= P.n_groups ? -1 : g_or_none;
    int skip = 0;
    int2 m = make_int2(0, 0);
    if (g >= 0) {
        const int blocks = __ldg(P.shared + g);
        m = members_of(P, g);
        skip = prefix_len(P, g);
        bad |= blocks < 0 || blocks > P.prefix_width || len < skip || place < 0 || place >= m.y - m.x;
        if (!bad) bad = __ldg(P.members + m.x + place) != b;
    }
    bad = __syncthreads_or(len >= 0 && bad) != 0;
    bool page = false;
    if (in == 0) {
        const long long keys = n ? (long long)len + n : 0;
        const int cols = (int)min((keys + P.block - 1) / P.block, (long long)P.width);
        page = keys > (long long)P.width * P.block;
        for (int col = skip / P.block + tid; col < cols; col += MERGE_NT) page |= block_in<false>(P, b, 0, col) < 0;
        if (g >= 0 && n)
            for (int col = tid; col < skip / P.block; col += MERGE_NT) page |= block_in<true>(P, g, 0, col) < 0;
        page = __syncthreads_or(page) != 0;
    }
    const int upto = min(row0 + P.merge_rows, n * P.G), q0 = place * rows;          // rows of nodes that there are; the prefix's row of the request's row 0
    grid_dependency_wait();
    if (in == 0) {
        bool late = false;
        for (int i = tid; i < P.ctas; i += MERGE_NT) late |= *(volatile int *)(P.late + i) != 0;
        late = __syncthreads_or(late) != 0;
        if (tid == 0)
            P.status[b] = len < 0 ? SPEC_DEV_OK : bad ? SPEC_DEV_TOPOLOGY : late ? SPEC_DEV_TIMEOUT : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
    }
    if (row0 >= upto) return;
    if (bad) {
        for (int i = tid; i < (upto - row0) * (D / 8); i += MERGE_NT) {
            const int r = row0 + i / (D / 8), node = node_of(P, r), head = h * P.G + r - node * P.G;
            *(uint4 *)((T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2] + i % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
            if (P.lse && i % (D / 8) == 0) P.lse[((long long)b * P.tree.N + node) * P.Hq + head] = -CUDART_INF_F;
        }
        return;
    }
    const int first_unit[2] = {row0 / S::ROWS, (q0 + row0) / S::ROWS};
    if (tid < 4 && (tid < 2 || skip)) {
        const int w = tid >> 1, u = first_unit[w] + (tid & 1), last = ((w ? q0 : 0) + upto - 1) / S::ROWS;
        if (u <= last) s_unit[w][tid & 1] = __ldcg(&P.unit[w][unit_of(P, w ? g : P.n_groups + b, u, h, S::ROWS)]);
    }
    __syncthreads();
    const long long whole0 = whole_row_of(P, P.n_groups + b, h, 0), whole1 = skip ? whole_row_of(P, g, h, q0) : 0;
    const unsigned live = upto - row0;
#pragma unroll 1
    for (unsigned i = tid; i < live * (D / 8); i += MERGE_NT) {
        const int ch = (int)(i / live), r = row0 + (int)(i - ch * live);
        // the unit's parts: of the request's own, then of the prefix's
        const int u0 = r / S::ROWS, u1 = (q0 + r) / S::ROWS;
        const int2 own = s_unit[0][u0 - first_unit[0]], pre = skip ? s_unit[1][u1 - first_unit[1]] : make_int2(0, 0);
        if (own.x < 0 && skip == 0) continue;                       // (not cut, and nothing to put it together with: written already)
        const int mine = min(own.y, P.ctas), all = mine + min(pre.y, P.ctas);
        struct Eight { float4 a, b; };
        const auto fetch = [&](int c, float2 &y, Eight &x) {
            const bool w = c >= mine;
            const int from = w ? pre.x : own.x, part = w ? c - mine : c;
            const float4 *at;
            long long step;
            if (from < 0) {
                const long long row = (w ? whole1 : whole0) + r;
                y = __ldcg(P.whole_ml[w] + row);
                at = (const float4 *)P.whole[w] + ((row >> 5) * (D / 4) + 2 * ch) * 32 + (row & 31);
                step = 32;
            } else {
                // (its own slot for the first part, the first slot of the CTAs behind)
                const long long slot = min(part ? (from / 2 + part) * 2 : from, 2 * P.ctas - 1);
                const int row = w ? q0 + r - u1 * S::ROWS : r - u0 * S::ROWS;
                y = __ldcg(P.ml + slot * S::ROWS + row);
                at = (const float4 *)P.part + (slot * (D / 4) + 2 * ch) * S::ROWS + row;
                step = S::ROWS;
            }
            x.a = __ldcg(at);
            x.b = __ldcg(at + step);
        };
        float ref = -CUDART_INF_F, l = 0.f;
        bool only = false;                     // (some part saw keys, all with a score of -inf)
        float o[8] = {};
        constexpr int AHEAD = 3;
#pragma unroll 1
        for (int c0 = 0; c0 < all; c0 += AHEAD) {
            Eight x[AHEAD];
            float2 y[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                y[k] = make_float2(-CUDART_INF_F, 0.f);
                if (c0 + k < all) fetch(c0 + k, y[k], x[k]);
            }
            float top = ref;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                top = fmaxf(top, y[k].x);
                only |= y[k].x == -CUDART_INF_F && y[k].y != 0.f;
            }
            const float f = ref == -CUDART_INF_F ? 0.f : ex2_approx(ref - top);
            ref = top;
            l *= f;
#pragma unroll
            for (int d = 0; d < 8; ++d) o[d] *= f;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                // (a part that saw nothing counts for nothing, whatever the others' reference)
                const float w = y[k].x == -CUDART_INF_F ? 0.f : ex2_approx(y[k].x - ref);
                if (w != 0.f) {
                    l = fmaf(w, y[k].y, l);
                    o[0] = fmaf(w, x[k].a.x, o[0]); o[1] = fmaf(w, x[k].a.y, o[1]); o[2] = fmaf(w, x[k].a.z, o[2]); o[3] = fmaf(w, x[k].a.w, o[3]);
                    o[4] = fmaf(w, x[k].b.x, o[4]); o[5] = fmaf(w, x[k].b.y, o[5]); o[6] = fmaf(w, x[k].b.z, o[6]); o[7] = fmaf(w, x[k].b.w, o[7]);
                }
            }
        }
        const int node = node_of(P, r), head = h * P.G + r - node * P.G;
        T *to = (T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2] + ch * 8;
        const float inv = l == 0.f ? only ? CUDART_NAN_F : 0.f : 1.f / l;
        *(uint4 *)to = make_uint4(Pair<T>::pack(o[0] * inv, o[1] * inv), Pair<T>::pack(o[2] * inv, o[3] * inv), Pair<T>::pack(o[4] * inv, o[5] * inv),
                                  Pair<T>::pack(o[6] * inv, o[7] * inv));
        if (P.lse && ch == 0) P.lse[((long long)b * P.tree.N + node) * P.Hq + head] = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
    }
}

}  // namespace attend
}  // namespace specv
