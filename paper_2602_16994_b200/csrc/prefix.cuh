// Attention over a paged cache for requests that share prefixes (spec_prefix_attention): what joins the parts.
//
// The kernel is the tree attention's, over more units: a group's prefix is seen by all rows of all of its members, so its units are (group, key head, up to
// 128 or 256 rows of member, node and query head), and its keys and values are read once for all of them instead of once a member.  The requests' own
// units begin behind their prefix.  All units' tiles are cut into one run per CTA, as there; every row of a member then has the parts of two
// units, each cut or not, and this kernel puts them together.
#pragma once
#include "attend.cuh"

namespace specv {
namespace attend {

constexpr int MERGE_NT = 256, MERGE_ROWS = 16;

// A CTA per request and MERGE_ROWS of its rows, in the order of key heads, then nodes, then heads of the group; a thread has four entries of a row.
template <typename T, typename S> __global__ void __launch_bounds__(MERGE_NT, 4) spec_prefix_join_kernel(const __grid_constant__ Params P)
{
    constexpr int D = S::D;
    const int tid = threadIdx.x, each = P.groups, b = blockIdx.x / (unsigned)each, row0 = (blockIdx.x - b * each) * MERGE_ROWS;
    grid_launch_dependents();                  // (the next kernel waits for this one by itself, and this one for the attention)
    // ---- what the inputs alone tell, while the attention still runs
    const int len = __ldg(P.tree.lengths + b), nn = tree_nodes(P.tree, b), n = len < 0 ? 0 : max(nn, 0);
    const int *parent = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
    bool bad = nn < 0, page = false;
    for (int i = tid; i < n; i += MERGE_NT) {
        const int p = __ldg(parent + i);
        bad |= i == 0 ? p != -1 : p < 0 || p >= i;
    }
    const int g_or_none = __ldg(P.group + b), g = g_or_none < 0 || g_or_none >= P.n_groups ? -1 : g_or_none;
    const int skip = g < 0 ? 0 : prefix_len(P, g);
    int2 m = make_int2(0, 0);
    int place = 0;
    bad |= g_or_none >= P.n_groups || !groups_in_order(P, tid, MERGE_NT);
    if (g >= 0) {
        const int blocks = __ldg(P.shared + g);
        m = members_of(P, g);
        place = __ldg(P.place + b);
        bad |= blocks < 0 || blocks > P.prefix_width || len < skip || place < 0 || place >= m.y - m.x || __ldg(P.members + m.x + place) != b;
    }
    bad = __syncthreads_or(len >= 0 && bad) != 0;
    if (row0 == 0) {
        const long long keys = n ? (long long)len + n : 0;
        const int cols = (int)min((keys + P.block - 1) / P.block, (long long)P.width);
        page = keys > (long long)P.width * P.block;
        for (int col = skip / P.block + tid; col < cols; col += MERGE_NT) page |= block_in<false>(P, b, 0, col) < 0;
        if (g >= 0 && n)
            for (int col = tid; col < skip / P.block; col += MERGE_NT) page |= block_in<true>(P, g, 0, col) < 0;
        page = __syncthreads_or(page) != 0;
    }
    grid_dependency_wait();
    if (row0 == 0) {
        bool late = false;
        for (int i = tid; i < P.ctas; i += MERGE_NT) late |= *(volatile int *)(P.late + i) != 0;
        late = __syncthreads_or(late) != 0;
        if (tid == 0)
            P.status[b] = len < 0 ? SPEC_DEV_OK : bad ? SPEC_DEV_TOPOLOGY : late ? SPEC_DEV_TIMEOUT : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
    }
    // ---- rows
    const int rows = P.tree.N * P.G;
    for (int i = tid; i < MERGE_ROWS * (D / 4); i += MERGE_NT) {
        const int at = row0 + i % MERGE_ROWS, ch = i / MERGE_ROWS;
        const int h = at / rows, r = at - h * rows, node = node_of(P, r), head = h * P.G + r - node * P.G;
        if (h >= P.Hkv || node >= n) continue;
        T *to = (T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2] + ch * 4;
        float *lse = P.lse && ch == 0 ? P.lse + ((long long)b * P.tree.N + node) * P.Hq + head : nullptr;
        if (bad) {
            *(uint2 *)to = make_uint2(0, 0);
            if (lse) *lse = -CUDART_INF_F;
            continue;
        }
        // the row's place in its unit, and the unit's parts: of the request's own, then of the prefix's
        int row[2], parts[2], first[2];
        long long whole[2];
        {
            const int e = P.n_groups + b, u = r / S::ROWS;
            const int2 x = __ldcg(&P.unit[0][unit_of(P, e, u, h, S::ROWS)]);
            first[0] = x.x; parts[0] = min(x.y, P.ctas); row[0] = r - u * S::ROWS;
            whole[0] = whole_row_of(P, e, h, r);
            if (x.x < 0 && skip == 0) continue;                     // (not cut, and nothing to put it together with: written already)
        }
        parts[1] = first[1] = row[1] = 0;
        whole[1] = 0;
        if (skip) {
            const int q = place * rows + r, u = q / S::ROWS;
            const int2 x = __ldcg(&P.unit[1][unit_of(P, g, u, h, S::ROWS)]);
            first[1] = x.x; parts[1] = min(x.y, P.ctas); row[1] = q - u * S::ROWS;
            whole[1] = whole_row_of(P, g, h, q);
        }
        const int all = parts[0] + parts[1];
        float ref = -CUDART_INF_F, l = 0.f;
        bool only = false;                     // (some part saw keys, all with a score of -inf)
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int AHEAD = 4;
        for (int c0 = 0; c0 < all; c0 += AHEAD) {
            float4 x[AHEAD];
            float2 y[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int c = min(c0 + k, all - 1), w = c >= parts[0], part = w ? c - parts[0] : c;
                if (first[w] < 0) {
                    y[k] = __ldcg(P.whole_ml[w] + whole[w]);
                    x[k] = __ldcg((const float4 *)P.whole[w] + ((whole[w] >> 5) * (D / 4) + ch) * 32 + (whole[w] & 31));
                } else {
                    // (its own slot for the first part, the first slot of the CTAs behind)
                    const long long slot = min(part ? (first[w] / 2 + part) * 2 : first[w], 2 * P.ctas - 1);
                    y[k] = __ldcg(P.ml + slot * S::ROWS + row[w]);
                    x[k] = __ldcg((const float4 *)P.part + (slot * (D / 4) + ch) * S::ROWS + row[w]);
                }
            }
            float top = ref;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                top = fmaxf(top, y[k].x);
                only |= y[k].x == -CUDART_INF_F && y[k].y != 0.f;
            }
            const float f = ref == -CUDART_INF_F ? 0.f : ex2_approx(ref - top);
            ref = top;
            l *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                // (a part that saw nothing counts for nothing, whatever the others' reference)
                const float w = c0 + k >= all || y[k].x == -CUDART_INF_F ? 0.f : ex2_approx(y[k].x - ref);
                if (w != 0.f) {
                    l = fmaf(w, y[k].y, l);
                    o.x = fmaf(w, x[k].x, o.x); o.y = fmaf(w, x[k].y, o.y); o.z = fmaf(w, x[k].z, o.z); o.w = fmaf(w, x[k].w, o.w);
                }
            }
        }
        const float inv = l == 0.f ? only ? CUDART_NAN_F : 0.f : 1.f / l;
        *(uint2 *)to = make_uint2(Pair<T>::pack(o.x * inv, o.y * inv), Pair<T>::pack(o.z * inv, o.w * inv));
        if (lse) *lse = l == 0.f ? -CUDART_INF_F : (ref + log2f(l)) * LN2;
    }
}

}  // namespace attend
}  // namespace specv
