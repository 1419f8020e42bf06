// libspecverify: attention for requests that share prefixes -- host side of its C ABI.
//
// Kernels: attend.cuh (the attention of a tree's nodes, over the units of prefixes and requests), prefix.cuh (what joins their parts).  As in
// specverify.cu, this file validates arguments, chooses the launch shape and enqueues; it never allocates and never synchronises.
#include <cmath>

#include "launch.h"
#include "prefix.cuh"

namespace specv {

int set_prefix_hooks(long long cycles, int hold)
{
    if (cudaMemcpyToSymbol(c_wait_cycles, &cycles, sizeof(cycles)) != cudaSuccess ||
        cudaMemcpyToSymbol(c_hold_slot, &hold, sizeof(hold)) != cudaSuccess) {
        cudaGetLastError();
        return SPEC_ERR_CUDA;
    }
    return SPEC_OK;
}

}  // namespace specv

using namespace specv;

// Two blocks of 128 rows share the loads of a tile where a prefix has, on average, more rows than one block, or a request has.  Long rows of calls, us with one and two
// blocks, 32 heads to 8 (D = 128): tokens of 2 groups over 16384 shared keys, up to 512 behind them, 128 rows a prefix 90 and 95, 160 rows 134 and 112, 256 rows 161
// and 148; 8 groups of two trees of 19 nodes over 8192 (152 rows) 154 and 102, of three (228) 164 and 112.  Where what lies behind the prefix is most of the work the
// second block costs more than it saves, since requests have few rows: 33 tokens, 8192 shared and up to 4096 behind 106 and 113, 160 tokens in 4 groups, 4096 and 4096,
// 424 and 458; lengths are not known here.  The rows are those of the members that the plan lists; a plan that lists requests without a group too is taken for one
// of longer prefixes (128 tokens, two of which share 8192 keys: 253, 243 with the two alone).
static bool two_blocks(const SpecPrefixAttention *p)
{
    const SpecAttention &a = p->attention;
    const int64_t rows = (int64_t)a.N * (a.Hq / a.Hkv);
    return a.D <= 128 && (rows > 128 || (p->n_groups > 0 && (int64_t)p->n_members * rows > (int64_t)p->n_groups * 128));
}
static int prefix_check(const SpecPrefixAttention *p)
{
    if (!p) return SPEC_ERR_NULL;
    const SpecAttention &a = p->attention;
    if (!a.q || !a.k_cache || !a.v_cache || !a.block_table || !a.lengths || !a.parent || !a.out || !a.status || !p->group ||
        (p->n_groups > 0 && (!p->members || !p->first || !p->place || !p->shared_blocks || !p->prefix_table)))
        return SPEC_ERR_NULL;
    if (bad_tree_shape(a.B, a.N, a.topo_seq_stride) || bad_pages(a.num_blocks, a.block_size, a.table_width) || a.table_stride < a.table_width ||
        a.Hkv < 1 || a.Hq < a.Hkv || a.Hq % a.Hkv || a.Hq > 65535 || p->n_groups < 0 || p->n_groups > 65535 || p->n_members < 0 ||
        p->n_members > a.B || (p->n_groups > 0 && (p->prefix_width < 1 || p->prefix_stride < p->prefix_width || p->n_members < 1)))
        return SPEC_ERR_SHAPE;
    if (a.dtype != SPEC_BF16 && a.dtype != SPEC_F16) return SPEC_ERR_DTYPE;
    if (!(a.scale >= 0.f && a.scale <= 3.4e38f) || a.window != 0 || a.sinks != 0) return SPEC_ERR_PARAM;
    if (a.D != 64 && a.D != 128 && a.D != 256) return SPEC_ERR_UNSUPPORTED;
    // (tiles and rows are counted in 32 bits)
    const double rows = (double)a.N * (a.Hq / a.Hkv), block = two_blocks(p) ? 256 : 128;
    const double keys = (double)std::min<int64_t>((int64_t)a.table_width * a.block_size, 0x7FFFFFFF) + a.N;
    const double prefix = (double)std::min<int64_t>((int64_t)p->prefix_width * a.block_size, 0x7FFFFFFF);
    const double tiles = a.B * (double)a.Hkv * std::ceil(rows / block) * (keys / attend::KT + 1 + attend::START) +
                         (p->n_groups ? a.Hkv * (p->n_members * rows / block + p->n_groups) * (prefix / attend::KT + 1 + attend::START) : 0.0);
    if (tiles > 2.0e9 || a.B * rows > 1.0e9 || a.B * (double)a.Hkv * std::ceil(rows / attend::MERGE_ROWS) > 2.0e9) return SPEC_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int j = 0; j < 3; ++j) all |= a.q_stride[j] | a.k_cache_stride[j] | a.v_cache_stride[j] | a.out_stride[j];
    if (all % 8 || !aligned(a.q, 16) || !aligned(a.k_cache, 16) || !aligned(a.v_cache, 16) || !aligned(a.out, 16)) return SPEC_ERR_UNSUPPORTED;
    return SPEC_OK;
}

struct PrefixLayout { int64_t part, ml, whole[2], whole_ml[2], unit[2], late, total; };
static PrefixLayout prefix_layout(const SpecPrefixAttention *p, int ctas)
{
    const SpecAttention &a = p->attention;
    const int64_t block = two_blocks(p) ? 256 : 128, rows = (int64_t)a.N * (a.Hq / a.Hkv);
    PrefixLayout L = {};
    const auto take = [&](int64_t bytes) { const int64_t at = L.total; L.total += (bytes + 255) / 256 * 256; return at; };
    L.part = take((int64_t)ctas * 2 * block * a.D * 4);
    L.ml = take((int64_t)ctas * 2 * block * 8);
    const int64_t many[2] = {p->n_groups ? (int64_t)a.B : 0, p->n_groups ? (int64_t)p->n_members : 0};
    for (int i = 0; i < 2; ++i) {
        const int64_t all = (many[i] * a.Hkv * rows + 31) / 32 * 32;
        L.whole[i] = take(all * a.D * 4);
        L.whole_ml[i] = take(all * 8);
    }
    L.unit[0] = take((int64_t)a.B * ((rows + block - 1) / block) * a.Hkv * 8);
    L.unit[1] = take(((int64_t)p->n_members * rows / block + p->n_groups + 2) * a.Hkv * 8);
    L.late = take((int64_t)ctas * 4);
    return L;
}

extern "C" {

int32_t spec_prefix_attention_workspace_bytes(const SpecPrefixAttention *p, int64_t *bytes)
{
    if (!bytes) return SPEC_ERR_NULL;
    const int rc = prefix_check(p);
    if (rc) return rc;
    *bytes = prefix_layout(p, sm_ctas()).total;
    return SPEC_OK;
}

int32_t spec_prefix_attention(const SpecPrefixAttention *given, void *ws, int64_t ws_bytes, void *stream)
{
    const int rc = prefix_check(given);
    if (rc) return rc;
    const SpecAttention *a = &given->attention;
    const int ctas = sm_ctas();
    const PrefixLayout L = prefix_layout(given, ctas);
    if (!ws || !aligned(ws, 256) || ws_bytes < L.total) return SPEC_ERR_WORKSPACE;
    const bool two = two_blocks(given);
    attend::Params p = {};
    p.tree = tree_args(a->N, a->lengths, a->n_nodes, a->parent, a->topo_seq_stride);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = a->Hq / a->Hkv;
    p.num_blocks = a->num_blocks; p.block = a->block_size; p.width = a->table_width;
    divisor(a->block_size, &p.block_mul, &p.block_shift);
    divisor(p.G, &p.group_mul, &p.group_shift);
    divisor(a->N, &p.nodes_mul, &p.nodes_shift);
    p.scale = std::max(a->scale, 1.17549435e-38f);      // (so that what is not seen, -inf, stays that under a scale of 0)
    p.q = a->q; p.k = a->k_cache; p.v = a->v_cache; p.table = a->block_table; p.table_stride = a->table_stride;
    p.out = a->out; p.lse = a->lse; p.status = a->status;
    for (int j = 0; j < 3; ++j) {
        p.q_stride[j] = a->q_stride[j]; p.k_stride[j] = a->k_cache_stride[j]; p.v_stride[j] = a->v_cache_stride[j];
        p.out_stride[j] = a->out_stride[j];
    }
    p.n_groups = given->n_groups; p.n_members = given->n_members; p.prefix_width = given->prefix_width; p.prefix_stride = given->prefix_stride;
    p.group = given->group; p.members = given->members; p.first = given->first; p.place = given->place; p.shared = given->shared_blocks;
    p.prefix_table = given->prefix_table;
    p.ctas = ctas;
    unsigned char *base = (unsigned char *)ws;
    p.part = (float *)(base + L.part);
    p.ml = (float2 *)(base + L.ml);
    for (int i = 0; i < 2; ++i) {
        p.whole[i] = (float *)(base + L.whole[i]);
        p.whole_ml[i] = (float2 *)(base + L.whole_ml[i]);
        p.unit[i] = (int2 *)(base + L.unit[i]);
    }
    p.late = (int *)(base + L.late);
    const int64_t rows = (int64_t)a->N * p.G;
    p.unit_blocks = (int)((rows + (two ? 255 : 127)) / (two ? 256 : 128));
    p.merge_rows = attend::MERGE_ROWS;
    const auto merging = [&] { return (rows + p.merge_rows - 1) / p.merge_rows * a->Hkv; };         // CTAs of a request in the joining kernel
    while (p.merge_rows * (a->D / 8) > attend::MERGE_NT && merging() * a->B < ctas * 4) p.merge_rows /= 2;
    p.groups = (int)merging();
    const bool half = a->dtype == SPEC_F16;
    // (boxes: 254 us for 64 requests of 19 nodes; by 16-byte copies 270)
    p.box = a->block_size % 8 ? 0 : a->block_size % 16 ? 8 : a->block_size % 32 ? 16 : 32;
    const int64_t sizes[4] = {a->D, a->Hkv, a->block_size, a->num_blocks};
    const auto cache_map = [&](CUtensorMap *map, const void *cache, const int64_t *s) {
        return tensor_map(map, cache, half, sizes, {s[2], s[1], s[0]}, {1, p.box, 1});
    };
    if (p.box && !(cache_map(&p.k_map, a->k_cache, a->k_cache_stride) && cache_map(&p.v_map, a->v_cache, a->v_cache_stride))) p.box = 0;
    const cudaStream_t st = (cudaStream_t)stream;
    const auto go = [&](auto shape, auto attend_kernel, auto join_kernel) -> int {
        using S = decltype(shape);
        const int smem = S::total + 1024;
        int e = prepare(attend_kernel, smem, false);
        if (!e) e = prepare(join_kernel, 0, false);
        if (e) return e;
        e = launch(attend_kernel, dim3(ctas), S::NT, smem, 0, st, p);
        return e ? e : launch(join_kernel, dim3((unsigned)(p.groups * a->B)), attend::MERGE_NT, 0, 0, st, p);
    };
#define GO(D, MT, WG)                                                                                                                          \
    (half ? go(attend::Shape<D, MT, WG, true>(), attend::spec_attend_kernel<__half, attend::Shape<D, MT, WG, true>>,                          \
               attend::spec_prefix_join_kernel<__half, attend::Shape<D, MT, WG, true>>)                                                       \
          : go(attend::Shape<D, MT, WG, true>(), attend::spec_attend_kernel<__nv_bfloat16, attend::Shape<D, MT, WG, true>>,                   \
               attend::spec_prefix_join_kernel<__nv_bfloat16, attend::Shape<D, MT, WG, true>>))
    if (a->D == 256) return GO(256, 1, 1);
    if (a->D == 128) return two ? GO(128, 2, 2) : GO(128, 1, 2);
    return two ? GO(64, 2, 2) : GO(64, 1, 2);
#undef GO
}

}  // extern "C"
