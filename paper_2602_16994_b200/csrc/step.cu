// libspecverify: the operators around a verification in a decoding loop -- host side of their C ABI.
//
// Kernels: slots.cuh (blocks, slots and positions of a step), rope.cuh (norm and rotation per head, keys and values into the
// cache), attend.cuh (attention of a tree's nodes over the paged cache), chain.cuh (verification from
// probabilities), commit.cuh (the accepted path moves in the cache).  As in specverify.cu, this file validates arguments,
// chooses the launch shape and enqueues; it never allocates and never synchronises.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attend.cuh"
#include "chain.cuh"
#include "commit.cuh"
#include "common.cuh"
#include "host.h"
#include "launch.h"
#include "rope.cuh"
#include "slots.cuh"
#include "specverify.h"

namespace specv {

int set_step_hooks(long long cycles, int hold)
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

extern "C" {

int32_t spec_cache_slots(const SpecSlots *a, void *stream)
{
    if (!a || !a->lengths || !a->parent || !a->block_table || !a->owned || !a->free_range || !a->slots || !a->positions || !a->owned_out ||
        !a->free_range_out || !a->status || (a->free_size > 0 && !a->free_blocks))
        return SPEC_ERR_NULL;
    if (bad_tree_shape(a->B, a->N, a->topo_seq_stride) || a->block_size < 1 || a->table_width < 1 || a->table_stride < a->table_width ||
        a->free_size < 0)
        return SPEC_ERR_SHAPE;
    if (a->owned_out == a->owned || a->owned_out == a->lengths || a->free_range_out == a->free_range) return SPEC_ERR_PARAM;
    slots::Params p = {};
    p.tree = tree_args(a->N, a->lengths, a->n_nodes, a->parent, a->topo_seq_stride);
    p.B = a->B; p.block = a->block_size; p.width = a->table_width; p.free_size = a->free_size;
    p.table = a->block_table; p.table_stride = a->table_stride;
    p.owned = a->owned; p.ring = a->free_blocks; p.range = a->free_range;
    p.slots = a->slots; p.positions = a->positions; p.owned_out = a->owned_out; p.range_out = a->free_range_out; p.status = a->status;
    const int rc = prepare(slots::spec_slots_kernel, 0, false);
    return rc ? rc : launch(slots::spec_slots_kernel, dim3((a->B + slots::WARPS - 1) / slots::WARPS + 1), slots::NT, slots::WARPS * a->N * 4, 0,
                  (cudaStream_t)stream, p);
}

int32_t spec_norm_rope_cache(const SpecNormRope *a, void *stream)
{
    if (!a || !a->q || !a->k || !a->v || (a->rot > 0 && !a->inv_freq) || !a->positions || !a->slots || !a->q_out || !a->k_cache || !a->v_cache)
        return SPEC_ERR_NULL;
    // (a CTA's step from token to token stays below 2^31)
    if (a->T < 1 || a->T > 0x7FFFFFFF - 4096 || a->Hq < 1 || a->Hkv < 1 || a->Hq > 65535 || a->Hkv > 65535 || a->num_blocks < 1 || a->block_size < 1 ||
        (int64_t)a->num_blocks * a->block_size > 0x7FFFFFFF)
        return SPEC_ERR_SHAPE;
    if (a->dtype != SPEC_F32 && a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_DTYPE;
    if ((a->pairs != 0 && a->pairs != 1) || !(a->eps >= 0.f) || a->rot < 0) return SPEC_ERR_PARAM;
    if (a->D < 8 || a->D > 256 || a->D % 8 || a->rot > a->D || a->rot % 16) return SPEC_ERR_UNSUPPORTED;
    rope::Params p = {};
    p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.D = a->D; p.rot = a->rot; p.pairs = a->pairs;
    divisor(a->block_size, &p.block_mul, &p.block_shift);
    p.block = a->block_size; p.n_slots = (long long)a->num_blocks * a->block_size;
    p.x[0] = a->q; p.x[1] = a->k; p.x[2] = a->v;
    const int64_t *in[3] = {a->q_stride, a->k_stride, a->v_stride};
    const int64_t esz = a->dtype == SPEC_F32 ? 4 : 2;
    int64_t all = (int64_t)(uintptr_t)a->q | (int64_t)(uintptr_t)a->k | (int64_t)(uintptr_t)a->v | (int64_t)(uintptr_t)a->q_out |
                  (int64_t)(uintptr_t)a->k_cache | (int64_t)(uintptr_t)a->v_cache | (int64_t)(uintptr_t)a->q_weight |
                  (int64_t)(uintptr_t)a->k_weight;
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 2; ++j) { p.x_stride[i][j] = in[i][j]; all |= in[i][j] * esz; }
    p.weight[0] = a->q_weight; p.weight[1] = a->k_weight; p.eps = a->eps; p.inv_D = 1.f / (float)a->D;
    p.inv_freq = a->inv_freq; p.positions = a->positions; p.slots = a->slots;
    p.q_out = a->q_out; p.cache[0] = a->k_cache; p.cache[1] = a->v_cache;
    for (int j = 0; j < 2; ++j) { p.q_out_stride[j] = a->q_out_stride[j]; all |= a->q_out_stride[j] * esz; }
    for (int j = 0; j < 3; ++j) {
        p.cache_stride[0][j] = a->k_cache_stride[j]; p.cache_stride[1][j] = a->v_cache_stride[j];
        all |= (a->k_cache_stride[j] | a->v_cache_stride[j]) * esz;
    }
    const bool vec = (all & 15) == 0;
    // sixteen entries to a thread where rows and rotated parts are made of such and lie on 16 bytes: fewer addresses and steps of the norm's sum than
    // with eight (6528 tokens of 48 heads of 128 entries: 39.4 us, with eight 40.6)
    const bool wide = vec && a->D % 16 == 0 && a->rot % 32 == 0;
    while (((wide ? 16 : 8) << p.lane_shift) < a->D) ++p.lane_shift;
    const auto go = [&](auto kernel, int most) {
        const int rc = prepare(kernel, 0, false);
        // as many CTAs as have room, each with as many tokens as the others
        const int each = (a->T + most - 1) / most;
        return rc ? rc : launch(kernel, dim3((a->T + each - 1) / each), rope::NT, 0, 0, (cudaStream_t)stream, p);
    };
#define GO(T)                                                                  \
    (wide  ? go(rope::spec_rope_kernel<T, true, 16>, 148 * rope::CTAS<16>)        \
     : vec ? go(rope::spec_rope_kernel<T, true, 8>, 148 * rope::CTAS<8>)          \
           : go(rope::spec_rope_kernel<T, false, 8>, 148 * rope::CTAS<8>))
    return a->dtype == SPEC_F32 ? GO(float) : a->dtype == SPEC_F16 ? GO(__half) : GO(__nv_bfloat16);
#undef GO
}

static int attention_check(const SpecAttention *a)
{
    if (!a || !a->q || !a->k_cache || !a->v_cache || !a->block_table || !a->lengths || !a->parent || !a->out || !a->status)
        return SPEC_ERR_NULL;
    if (bad_tree_shape(a->B, a->N, a->topo_seq_stride) || bad_pages(a->num_blocks, a->block_size, a->table_width) ||
        a->table_stride < a->table_width || a->Hkv < 1 || a->Hq < a->Hkv || a->Hq % a->Hkv || a->Hq > 65535)
        return SPEC_ERR_SHAPE;
    if (a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_DTYPE;
    if (!(a->scale >= 0.f && a->scale <= 3.4e38f) || a->window < 0 || a->sinks < 0) return SPEC_ERR_PARAM;
    if (a->D != 64 && a->D != 128 && a->D != 256) return SPEC_ERR_UNSUPPORTED;
    // (tiles are counted in 32 bits)
    const int64_t blocks = ((int64_t)a->N * (a->Hq / a->Hkv) + 127) / 128;
    const int64_t keys = std::min<int64_t>((int64_t)a->table_width * a->block_size, 0x7FFFFFFF) + a->N;
    if ((double)a->B * a->Hkv * (double)blocks * (double)(keys / attend::KT + 1 + attend::START) > 2.0e9) return SPEC_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int j = 0; j < 3; ++j) all |= a->q_stride[j] | a->k_cache_stride[j] | a->v_cache_stride[j] | a->out_stride[j];
    if (all % 8 || !aligned(a->q, 16) || !aligned(a->k_cache, 16) || !aligned(a->v_cache, 16) || !aligned(a->out, 16))
        return SPEC_ERR_UNSUPPORTED;
    return SPEC_OK;
}

// Two blocks of 128 rows share the loads of a tile where a request has more rows than one block.
static bool two_blocks(const SpecAttention *a) { return a->D <= 128 && (int64_t)a->N * (a->Hq / a->Hkv) > 128; }

struct AttentionLayout { int64_t part, ml, joint, late, total; };
static AttentionLayout attention_layout(const SpecAttention *a, int ctas)
{
    const int64_t rows = two_blocks(a) ? 256 : 128;
    AttentionLayout L = {};
    L.ml = (int64_t)ctas * 2 * rows * a->D * 4;
    L.joint = L.ml + (int64_t)ctas * 2 * rows * 8;
    L.late = L.joint + (int64_t)ctas * 16;
    L.total = L.late + ((int64_t)ctas * 4 + 255) / 256 * 256;
    return L;
}

int32_t spec_tree_attention_workspace_bytes(const SpecAttention *a, int64_t *bytes)
{
    if (!bytes) return SPEC_ERR_NULL;
    const int rc = attention_check(a);
    if (rc) return rc;
    *bytes = attention_layout(a, sm_ctas()).total;
    return SPEC_OK;
}

int32_t spec_tree_attention(const SpecAttention *a, void *ws, int64_t ws_bytes, void *stream)
{
    const int rc = attention_check(a);
    if (rc) return rc;
    const int ctas = sm_ctas();
    const AttentionLayout L = attention_layout(a, ctas);
    if (!ws || !aligned(ws, 256) || ws_bytes < L.total) return SPEC_ERR_WORKSPACE;
    attend::Params p = {};
    p.tree = tree_args(a->N, a->lengths, a->n_nodes, a->parent, a->topo_seq_stride);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = a->Hq / a->Hkv;
    p.num_blocks = a->num_blocks; p.block = a->block_size; p.width = a->table_width;
    divisor(a->block_size, &p.block_mul, &p.block_shift);
    divisor(p.G, &p.group_mul, &p.group_shift);
    p.window = a->window; p.sinks = a->sinks;
    p.scale = std::max(a->scale, 1.17549435e-38f);      // (so that what is not seen, -inf, stays that under a scale of 0)
    p.q = a->q; p.k = a->k_cache; p.v = a->v_cache; p.table = a->block_table; p.table_stride = a->table_stride;
    p.out = a->out; p.lse = a->lse; p.status = a->status;
    for (int j = 0; j < 3; ++j) {
        p.q_stride[j] = a->q_stride[j]; p.k_stride[j] = a->k_cache_stride[j]; p.v_stride[j] = a->v_cache_stride[j];
        p.out_stride[j] = a->out_stride[j];
    }
    p.ctas = ctas;
    p.part = (float *)((unsigned char *)ws + L.part);
    p.ml = (float2 *)((unsigned char *)ws + L.ml);
    p.joint = (int4 *)((unsigned char *)ws + L.joint);
    p.late = (int *)((unsigned char *)ws + L.late);
    const bool half = a->dtype == SPEC_F16;
    p.box = a->block_size % 8 ? 0 : a->block_size % 16 ? 8 : a->block_size % 32 ? 16 : 32;
    const int64_t sizes[4] = {a->D, a->Hkv, a->block_size, a->num_blocks}, q_sizes[4] = {a->D, a->Hq, a->N, a->B};
    const auto cache_map = [&](CUtensorMap *map, const void *cache, const int64_t *s) {
        return tensor_map(map, cache, half, sizes, {s[2], s[1], s[0]}, {1, p.box, 1});
    };
    if (p.box && !(cache_map(&p.k_map, a->k_cache, a->k_cache_stride) && cache_map(&p.v_map, a->v_cache, a->v_cache_stride))) p.box = 0;
    p.q_boxes = 128 % p.G == 0 && tensor_map(&p.q_map, a->q, half, q_sizes, {a->q_stride[2], a->q_stride[1], a->q_stride[0]}, {p.G, 128 / p.G, 1});
    const cudaStream_t st = (cudaStream_t)stream;
    const auto go = [&](auto shape, auto attend_kernel, auto join_kernel) -> int {
        using S = decltype(shape);
        const int smem = S::total + 1024;
        p.groups = ((int)std::min<int64_t>(S::ROWS, (int64_t)p.tree.N * p.G) + attend::JOIN_ROWS - 1) / attend::JOIN_ROWS;
        int e = prepare(attend_kernel, smem, false);
        if (!e) e = prepare(join_kernel, 0, false);
        if (e) return e;
        e = launch(attend_kernel, dim3(ctas), S::NT, smem, 0, st, p);
        return e ? e : launch(join_kernel, dim3((unsigned)(ctas * p.groups + a->B)), attend::JOIN_NT, 0, 0, st, p);
    };
#define GO(D, MT, WG)                                                                                                                      \
    (half ? go(attend::Shape<D, MT, WG>(), attend::spec_attend_kernel<__half, attend::Shape<D, MT, WG>>,                                  \
               attend::spec_join_kernel<__half, attend::Shape<D, MT, WG>>)                                                                \
          : go(attend::Shape<D, MT, WG>(), attend::spec_attend_kernel<__nv_bfloat16, attend::Shape<D, MT, WG>>,                           \
               attend::spec_join_kernel<__nv_bfloat16, attend::Shape<D, MT, WG>>))
    if (a->D == 256) return GO(256, 1, 1);
    if (a->D == 128) return two_blocks(a) ? GO(128, 2, 2) : GO(128, 1, 2);
    return two_blocks(a) ? GO(64, 2, 2) : GO(64, 1, 2);
#undef GO
}

int32_t spec_cache_commit(const SpecCommit *a, void *stream)
{
    if (!a || !a->cache || !a->block_table || !a->lengths || !a->parent || !a->accepted_node || !a->lengths_out || !a->status)
        return SPEC_ERR_NULL;
    if (bad_tree_shape(a->B, a->N, a->topo_seq_stride) || bad_pages(a->num_blocks, a->block_size, a->table_width) ||
        a->table_stride < a->table_width || a->caches < 1 || a->row_bytes < 1 || a->row_bytes > 0x7FFFFFFF)
        return SPEC_ERR_SHAPE;
    if (a->lengths_out == a->lengths || a->lengths_out == a->accepted_node) return SPEC_ERR_PARAM;
    commit::Params p = {};
    p.tree = tree_args(a->N, a->lengths, a->n_nodes, a->parent, a->topo_seq_stride);
    p.B = a->B; p.caches = a->caches; p.num_blocks = a->num_blocks; p.block = a->block_size; p.width = a->table_width;
    p.cache = (unsigned char *)a->cache;
    int64_t all = (int64_t)(uintptr_t)a->cache | a->row_bytes;
    for (int j = 0; j < 3; ++j) { p.stride[j] = a->stride[j]; all |= a->stride[j]; }
    p.table = a->block_table; p.table_stride = a->table_stride; p.accepted = a->accepted_node;
    p.lengths_out = a->lengths_out; p.status = a->status;
    const int unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
    p.words = (unsigned)(a->row_bytes / unit);
    p.per = std::max(1, commit::NT / (int)p.words);
    const dim3 grid((a->caches + p.per - 1) / p.per, a->B);
    const auto go = [&](auto kernel) {
        const int rc = prepare(kernel, 0, false);
        return rc ? rc : launch(kernel, grid, commit::NT, 0, 0, (cudaStream_t)stream, p);
    };
    return unit == 16  ? go(commit::spec_commit_kernel<uint4>)
           : unit == 4 ? go(commit::spec_commit_kernel<uint32_t>)
                       : go(commit::spec_commit_kernel<unsigned char>);
}

int32_t spec_verify_probs(const SpecChains *a, void *stream)
{
    if (!a || !a->target_probs || !a->cu_drafts || !a->u_bonus || !a->accept_len || !a->out_tokens || !a->bonus_token || !a->status ||
        (a->n_drafts > 0 && (!a->token || !a->u_accept)))
        return SPEC_ERR_NULL;
    if (a->B < 1 || a->B > (1 << 26) || a->V < 1 || a->max_drafts < 0 || a->max_drafts > (1 << 20) || a->n_drafts < 0 || a->target_stride < a->V ||
        (a->draft_probs && a->draft_stride < a->V))
        return SPEC_ERR_SHAPE;
    if (a->dtype != SPEC_F32 && a->dtype != SPEC_BF16) return SPEC_ERR_DTYPE;
    // the largest cluster whose slices are worth a CTA and that leaves one wave of four CTAs per SM (128 requests of 151936 entries: 37 us with
    // eight CTAs each, in two waves)
    int C = 1;
    while (C < chain::CMAX && a->V / (2 * C) >= 4096 && (int64_t)a->B * 2 * C <= 148 * 4) C *= 2;
    while (C < chain::CMAX && (int64_t)a->V > (int64_t)C * chain::TILES * chain::TILE) C *= 2;
    if ((int64_t)a->V > (int64_t)C * chain::TILES * chain::TILE) return SPEC_ERR_UNSUPPORTED;
    chain::Params p = {};
    p.B = a->B; p.V = a->V; p.most = a->max_drafts; p.n_drafts = a->n_drafts;
    p.SL = ((a->V + C - 1) / C + chain::TILE - 1) / chain::TILE * chain::TILE;
    p.p = a->target_probs; p.q = a->n_drafts ? a->draft_probs : nullptr; p.p_stride = a->target_stride; p.q_stride = a->draft_stride;
    p.token = a->token; p.cu = a->cu_drafts; p.u_accept = a->u_accept; p.u_bonus = a->u_bonus;
    p.accept_len = a->accept_len; p.out_tokens = a->out_tokens; p.bonus = a->bonus_token; p.status = a->status;
    const auto go = [&](auto kernel) {
        const int rc = prepare(kernel, 0, true);
        return rc ? rc : launch(kernel, dim3((unsigned)(a->B * C)), chain::NT, 0, C, (cudaStream_t)stream, p);
    };
    return a->dtype == SPEC_F32 ? go(chain::spec_chain_kernel<float>) : go(chain::spec_chain_kernel<unsigned short>);
}

}  // extern "C"
