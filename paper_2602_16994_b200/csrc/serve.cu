// libspecverify: bounded caches and what a service answers with -- host side of their C ABI.
//
// Kernels: logprobs.cuh (log probabilities, entropy, most probable tokens), weigh.cuh (attention weight that
// entries of a cache get), evict.cuh (entries of a cache that are kept).
// As in specverify.cu, this file validates arguments, chooses the launch shape and enqueues; it never allocates and never synchronises.
#include "evict.cuh"
#include "launch.h"
#include "logprobs.cuh"
#include "weigh.cuh"

namespace specv {

int set_serve_hooks(long long cycles, int hold)
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

int32_t spec_token_logprobs(const SpecLogprobs *a, void *stream)
{
    if (!a || !a->logits || !a->entropy || !a->status || (a->K > 0 && (!a->token || !a->logprob)) ||
        (a->top > 0 && (!a->top_tokens || !a->top_logprobs)) || (a->parent && !a->accepted_node))
        return SPEC_ERR_NULL;
    if (a->B < 1 || a->N < 1 || a->V < 1 || a->K < 0 || a->seq_stride < 0 || a->node_stride < 0 || (int64_t)a->B * a->N > (1 << 26) ||
        (a->parent && (a->K > 1 || a->N > SPEC_MAX_NODES)) || (a->topo_seq_stride != 0 && a->topo_seq_stride < a->N))
        return SPEC_ERR_SHAPE;
    if (a->dtype != SPEC_F32 && a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_DTYPE;
    if (!(a->temperature >= 1e-30f && a->temperature <= 1e30f) || a->top < 0 || a->top > SPEC_MAX_TOP || a->top > a->V) return SPEC_ERR_PARAM;
    if (!aligned(a->logits, a->dtype == SPEC_F32 ? 4 : 2)) return SPEC_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)a->B * a->N;
    // The largest cluster that leaves every CTA two batches of loads (none for a row of four batches, whose last exchange costs more than it saves) and the chip one
    // CTA an SM, two thirds of that in clusters of eight, which leave SMs of a GPC over; of the rows along paths some four a sequence are there.  Measured
    // (bf16, top 20, us) with 1, 2, 4, 8, 16 CTAs a row: 1 row of 32000 entries 9.5, 10.3, 10.1, 10.9, 15; of 128256 15.0, 13.4, 11.8, 11.5, 15;
    // 16 rows of 151936 16.5, 14.6, 12.7, 13.8, 22; 64 of them 16.8, 15.0, 15.2, 28, 64.
    const int batch = logp::NT * logp::BATCH * (a->dtype == SPEC_F32 ? 4 : 8);
    const int64_t there = a->parent ? std::min<int64_t>(rows, (int64_t)a->B * 4) : rows;
    int C = 1;
    while (C < logp::CMAX && a->V > std::max(4, 2 * C) * batch && there * 2 * C <= (C == 4 ? sm_ctas() * 2 / 3 : sm_ctas())) C *= 2;
    logp::Params p = {};
    p.B = a->B; p.N = a->N; p.V = a->V; p.K = a->K; p.top = a->top; p.C = C;
    p.logits = a->logits; p.seq_stride = a->seq_stride; p.node_stride = a->node_stride;
    p.parent = a->parent; p.accepted = a->accepted_node; p.topo_seq_stride = a->topo_seq_stride; p.token = a->token;
    p.T = a->temperature; p.c = 1.4426950408889634f / a->temperature; p.room = 8.f / p.c;
    // (along paths 32 places at once: most end before, and a CTA without one ends at once; 8 sequences: 13.4 us for all 19 places, 13.9 for 8 at once, 21 for 4)
    p.step = a->parent ? std::min(a->N, 32) : a->N;
    p.logprob = a->logprob; p.entropy = a->entropy; p.top_logprobs = a->top_logprobs; p.top_tokens = a->top_tokens; p.status = a->status;
    const auto go = [&](auto kernel) {
        const int rc = prepare(kernel, std::max(logp::RING, 48 * 1024 + 1), false);          // (beside the static part)
        return rc ? rc : launch(kernel, dim3((unsigned)((a->parent ? (int64_t)a->B * p.step : rows) * C)), logp::NT, logp::RING, C > 1 ? C : 0, (cudaStream_t)stream, p);
    };
    return a->dtype == SPEC_F32  ? go(logp::spec_logprobs_kernel<float>)
           : a->dtype == SPEC_F16 ? go(logp::spec_logprobs_kernel<__half>)
                                  : go(logp::spec_logprobs_kernel<__nv_bfloat16>);
}

static int weights_check(const SpecWeights *a)
{
    if (!a || !a->q || !a->k_cache || !a->lse || !a->block_table || !a->lengths || !a->parent || !a->weights || !a->status) return SPEC_ERR_NULL;
    if (bad_tree_shape(a->B, a->N, a->topo_seq_stride) || bad_pages(a->num_blocks, a->block_size, a->table_width) ||
        a->table_stride < a->table_width || a->Hkv < 1 || a->Hq < a->Hkv || a->Hq % a->Hkv || a->Hq > 65535)
        return SPEC_ERR_SHAPE;
    if (a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_DTYPE;
    if (!(a->scale >= 0.f && a->scale <= 3.4e38f)) return SPEC_ERR_PARAM;
    if (a->D != 64 && a->D != 128 && a->D != 256) return SPEC_ERR_UNSUPPORTED;
    // (tiles of all heads, and steps of a run, are counted in 32 bits)
    const double tiles = ((double)std::min<int64_t>((int64_t)a->table_width * a->block_size, 0x7FFFFFFF) / weigh::KT + 2) * a->Hkv;
    const double steps = ((double)a->N * (a->Hq / a->Hkv)) / 64 + 1;
    if (a->B * tiles > 1.0e9 || a->B * tiles * steps / sm_ctas() > 1.0e9) return SPEC_ERR_UNSUPPORTED;          // (a tile's length is 2)
    int64_t all = 0;
    for (int j = 0; j < 3; ++j) all |= a->q_stride[j] | a->k_cache_stride[j];
    if (all % 8 || !aligned(a->q, 16) || !aligned(a->k_cache, 16)) return SPEC_ERR_UNSUPPORTED;
    return SPEC_OK;
}

struct WeightsLayout { int64_t part, joint, late, total; };
static WeightsLayout weights_layout(int ctas)
{
    WeightsLayout L = {};
    L.joint = (int64_t)ctas * 512 * 4;
    L.late = L.joint + (int64_t)ctas * 16;
    L.total = L.late + ((int64_t)ctas * 4 + 255) / 256 * 256;
    return L;
}

int32_t spec_cache_weights_workspace_bytes(const SpecWeights *a, int64_t *bytes)
{
    if (!bytes) return SPEC_ERR_NULL;
    const int rc = weights_check(a);
    if (rc) return rc;
    *bytes = weights_layout(sm_ctas()).total;
    return SPEC_OK;
}

int32_t spec_cache_weights(const SpecWeights *a, void *ws, int64_t ws_bytes, void *stream)
{
    const int rc = weights_check(a);
    if (rc) return rc;
    const int ctas = sm_ctas();
    const WeightsLayout L = weights_layout(ctas);
    if (!ws || !aligned(ws, 256) || ws_bytes < L.total) return SPEC_ERR_WORKSPACE;
    weigh::Params p = {};
    p.tree = tree_args(a->N, a->lengths, a->n_nodes, a->parent, a->topo_seq_stride);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = a->Hq / a->Hkv;
    p.num_blocks = a->num_blocks; p.block = a->block_size; p.width = a->table_width; p.fresh = a->fresh != 0;
    divisor(a->block_size, &p.block_mul, &p.block_shift);
    divisor(p.G, &p.group_mul, &p.group_shift);
    p.c = a->scale * weigh::LOG2E;
    p.q = a->q; p.k = a->k_cache; p.lse = a->lse; p.table = a->block_table; p.table_stride = a->table_stride;
    p.protect = a->protected_len; p.weights = a->weights; p.status = a->status;
    for (int j = 0; j < 3; ++j) { p.q_stride[j] = a->q_stride[j]; p.k_stride[j] = a->k_cache_stride[j]; }
    p.ctas = ctas;
    p.part = (float *)((unsigned char *)ws + L.part);
    p.joint = (int4 *)((unsigned char *)ws + L.joint);
    p.late = (int *)((unsigned char *)ws + L.late);
    const bool half = a->dtype == SPEC_F16;
    p.box = a->block_size % 8 ? 0 : a->block_size % 16 ? 8 : a->block_size % 32 ? 16 : 32;
    const int64_t sizes[4] = {a->D, a->Hkv, a->block_size, a->num_blocks};
    if (p.box && !tensor_map(&p.k_map, a->k_cache, half, sizes, {a->k_cache_stride[2], a->k_cache_stride[1], a->k_cache_stride[0]}, {1, p.box, 1}))
        p.box = 0;
    const auto go = [&](auto shape, auto kernel) -> int {
        using S = decltype(shape);
        if (S::QB % p.G == 0) {
            p.q_nodes = std::min(a->N, S::QB / p.G);
            const int64_t q_sizes[4] = {a->D, a->Hq, a->N, a->B};
            if (!tensor_map(&p.q_map, a->q, half, q_sizes, {a->q_stride[2], a->q_stride[1], a->q_stride[0]}, {p.G, p.q_nodes, 1})) p.q_nodes = 0;
        }
        const int smem = S::total + 1024;
        int e = prepare(kernel, smem, false);
        if (!e) e = prepare(weigh::spec_weigh_join_kernel, 0, false);
        if (e) return e;
        e = launch(kernel, dim3(ctas), weigh::NT, smem, 0, (cudaStream_t)stream, p);
        return e ? e : launch(weigh::spec_weigh_join_kernel, dim3(ctas + a->B), weigh::JOIN_NT, 0, 0, (cudaStream_t)stream, p);
    };
#define GO(D)                                                                                                  \
    (half ? go(weigh::Shape<D>(), weigh::spec_weigh_kernel<__half, weigh::Shape<D>>)                           \
          : go(weigh::Shape<D>(), weigh::spec_weigh_kernel<__nv_bfloat16, weigh::Shape<D>>))
    return a->D == 256 ? GO(256) : a->D == 128 ? GO(128) : GO(64);
#undef GO
}

static int evict_check(const SpecEvict *a)
{
    if (!a || !a->cache || !a->weights || !a->block_table || !a->lengths || !a->owned || !a->free_range || !a->lengths_out || !a->owned_out ||
        !a->free_range_out || !a->status || (a->free_size > 0 && !a->free_blocks))
        return SPEC_ERR_NULL;
    if (a->B < 1 || a->B > 65535 || bad_pages(a->num_blocks, a->block_size, a->table_width) || a->table_stride < a->table_width || a->caches < 1 ||
        a->row_bytes < 1 || a->row_bytes > 0x7FFFFFFF || a->free_size < 0)
        return SPEC_ERR_SHAPE;
    if (a->budget < 1 || a->recent < 0 || a->lengths_out == a->lengths || a->owned_out == a->owned || a->owned_out == a->lengths ||
        a->lengths_out == a->owned || a->free_range_out == a->free_range)
        return SPEC_ERR_PARAM;
    return SPEC_OK;
}
// (a request keeps no more entries than its row of the table has room for)
static int64_t most_moves(const SpecEvict *a) { return std::min<int64_t>(a->budget, (int64_t)a->table_width * a->block_size); }
static int64_t evict_bytes(const SpecEvict *a) { return ((int64_t)a->B * 8 + 255) / 256 * 256 + (int64_t)a->B * most_moves(a) * 8; }

int32_t spec_cache_evict_workspace_bytes(const SpecEvict *a, int64_t *bytes)
{
    if (!bytes) return SPEC_ERR_NULL;
    const int rc = evict_check(a);
    if (rc) return rc;
    *bytes = evict_bytes(a);
    return SPEC_OK;
}

int32_t spec_cache_evict(const SpecEvict *a, void *ws, int64_t ws_bytes, void *stream)
{
    int rc = evict_check(a);
    if (rc) return rc;
    if (!ws || !aligned(ws, 256) || ws_bytes < evict_bytes(a)) return SPEC_ERR_WORKSPACE;
    evict::Params p = {};
    p.B = a->B; p.caches = a->caches; p.budget = a->budget; p.recent = a->recent;
    p.num_blocks = a->num_blocks; p.block = a->block_size; p.width = a->table_width; p.free_size = a->free_size;
    p.cache = (unsigned char *)a->cache; p.weights = a->weights; p.table = a->block_table; p.table_stride = a->table_stride;
    p.lengths = a->lengths; p.owned = a->owned; p.protect = a->protected_len; p.range = a->free_range; p.ring = a->free_blocks;
    p.lengths_out = a->lengths_out; p.owned_out = a->owned_out; p.range_out = a->free_range_out; p.status = a->status;
    p.plan = (int2 *)ws;
    p.moves = (int2 *)((unsigned char *)ws + ((int64_t)a->B * 8 + 255) / 256 * 256);
    p.row_moves = most_moves(a);
    int64_t all = (int64_t)(uintptr_t)a->cache | a->row_bytes;
    for (int j = 0; j < 3; ++j) { p.stride[j] = a->stride[j]; all |= a->stride[j]; }
    const int unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
    p.total = (unsigned)(a->row_bytes / unit);
    // Slices of a row: 256 bytes, or fewer, down to 32, where that leaves fewer CTAs than two to an SM (a CTA goes through the kept entries in order): one request of
    // 13738 entries 75 us with 32 bytes, 256 with 256; 16 requests 614 and 359.
    p.words = std::min(p.total, 16u);
    while (p.words > 2 && (int64_t)((p.total + p.words - 1) / p.words) * a->caches * a->B < sm_ctas() * 2) p.words /= 2;
    p.slices = (int)((p.total + p.words - 1) / p.words);
    if ((int64_t)p.slices * a->caches + 1 > 0x7FFFFFFF) return SPEC_ERR_UNSUPPORTED;
    const cudaStream_t st = (cudaStream_t)stream;
    // (a row of the table, and weights of as many entries as a request can have)
    const int smem = (evict::COLS + (int)std::min<int64_t>(evict::KEYS, (int64_t)a->table_width * a->block_size)) * 4;
    rc = prepare(evict::spec_evict_select_kernel, (evict::COLS + evict::KEYS) * 4, false);
    if (!rc) rc = launch(evict::spec_evict_select_kernel, dim3(a->B), evict::NT, smem, 0, st, p);
    if (rc) return rc;
    const dim3 grid((unsigned)(p.slices * a->caches + 1), a->B);
    const auto go = [&](auto kernel) {
        const int e = prepare(kernel, 0, false);
        return e ? e : launch(kernel, grid, evict::MOVE_NT, 0, 0, st, p);
    };
    const bool few = (int64_t)p.slices * a->caches * a->B < sm_ctas() * 4;
    return unit == 16  ? few ? go(evict::spec_evict_move_kernel<uint4, 16>) : go(evict::spec_evict_move_kernel<uint4, 4>)
           : unit == 4 ? go(evict::spec_evict_move_kernel<uint32_t, 4>)
                       : go(evict::spec_evict_move_kernel<unsigned char, 4>);
}

}  // extern "C"
