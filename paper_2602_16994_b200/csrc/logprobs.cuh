// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits (spec_token_logprobs).
//
// Mathematics.  With m the largest logit and d = z - m: S = sum e^(d / T), U = sum e^(d / T) d; log p(t) = d_t / T - log S,
// H = log S - U / (S T): both terms of H are at least 0.  A thread takes a reference of its own in place of m, which may lie up to 8 powers of two below its
// largest logit, and moves its sums when that rises further; threads, then CTAs of a cluster, put theirs together about the largest of all.  Terms of U about
// a lower reference are positive, and moving it takes them away again: what that leaves is an error of H of up to about 8 ln 2 = 5.5 times that of an
// exponential (2^-22), whatever H is.  A reference that far below stands for a logit with a probability of at least 2^-8 beside the largest, so H is then above
// 0.02 and stays positive; where the reference is the largest logit itself, no term is positive.
//
// The most probable tokens.  A thread's maximum is that of its logits.  The n-th largest of a CTA's 256 maxima bounds the n-th largest logit from below, since
// n logits are at least that: after the one pass over the row only the stretches of a thread's logits are read again (from L2) whose
// maximum reaches the bound, about n of 1024, and the candidates of a CTA are put in order by counting.  The bound has the upper 16 bits of a maximum's image.
// Rows of which more entries of a CTA reach it than the candidates' room take longer.  Ties at the bound itself (rows under a mask, where it is -inf, and of few
// values) are filled up in index order, after a pass from the front (one value in all of 2048 rows of 151936 bf16 entries 861 us, top 20; normal ones 135).
// Where that many lie above the bound, the best are taken one at a time, in `top` more passes over the CTA's part of the row: fp32 and fp16 entries that the upper
// bits do not tell apart (normal rows of 50257 fp32 entries about 60000: 64 of them 266 us, about 0 16; 512 of 151936 about 1000: 2750, about 0 88), and ties of
// negative entries in any type, whose bits the bound's lower edge does not name (2048 rows of -1 in bf16: 6450 us).
//
// What bounds it.  One read of the rows: 2048 rows of 151936 bf16 entries in 135 us, 0.71 of the copy bandwidth (140 in a long row of calls; without the most
// probable 107 us, 0.90; with them the exponentials, the maxima and the search share the issue slots: 59 % of them).  Few rows: latency, of one launch, one row and the exchange in the cluster
// (1 row 9 to 12 us).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cut.cuh"
#include "tree.cuh"

namespace specv {
namespace logp {

constexpr int NT = 256, WARPS = NT / 32, BATCH = 4, SEGS = 4, ROOM = 512, CMAX = 8;
constexpr int STAGES = 3, RING = STAGES * BATCH * NT * 16;             // a thread's batches on their way, in shared memory (no barrier: it reads its own)
constexpr float LOW = -3.0e38f;                        // stands for -inf where 0 times it has to be 0

struct Params {
    int B, N, V, K, top, C, step;                      // step: places on a path that are gone through at once
    const void *logits;
    long long seq_stride, node_stride;
    const int *parent, *accepted, *token;
    long long topo_seq_stride;
    float c, T, room;                                  // log2(e) / T, T, 8 / c
    float *logprob, *entropy, *top_logprobs;
    int *top_tokens, *status;
};

template <typename T> struct Chunk;                    // 16 bytes of logits
template <> struct Chunk<float> {
    static constexpr int E = 4;
    static constexpr uint32_t MASKED = 0xFF800000u;    // a word of -inf
    static __device__ __forceinline__ void open(const uint4 &w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ float one(float x) { return x; }
    static __device__ __forceinline__ uint32_t top2(uint32_t a, uint32_t b)
    {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
        return __float_as_uint(r);
    }
    static __device__ __forceinline__ float last(uint32_t w) { return __uint_as_float(w); }
};
__device__ __forceinline__ float nan_max(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <> struct Chunk<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t MASKED = 0xFF80FF80u;
    static __device__ __forceinline__ void open(const uint4 &w, float (&x)[8])
    {
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]); }
    }
    static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ uint32_t top2(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float last(uint32_t w) { return nan_max(bf16_lo(w), bf16_hi(w)); }
};
template <> struct Chunk<__half> {
    static constexpr int E = 8;
    static constexpr uint32_t MASKED = 0xFC00FC00u;
    static __device__ __forceinline__ void open(const uint4 &w, float (&x)[8])
    {
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*(const __half2 *)&v[i]);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
    static __device__ __forceinline__ uint32_t top2(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float last(uint32_t w)
    {
        const float2 f = __half22float2(*(const __half2 *)&w);
        return nan_max(f.x, f.y);
    }
};

__device__ __forceinline__ void copy_chunk(uint32_t to, const uint4 *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// a candidate, larger is better: the logit's order, then the lower index
__device__ __forceinline__ unsigned long long rank_key(float z, int index)
{
    return ((unsigned long long)cut::key_of(z) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(unsigned long long k) { return cut::value_of((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }

struct Sums {                                          // of a CTA: largest logit, S and U about it
    double S, U;
    float m;
    int bad;
};
struct Shared {
    Sums sums;
    unsigned long long best[SPEC_MAX_TOP];             // 0: none
    unsigned long long found[ROOM + SPEC_MAX_TOP > CMAX * SPEC_MAX_TOP ? ROOM + SPEC_MAX_TOP : CMAX * SPEC_MAX_TOP];
    __align__(16) float maxima[NT];
    float stretch[SEGS][NT];
    unsigned short units[SEGS * NT];
    double warp_S[WARPS], warp_U[WARPS], log_S;
    float warp_m[WARPS];
    int count, n_units, depth, why;
    unsigned short path[SPEC_MAX_NODES];
    float bound;
    int warp_count[WARPS];
};
template <typename X> __device__ __forceinline__ const X *of_rank(const X *p, int rank)      // the same place in another CTA of the cluster
{
    uint64_t to;
    asm("mapa.u64 %0, %1, %2;" : "=l"(to) : "l"((uint64_t)p), "r"(rank));
    return (const X *)to;
}

// All threads: the `top` largest of found[0 .. n), in order, to best.
__device__ __forceinline__ void order(Shared *S, int n, int top, int tid)
{
    for (int i = tid; i < n; i += NT) {
        const unsigned long long x = S->found[i];
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) before += S->found[j] > x;
        if (before < top && x) S->best[before] = x;
    }
    __syncthreads();
}

template <typename T> __global__ void __launch_bounds__(NT, 3) spec_logprobs_kernel(const __grid_constant__ Params P)
{
    using X = Chunk<T>;
    constexpr int E = X::E;
    __shared__ Shared sh;
    Shared *S = &sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = P.C;
    const int rank = C > 1 ? (int)cluster_ctarank() : 0, row_of_grid = (int)(blockIdx.x / (unsigned)C);
    // (along paths the roots' rows come first, then those below: the rows that there are ahead of those that there are not)
    const int b = P.parent ? row_of_grid % P.B : row_of_grid / P.N, i0 = P.parent ? row_of_grid / P.B : row_of_grid - b * P.N;
    grid_dependency_wait();
    if (P.parent) {
        // the path: the parents on chip (they may be as many as fit the ring), then one thread goes up
        int *up = (int *)dyn_smem;
        const int *parent = P.parent + (long long)b * P.topo_seq_stride;
        for (int x = tid; x < P.N; x += NT) up[x] = __ldg(parent + x);
        const int acc = __ldg(P.accepted + b);
        __syncthreads();
        if (tid == 0) {
            int depth = 0, at = acc, bad = acc < -1 || acc >= P.N;
            if (!bad) {
                for (; at > 0; ++depth) {
                    const int above = up[at];
                    if (above < 0 || above >= at) { bad = 1; break; }
                    at = above;
                }
                bad |= acc >= 0 && up[0] != -1;
            }
            S->depth = bad ? -1 : acc < 0 ? -1 : depth;
            S->why = bad ? SPEC_DEV_TOPOLOGY : SPEC_DEV_OK;
            if (!bad && acc >= 0)
                for (int d = depth, node = acc; d >= 0; --d, node = up[node]) S->path[d] = (unsigned short)node;
        }
        __syncthreads();
    }
    for (int i = i0; i < P.N; i += P.step) {
    const int out = b * P.N + i;
    const int node = !P.parent ? i : i <= S->depth ? S->path[i] : -1, why = P.parent ? S->why : SPEC_DEV_OK;
    __syncthreads();                                   // (what the row before left in shared memory has been read)
    if (node < 0) {                                    // (all CTAs of the cluster alike)
        if (rank == 0) {
            for (int k = tid; k < P.K; k += NT) P.logprob[(long long)out * P.K + k] = 0.f;
            for (int k = tid; k < P.top; k += NT) { P.top_tokens[(long long)out * P.top + k] = -1; P.top_logprobs[(long long)out * P.top + k] = 0.f; }
            if (tid == 0) { P.entropy[out] = 0.f; P.status[out] = why; }
        }
        continue;
    }
    const T *row = (const T *)P.logits + (long long)b * P.seq_stride + (long long)node * P.node_stride;
    // (the first given tokens and their logits, asked for ahead of the row)
    const int my_token = rank == 0 && tid < P.K ? __ldg(P.token + (long long)out * P.K + tid) : -1;
    const float my_logit = my_token >= 0 && my_token < P.V ? X::one(row[my_token]) : 0.f;
    // ---- the row in 16-byte chunks, a few entries ahead of them and behind
    const int head = min(P.V, (int)((16u - (unsigned)((uintptr_t)row & 15u)) & 15u) / (int)sizeof(T));
    const int chunks = (P.V - head) / E, tail = P.V - head - chunks * E;
    const int per = (chunks + C - 1) / C, k0 = min(chunks, rank * per), k1 = min(chunks, k0 + per);
    const uint4 *body = (const uint4 *)(row + head) + k0;
    const int n = k1 - k0, batches = (n + NT * BATCH - 1) / (NT * BATCH), each = (batches + SEGS - 1) / SEGS;   // batches of a stretch
    // the ends go to the first CTA: entry -1: none
    const int edge = rank || tid >= head + tail ? -1 : tid < head ? tid : P.V - tail + tid - head;

    // The thread's largest logit m, its reference (behind m by 8 powers of two at most, so that it rarely moves: `over` is where it has to), and the sums about
    // it.
    float m = -CUDART_INF_F, ref = 0.f, over = -CUDART_INF_F, run = -CUDART_INF_F;
    bool bad = false;
    unsigned long long s2 = 0ull, u2 = 0ull;
    const unsigned long long c2 = pack_f32x2(P.c, P.c);
    const auto raise = [&](float to) {
        const float d = ref - to, f = over == -CUDART_INF_F ? 0.f : ex2_approx(d * P.c);
        const unsigned long long f2 = pack_f32x2(f, f), d2 = pack_f32x2(f == 0.f ? 0.f : d, f == 0.f ? 0.f : d);
        u2 = fma_f32x2(fma_f32x2(s2, d2, u2), f2, 0ull);
        s2 = fma_f32x2(s2, f2, 0ull);
        ref = to;
        over = to + P.room;
    };
    // (a masked logit: 0 times -inf where its distance is not bounded)
    const auto add2 = [&](float x, float y, unsigned long long r2, bool bound) {
        unsigned long long d2 = add_f32x2(pack_f32x2(x, y), r2);
        if (bound) {
            unpack_f32x2(d2, x, y);
            d2 = pack_f32x2(fmaxf(x, LOW), fmaxf(y, LOW));
        }
        const unsigned long long y2 = fma_f32x2(d2, c2, 0ull);
        unpack_f32x2(y2, x, y);
        const unsigned long long e2 = pack_f32x2(ex2_approx(x), ex2_approx(y));
        s2 = add_f32x2(s2, e2);
        u2 = fma_f32x2(e2, d2, u2);
    };
    const uint4 none = make_uint4(X::MASKED, X::MASKED, X::MASKED, X::MASKED);
    uint4 *ring = (uint4 *)dyn_smem;
    const auto fetch = [&](int batch) {
        if ((batch + 1) * (BATCH * NT) <= n) {
#pragma unroll
            for (int j = 0; j < BATCH; ++j)
                copy_chunk(smem_u32(ring + ((batch % STAGES) * BATCH + j) * NT + tid), body + (batch * BATCH + j) * NT + tid);
        } else if (batch < batches) {
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int k = (batch * BATCH + j) * NT + tid;
                uint4 *to = ring + ((batch % STAGES) * BATCH + j) * NT + tid;
                if (k < n) copy_chunk(smem_u32(to), body + k);
                else *to = none;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int g = 0; g < STAGES - 1; ++g) fetch(g);
    for (int g = 0, left = each, seg = 0; g < batches; ++g) {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        uint4 w[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) w[j] = ring[((g % STAGES) * BATCH + j) * NT + tid];
        uint32_t t = X::MASKED;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) t = X::top2(t, X::top2(X::top2(w[j].x, w[j].y), X::top2(w[j].z, w[j].w)));
        const float top = X::last(t);
        run = fmaxf(run, top);
        m = fmaxf(m, top);
        bad |= !(top < CUDART_INF_F);
        if (top > over) raise(top);
        const unsigned long long r2 = pack_f32x2(-ref, -ref), s_before = s2, u_before = u2;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            float x[E];
            X::open(w[j], x);
#pragma unroll
            for (int e = 0; e < E; e += 2) add2(x[e], x[e + 1], r2, false);
        }
        float ux, uy;
        unpack_f32x2(u2, ux, uy);
        if (__any_sync(0xffffffffu, !(fabsf(ux + uy) < CUDART_INF_F))) {
            // masked logits among them: once more, bounded
            s2 = s_before; u2 = u_before;
#pragma unroll 1
            for (int j = 0; j < BATCH; ++j) {
                float x[E];
                const uint4 v = ring[((g % STAGES) * BATCH + j) * NT + tid];
                X::open(v, x);
#pragma unroll
                for (int e = 0; e < E; e += 2) add2(x[e], x[e + 1], r2, true);
            }
        }
        fetch(g + STAGES - 1);
        if (--left == 0) { S->stretch[seg++][tid] = run; run = -CUDART_INF_F; left = each; }
        if (g + 1 == batches && left != each) S->stretch[seg][tid] = run;
    }
    float edge_x = -CUDART_INF_F;
    if (edge >= 0) {
        edge_x = X::one(row[edge]);
        bad |= !(edge_x < CUDART_INF_F);
        m = fmaxf(m, edge_x);
        if (edge_x > over) raise(edge_x);
        add2(edge_x, -CUDART_INF_F, pack_f32x2(-ref, -ref), true);
    }
    // ---- the CTA's sums
    {
        float top = m;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float x, y, p, q;
        unpack_f32x2(s2, x, y);
        unpack_f32x2(u2, p, q);
        const double d = m == -CUDART_INF_F ? 0.0 : (double)ref - (double)top;
        const float f = m == -CUDART_INF_F ? 0.f : ex2_approx((ref - top) * P.c);
        double s = (double)x + (double)y, u = (double)p + (double)q;
        u = f == 0.f ? 0.0 : (u + s * d) * (double)f;
        s *= (double)f;
        s = warp_sum(s);
        u = warp_sum(u);
        bad = __syncthreads_or(bad) != 0;
        if (lane == 0) { S->warp_m[warp] = top; S->warp_S[warp] = s; S->warp_U[warp] = u; }
        S->maxima[tid] = m;
        if (tid == 0) { S->count = 0; S->n_units = 0; S->bound = -CUDART_INF_F; }
        if (tid < SPEC_MAX_TOP) S->best[tid] = 0ull;
        __syncthreads();
    }
    // a warp puts the sums of its lanes together (a lane without any: m = -inf)
    const auto join = [&](float m1, double S1, double U1, bool wrong) {
        float top = m1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const double f = m1 == -CUDART_INF_F ? 0.0 : (double)ex2_approx((m1 - top) * P.c);
        // (0 times a distance that is infinite, of parts that are nothing)
        Sums a;
        a.U = warp_sum(f == 0.0 ? 0.0 : (U1 + S1 * ((double)m1 - (double)top)) * f);
        a.S = warp_sum(f == 0.0 ? 0.0 : S1 * f);
        a.m = top;
        a.bad = __any_sync(0xffffffffu, wrong);
        return a;
    };
    if (warp == 0) {
        const bool has = lane < WARPS;
        const Sums a = join(has ? S->warp_m[lane] : -CUDART_INF_F, has ? S->warp_S[lane] : 0.0, has ? S->warp_U[lane] : 0.0, bad);
        if (lane == 0) S->sums = a;
    }
    // ---- the CTA's most probable tokens
    if (P.top && !bad) {                               // (the same for all threads of the CTA)
        // One warp looks for the bound, by the upper 16 bits of an order-preserving image of the maxima: the largest that `top` maxima reach.
        if (warp == WARPS - 1) {
            uint32_t key[NT / 32], found = 0u;
#pragma unroll
            for (int j = 0; j < NT / 32; ++j) key[j] = cut::key_of(S->maxima[j * 32 + lane]) >> 16;
#pragma unroll 1
            for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
                int reach = 0;
#pragma unroll
                for (int j = 0; j < NT / 32; ++j) reach += __popc(__ballot_sync(0xffffffffu, key[j] >= (found | bit)));
                if (reach >= P.top) found |= bit;
            }
            // (what has the image of -inf, or of a number below all others, bounds nothing)
            const float x = cut::value_of(found << 16);
            if (lane == 0) S->bound = found > 0x007Fu && x == x ? x : -CUDART_INF_F;
        }
        __syncthreads();
        const float bound = S->bound;
        const auto put = [&](float x, int index) {
            const int at = atomicAdd(&S->count, 1);
            if (at < ROOM) S->found[at] = rank_key(x, index);
        };
        // entries that `wanted` names, of the stretches whose maximum it names
        const auto gather = [&](auto wanted) {
            for (int s = 0; s < SEGS && s * each < batches; ++s)
                if (wanted(S->stretch[s][tid])) S->units[atomicAdd(&S->n_units, 1)] = (unsigned short)(s * NT + tid);
            if (edge >= 0 && wanted(edge_x)) put(edge_x, edge);
            __syncthreads();
            // (four stretches of a warp on their way at once)
            for (int u0 = warp; u0 < S->n_units; u0 += 4 * WARPS) {
                for (int q0 = 0; q0 < each * BATCH; q0 += 32) {
                    uint4 w[4];
                    int at[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int u = u0 + v * WARPS, q = q0 + lane;
                        at[v] = -1;
                        w[v] = none;
                        if (u < S->n_units && q < each * BATCH) {
                            const int k = (S->units[u] / NT * each * BATCH + q) * NT + S->units[u] % NT;
                            if (k < n) { at[v] = k; w[v] = __ldg(body + k); }
                        }
                    }
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        if (at[v] < 0) continue;
                        float x[E];
                        X::open(w[v], x);
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (wanted(x[e])) put(x[e], head + (k0 + at[v]) * E + e);
                    }
                }
            }
            __syncthreads();
        };
        if (bound > -CUDART_INF_F) gather([&](float x) { return x >= bound; });
        int have = S->count;
        if (bound == -CUDART_INF_F || have > ROOM) {
            // more ties than room, or a mask: what lies above the bound, then as many of the bound's entries as are lacking, the lowest first
            __syncthreads();
            if (tid == 0) { S->count = 0; S->n_units = 0; }
            __syncthreads();
            gather([&](float x) { return x > bound; });
            have = S->count;
            if (have <= ROOM) {
                int lacking = P.top - have;
                // in index order: the entries ahead of the chunks, the chunks, the entries behind
                bool behind = false;
                for (int round = -1; lacking > 0 && !behind; ++round) {
                    int mine = 0, at[E] = {};
                    behind = round >= 0 && round * NT >= n;
                    if (round < 0) {
                        if (edge >= 0 && tid < head && edge_x == bound) at[mine++] = edge;
                    } else if (behind) {
                        if (edge >= 0 && tid >= head && edge_x == bound) at[mine++] = edge;
                    } else if (round * NT + tid < n) {
                        const int k = round * NT + tid;
                        float x[E];
                        X::open(__ldg(body + k), x);
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (x[e] == bound) at[mine++] = head + (k0 + k) * E + e;
                    }
                    int incl = mine;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int y = __shfl_up_sync(0xffffffffu, incl, o);
                        if (lane >= o) incl += y;
                    }
                    if (lane == 31) S->warp_count[warp] = incl;
                    __syncthreads();
                    int ahead = incl - mine, all = 0;
                    for (int w = 0; w < WARPS; ++w) {
                        if (w < warp) ahead += S->warp_count[w];
                        all += S->warp_count[w];
                    }
                    for (int e = 0; e < mine && ahead + e < lacking; ++e) S->found[have + ahead + e] = rank_key(bound, at[e]);
                    __syncthreads();
                    const int got = min(all, lacking);
                    have += got;
                    lacking -= got;
                }
            } else {
                // more than the room above the bound as well (entries that its 16 bits do not tell apart): one at a time, the best behind the last
                unsigned long long last = ~0ull;
                for (int a = 0; a < P.top; ++a) {
                    unsigned long long best = 0ull;
                    const auto look = [&](float x, int index) {
                        const unsigned long long key = rank_key(x, index);
                        if (key < last && key > best) best = key;
                    };
                    if (edge >= 0) look(edge_x, edge);
                    for (int k = tid; k < n; k += NT) {
                        float x[E];
                        X::open(__ldg(body + k), x);
#pragma unroll
                        for (int e = 0; e < E; ++e) look(x[e], head + (k0 + k) * E + e);
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    __syncthreads();
                    if (lane == 0) S->found[warp] = best;
                    __syncthreads();
                    for (int w = 0; w < WARPS; ++w) best = max(best, S->found[w]);
                    if (tid == 0) S->found[WARPS + a] = best;
                    last = best;
                    __syncthreads();
                }
                if (tid < WARPS) S->found[tid] = 0ull;
                have = WARPS + P.top;
                __syncthreads();
            }
        }
        order(S, have, P.top, tid);
    }
    __syncthreads();
    // ---- the cluster's
    if (C > 1) {
        cluster_sync_all();
        if (rank == 0) {
            for (int k = tid; k < C * P.top; k += NT) S->found[k] = of_rank(S->best, k / P.top)[k % P.top];
            __syncthreads();                           // (its own list is read before it is written again)
            if (warp == 0) {
                const bool has = lane < C;
                const Sums o = *of_rank(&S->sums, has ? lane : 0);
                const Sums a = join(has ? o.m : -CUDART_INF_F, o.S, o.U, has && o.bad);
                __syncwarp();
                if (lane == 0) S->sums = a;
            }
            if (tid < SPEC_MAX_TOP) S->best[tid] = 0ull;
            __syncthreads();
            if (P.top) order(S, C * P.top, P.top, tid);
        }
        cluster_sync_all();                            // (no CTA goes on while the first one reads it)
        if (rank) continue;
    }
    // ---- results
    const Sums a = S->sums;
    const bool wrong = a.bad || a.m == -CUDART_INF_F;
    if (tid == 0) S->log_S = wrong ? 0.0 : log(a.S);
    __syncthreads();
    const double log_S = S->log_S, T_d = (double)P.T;
    const auto value = [&](float z) { return wrong ? CUDART_NAN_F : (float)(((double)z - (double)a.m) / T_d - log_S); };
    bool no_token = false;
    for (int k = tid; k < P.K; k += NT) {
        const int token = k < NT ? my_token : __ldg(P.token + (long long)out * P.K + k);
        float v = 0.f;
        if (token < -1 || token >= P.V) { v = CUDART_NAN_F; no_token = true; }
        else if (token >= 0) v = value(k < NT ? my_logit : X::one(row[token]));
        P.logprob[(long long)out * P.K + k] = v;
    }
    for (int k = tid; k < P.top; k += NT) {
        const unsigned long long key = S->best[k];
        P.top_tokens[(long long)out * P.top + k] = wrong ? -1 : key_index(key);
        P.top_logprobs[(long long)out * P.top + k] = value(key_value(key));
    }
    no_token = __syncthreads_or(no_token) != 0;
    if (tid == 0) {
        P.entropy[out] = wrong ? CUDART_NAN_F : (float)(log_S - a.U / (a.S * T_d));
        P.status[out] = wrong ? SPEC_DEV_NONFINITE : no_token ? SPEC_DEV_TOKEN : SPEC_DEV_OK;
    }
    }
}

}  // namespace logp
}  // namespace specv
