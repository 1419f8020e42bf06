// Verification of drafted chains from probabilities (spec_verify_probs).
#pragma once
#include <cooperative_groups.h>

#include <type_traits>

#include "common.cuh"

namespace specv {
namespace chain {
namespace cg = cooperative_groups;

// A cluster per request, a slice of the vocabulary per CTA.  Every CTA finds the accepted drafts by itself (a lane per draft: the
// chain is one round of dependent loads, whatever its length), then the cluster draws from the one row, or pair of rows, that the
// chain stopped at: the sums of tiles of 512 weights stay in shared memory, the slices' sums are exchanged, and the CTA that the
// target falls into finds the tile and reads it once more.  Weights, sums and comparisons are fp64: fp32 sums over 1e5 weights would move the
// borders between tokens by more than the tokens' own masses.  The bytes of one row of p and of q per request are the floor: 8 requests of
// 128256 entries take 8.3 us (floor 1.3: the walk, the row, its exchange and the tile are four rounds of latency), 128 looked-up ones of 151936 entries
// 22.5 (floor 12; 24.4 with q's zeros converted and subtracted too: a conversion to 64 bits costs several of the other instructions).
constexpr int NT = 256, WARPS = NT / 32, TILE = 512, TILES = 1024, CMAX = 16;      // a tile: four loads of 128 entries by a warp

struct Params {
    int B, V, SL, most;                 // SL: weights of a slice, a multiple of TILE
    long long n_drafts;
    const void *p, *q;
    long long p_stride, q_stride;
    const int *token, *cu;
    const float *u_accept, *u_bonus;
    int *accept_len, *out_tokens, *bonus, *status;
};

template <typename T> __device__ __forceinline__ float value(const T *p);
template <> __device__ __forceinline__ float value<float>(const float *p) { return __ldg(p); }
template <> __device__ __forceinline__ float value<unsigned short>(const unsigned short *p) { return __uint_as_float((uint32_t)__ldg(p) << 16); }

// four consecutive entries of a row; beyond the slice: 0
template <typename T> __device__ __forceinline__ float4 entries(const T *row, int t, int end, bool vec)
{
    if (vec && t + 3 < end) {
        if constexpr (sizeof(T) == 4) return __ldg(reinterpret_cast<const float4 *>(row + t));
        const uint2 w = __ldg(reinterpret_cast<const uint2 *>(row + t));
        return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
    }
    return make_float4(t < end ? value(row + t) : 0.f, t + 1 < end ? value(row + t + 1) : 0.f, t + 2 < end ? value(row + t + 2) : 0.f,
                       t + 3 < end ? value(row + t + 3) : 0.f);
}
// The rows that a draw reads: (p - q)+ where q is given, p without entry `hole` otherwise.
template <typename T> struct Rows {
    const T *p, *q;
    int hole;
    bool vec;
    template <bool Q> __device__ __forceinline__ void raw(int t, int end, float4 &a, float4 &b) const
    {
        a = entries(p, t, end, vec);
        b = Q && q ? entries(q, t, end, vec) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (hole >= t && hole < t + 4) {
            if (hole == t) a.x = 0.f;
            if (hole == t + 1) a.y = 0.f;
            if (hole == t + 2) a.z = 0.f;
            if (hole == t + 3) a.w = 0.f;
        }
    }
    // (the difference's sign is right in fp32, whose small numbers have no gap at 0; NaN stays, and what two infinities leave is NaN too)
    template <bool Q> static __device__ __forceinline__ double weight(float p, float q)
    {
        if constexpr (!Q) return (double)(p <= 0.f ? 0.f : p);
        const bool none = p - q <= 0.f;
        return (double)(none ? 0.f : p) - (double)(none ? 0.f : q);
    }
    template <bool Q> static __device__ __forceinline__ double sum(const float4 &a, const float4 &b)
    {
        return (weight<Q>(a.x, b.x) + weight<Q>(a.y, b.y)) + (weight<Q>(a.z, b.z) + weight<Q>(a.w, b.w));
    }
};

// first lane with running sum > tau (and weight); else the last with weight and rest = inf; -1 where there is none
__device__ __forceinline__ int first_above(double v, double tau, double &rest)
{
    const int lane = threadIdx.x & 31;
    double incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, v > 0.0 && incl > tau), pos = __ballot_sync(0xffffffffu, v > 0.0);
    const int at = hit ? __ffs(hit) - 1 : 31 - __clz(pos);
    const double before = __shfl_sync(0xffffffffu, incl - v, at < 0 ? 0 : at);
    rest = hit ? fmax(tau - before, 0.0) : CUDART_INF;
    return pos ? at : -1;
}

template <typename T> __global__ void __launch_bounds__(NT) spec_chain_kernel(const Params P)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ double tile[TILES], total[2][CMAX];
    grid_dependency_wait();
    int *out = P.out_tokens + (long long)b * (P.most + 1);
    // the accepted drafts (every warp alike)
    const long long first = __ldg(P.cu + b), end_draft = __ldg(P.cu + b + 1);
    const long long n = end_draft - first;
    int status = first < 0 || n < 0 || end_draft > P.n_drafts || n > P.most ? SPEC_DEV_TOPOLOGY : SPEC_DEV_OK;
    int len = 0;
    const T *p0 = (const T *)P.p + (first + b) * P.p_stride, *q0 = P.q ? (const T *)P.q + first * P.q_stride : nullptr;
    for (int i0 = 0; status == SPEC_DEV_OK && i0 < n; i0 += 32) {
        const int i = i0 + lane;
        bool stop = false;
        int wrong = SPEC_DEV_OK;
        if (i < n) {
            const int x = __ldg(P.token + first + i);
            if (x < 0 || x >= P.V) {
                wrong = SPEC_DEV_TOKEN;
            } else {
                const double px = (double)value(p0 + (long long)i * P.p_stride + x);
                const double qx = q0 ? (double)value(q0 + (long long)i * P.q_stride + x) : 1.0;
                if (!(px >= 0.0 && px < CUDART_INF && qx >= 0.0 && qx < CUDART_INF)) wrong = SPEC_DEV_NONFINITE;
                const double ratio = px > 0.0 ? (qx > 0.0 ? px / qx : 1.0) : 0.0;
                stop = !((double)__ldg(P.u_accept + first + i) < fmin(ratio, 1.0));
            }
        }
        const unsigned bad = __ballot_sync(0xffffffffu, wrong != SPEC_DEV_OK), rejected = __ballot_sync(0xffffffffu, stop);
        const int at = rejected ? __ffs(rejected) - 1 : 32;
        const unsigned upto = at >= 31 ? 0xffffffffu : (2u << at) - 1u;      // what lies behind the first rejected draft does not matter
        if (bad & upto) status = __shfl_sync(0xffffffffu, wrong, __ffs(bad & upto) - 1);
        if (rejected) { len = i0 + at; break; }
        len = (int)min((long long)i0 + 32, n);
    }
    const bool whole = len == n;                                             // all drafts accepted
    Rows<T> rows;
    rows.p = p0 + (long long)len * P.p_stride;
    rows.q = whole || !q0 ? nullptr : q0 + (long long)len * P.q_stride;
    rows.hole = -1;
    if (status == SPEC_DEV_OK && !whole && !q0) rows.hole = __ldg(P.token + first + len);
    const int t0 = rank * P.SL, end = min(P.V, t0 + P.SL), tiles = max(0, (end - t0 + TILE - 1) / TILE);
    double all = 0.0, mine = 0.0;
    const int per = ((tiles + 31) / 32) | 1, r0 = lane * per, r1 = min(tiles, r0 + per);
    if (status == SPEC_DEV_OK) {
        // (the second round: what was left of p is 0 everywhere, the draw is from p)
        for (int round = 0; round < 2; ++round) {
            rows.vec = (((uintptr_t)rows.p | (uintptr_t)rows.q) & (4 * sizeof(T) - 1)) == 0;
            const auto sums = [&](auto with_q) {         // (a loop of its own without q: half of the conversions to 64 bits)
                constexpr bool Q = decltype(with_q)::value;
                for (int i = warp; i < tiles; i += WARPS) {
                    const int t = t0 + i * TILE + lane * 4;
                    float4 x[4], y[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) rows.template raw<Q>(t + k * 128, end, x[k], y[k]);
                    double s = (rows.template sum<Q>(x[0], y[0]) + rows.template sum<Q>(x[1], y[1])) +
                               (rows.template sum<Q>(x[2], y[2]) + rows.template sum<Q>(x[3], y[3]));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                    if (lane == 0) tile[i] = s;
                }
            };
            if (rows.q) sums(std::true_type());
            else sums(std::false_type());
            __syncthreads();
            // a run of tiles per lane (of every warp alike: the slice's sum is needed by all)
            mine = 0.0;
            for (int i = r0; i < r1; ++i) mine += tile[i];
            const double slice = warp_sum(mine);
            if (C > 1) {
                cluster.sync();              // peers must be running, and through with the round before, when their shared memory is written
                if (tid < C) *cluster.map_shared_rank(&total[round][rank], tid) = slice;
                cluster.sync();
            } else {
                if (tid == 0) total[round][0] = slice;
                __syncthreads();
            }
            all = 0.0;
            for (int r = 0; r < C; ++r) all += total[round][r];
            if (!(all == 0.0) || whole) {
                if (!(all > 0.0 && all < CUDART_INF)) status = SPEC_DEV_NONFINITE;
                const double share = lane < C ? total[round][lane] : 0.0;
                mine = status == SPEC_DEV_OK ? mine : 0.0;
                double tau, tau2, tau3;
                const long long row = first + b + len;
                const int owner = status == SPEC_DEV_OK ? first_above(share, (double)__ldg(P.u_bonus + row) * all, tau) : 0;
                if (status == SPEC_DEV_OK && owner == rank && warp == 0) {
                    const int l = first_above(mine, tau, tau2);
                    int ti = -1;                             // the tile inside the lane's run, by that lane
                    double rest = tau2;
                    if (lane == l) {
                        int last = -1;
                        double run = 0.0, upto = 0.0;
                        for (int i = r0; i < r1; ++i) {
                            const double x = tile[i];
                            if (x > 0.0) last = i;
                            if (x > 0.0 && run + x > tau2) { ti = i; upto = run; break; }
                            run += x;
                        }
                        if (ti >= 0) rest = tau2 - upto;
                        else { ti = last; rest = CUDART_INF; }
                    }
                    ti = __shfl_sync(0xffffffffu, ti, l < 0 ? 0 : l);
                    rest = __shfl_sync(0xffffffffu, rest, l < 0 ? 0 : l);
                    // the tile's quarters in order, then the lane's four entries.  Where rounding leaves none above the target, the last with weight
                    int at = -1;
                    for (int k = 0; k < TILE; k += 128) {
                        const int t = t0 + ti * TILE + k + lane * 4;
                        float4 x, y;
                        rows.template raw<true>(t, end, x, y);
                        const double w[4] = {rows.template weight<true>(x.x, y.x), rows.template weight<true>(x.y, y.y),
                                             rows.template weight<true>(x.z, y.z), rows.template weight<true>(x.w, y.w)};
                        const double mine4 = (w[0] + w[1]) + (w[2] + w[3]), sum4 = warp_sum(mine4);
                        const int who = first_above(mine4, rest, tau3);
                        if (who < 0) continue;
                        int found = -1, last = -1;
                        double run = 0.0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            run += w[j];
                            if (w[j] > 0.0) last = j;
                            if (found < 0 && w[j] > 0.0 && run > tau3) found = j;
                        }
                        at = __shfl_sync(0xffffffffu, t + (found >= 0 ? found : last), who);
                        if (__shfl_sync(0xffffffffu, tau3, who) != CUDART_INF) break;
                        rest -= sum4;
                    }
                    const int token = at;
                    for (int i = lane; i <= P.most; i += 32)
                        out[i] = i < len ? __ldg(P.token + first + i) : i == len ? token : -1;
                    if (lane == 0) { P.accept_len[b] = len; P.bonus[b] = token; P.status[b] = SPEC_DEV_OK; }
                }
                break;
            }
            rows.q = nullptr;
            rows.hole = -1;
        }
        if (status == SPEC_DEV_OK && !(all > 0.0)) status = SPEC_DEV_NONFINITE;
    }
    if (status != SPEC_DEV_OK && rank == 0 && warp == 0) {
        for (int i = lane; i <= P.most; i += 32) out[i] = -1;
        if (lane == 0) { P.accept_len[b] = -1; P.bonus[b] = -1; P.status[b] = status; }
    }
}

}  // namespace chain
}  // namespace specv
