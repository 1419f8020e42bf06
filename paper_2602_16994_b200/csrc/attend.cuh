// Attention of the nodes of draft trees over a paged cache (spec_tree_attention).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tree.cuh"

namespace specv {
namespace attend {

struct Params {
    TreeArgs tree;
    int B, Hq, Hkv, D, num_blocks, block, width, window, sinks;
    float scale;
    const void *q, *k, *v;
    long long q_stride[3], k_stride[3], v_stride[3];
    const int *table;
    long long table_stride;
    void *out;
    long long out_stride[3];
    float *lse;
    int *status;
};

__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

constexpr int NT = 128, GB = 4;

// A CTA per node, key head and request; a thread per key for the scores, a thread per entry of the head for the sums.
template <typename T> __global__ void __launch_bounds__(NT) spec_attend_kernel(const Params P)
{
    __shared__ int parent[SPEC_MAX_NODES], depth_of[SPEC_MAX_NODES];
    __shared__ unsigned char above[SPEC_MAX_NODES];
    __shared__ float q[GB][256], p[GB][NT], red[GB][4];
    __shared__ long long vrow[NT];
    grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.z, node = blockIdx.y, h = blockIdx.x, D = P.D;
    const int len = __ldg(P.tree.lengths + b), nn = tree_nodes(P.tree, b), n = max(nn, 0);
    const bool teller = node == 0 && h == 0;
    if (len < 0 || nn < 0) {
        if (teller && tid == 0) P.status[b] = len >= 0 ? SPEC_DEV_TOPOLOGY : SPEC_DEV_OK;
        return;
    }
    const int *row = P.tree.parent + (long long)b * P.tree.topo_seq_stride;
    bool bad = false;
    for (int i = tid; i < n; i += NT) {
        const int pa = __ldg(row + i);
        bad |= i == 0 ? pa != -1 : pa < 0 || pa >= i;
        parent[i] = pa;
        above[i] = 0;
    }
    bad = __syncthreads_or(bad) != 0;
    const int *table = P.table + (long long)b * P.table_stride;
    const auto block_of = [&](long long at) -> int {
        const long long col = at / P.block;
        const int id = col < P.width ? __ldg(table + col) : -1;
        return id < 0 || id >= P.num_blocks ? -1 : id;
    };
    if (teller) {
        bool page = false;
        for (long long j = tid; j < (long long)len + n; j += NT) {
            const bool seen = j >= len || P.window == 0 || j < P.sinks || j > (long long)len - P.window;
            page |= seen && block_of(j) < 0;
        }
        page = __syncthreads_or(page) != 0;
        if (tid == 0) P.status[b] = bad ? SPEC_DEV_TOPOLOGY : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
    }
    if (node >= n) return;
    if (!bad && tid == 0) {
        int d = 0;
        for (int i = node; i > 0; i = parent[i]) ++d;
        for (int i = node, e = d; i >= 0; i = parent[i], --e) { above[i] = 1; depth_of[i] = e; }
    }
    __syncthreads();
    const int G = P.Hq / P.Hkv;
    const long long t = bad ? 0 : (long long)len + depth_of[node];
    const T *k_head = (const T *)P.k + h * P.k_stride[2], *v_head = (const T *)P.v + h * P.v_stride[2];
    for (int g0 = 0; g0 < G; g0 += GB) {
        const int gn = min(GB, G - g0);
        for (int i = tid; i < gn * D; i += NT)
            q[i / D][i % D] = to_f(((const T *)P.q)[b * P.q_stride[0] + node * P.q_stride[1] + (h * G + g0 + i / D) * P.q_stride[2] + i % D]);
        float m[GB], l[GB], acc[GB][2];
        for (int g = 0; g < GB; ++g) { m[g] = -CUDART_INF_F; l[g] = 0.f; acc[g][0] = acc[g][1] = 0.f; }
        __syncthreads();
        const long long keys = bad ? 0 : (long long)len + n;
        for (long long j0 = 0; j0 < keys; j0 += NT) {
            const long long j = j0 + tid;
            bool seen = j < len || (j < keys && above[j - len]);
            if (seen && P.window) {
                const long long pos = j < len ? j : (long long)len + depth_of[j - len];
                seen = pos > t - P.window || pos < P.sinks;
            }
            if (!__syncthreads_or(seen)) continue;
            const int id = seen ? block_of(j) : -1;
            seen = id >= 0;
            float s[GB];
            for (int g = 0; g < GB; ++g) s[g] = -CUDART_INF_F;
            vrow[tid] = seen ? id * P.v_stride[0] + (j % P.block) * P.v_stride[1] : -1;
            if (seen) {
                const T *k = k_head + id * P.k_stride[0] + (j % P.block) * P.k_stride[1];
                for (int g = 0; g < gn; ++g) s[g] = 0.f;
                for (int d = 0; d < D; ++d) {
                    const float x = to_f(k[d]);
                    for (int g = 0; g < gn; ++g) s[g] = fmaf(q[g][d], x, s[g]);
                }
                for (int g = 0; g < gn; ++g) s[g] *= P.scale;
            }
            for (int g = 0; g < gn; ++g) {
                float x = s[g];
                for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
                if (lane == 0) red[g][warp] = x;
            }
            __syncthreads();
            for (int g = 0; g < gn; ++g) {
                const float top = fmaxf(m[g], fmaxf(fmaxf(red[g][0], red[g][1]), fmaxf(red[g][2], red[g][3])));
                const float ref = top == -CUDART_INF_F ? 0.f : top;
                const float c = expf(m[g] - ref);
                m[g] = top;
                l[g] *= c; acc[g][0] *= c; acc[g][1] *= c;
                p[g][tid] = seen ? expf(s[g] - ref) : 0.f;
            }
            __syncthreads();
            for (int i = 0; i < NT; ++i) {
                if (vrow[i] < 0) continue;
                const float v0 = tid < D ? to_f(v_head[vrow[i] + tid]) : 0.f, v1 = tid + NT < D ? to_f(v_head[vrow[i] + tid + NT]) : 0.f;
                for (int g = 0; g < gn; ++g) {
                    l[g] += p[g][i];
                    acc[g][0] = fmaf(p[g][i], v0, acc[g][0]);
                    acc[g][1] = fmaf(p[g][i], v1, acc[g][1]);
                }
            }
            __syncthreads();
        }
        for (int g = 0; g < gn; ++g) {
            const int head = h * G + g0 + g;
            T *o = (T *)P.out + b * P.out_stride[0] + node * P.out_stride[1] + head * P.out_stride[2];
            const float r = l[g] == 0.f ? 0.f : 1.f / l[g];
            if (tid < D) o[tid] = (T)(acc[g][0] * r);
            if (tid + NT < D) o[tid + NT] = (T)(acc[g][1] * r);
            if (P.lse && tid == 0)
                P.lse[((long long)b * P.tree.N + node) * P.Hq + head] = l[g] == 0.f ? -CUDART_INF_F : m[g] + logf(l[g]);
        }
        __syncthreads();
    }
}

}  // namespace attend
}  // namespace specv
