// Norm and rotation of queries and keys per head, keys and values into the cache (spec_norm_rope_cache).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace specv {
namespace rope {

constexpr int NT = 256, WARPS = NT / 32, ROT_MAX = 256;

struct Params {
    int T, Hq, Hkv, D, rot, pairs, lanes;          // lanes: threads of a head's row, a power of two >= D / 8
    int block;
    long long n_slots;
    const void *x[3];                              // q, k, v
    long long x_stride[3][2];
    const void *weight[2];
    float eps;
    const float *inv_freq;
    const int *positions, *slots;
    void *q_out, *cache[2];
    long long q_out_stride[2], cache_stride[2][3];
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }

// eight entries of a row in registers
template <typename T> struct __align__(16) Eight { T v[8]; };
template <typename T, bool VEC> __device__ __forceinline__ Eight<T> load8(const T *p)
{
    Eight<T> e;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(&e)[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = p[i];
    }
    return e;
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(T *p, const Eight<T> &e)
{
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(&e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = e.v[i];
    }
}

// A CTA per token: its angles once for all heads (the position times a frequency, in turns, reduced in fp64: fp32 would lose 1e-2 of
// an angle at position 1e5), then a row per `lanes` threads, eight entries each.  Loads of the rows go out before the angles are
// computed.  Bound by the bytes of the projections.
template <typename T, bool VEC> __global__ void __launch_bounds__(NT) spec_rope_kernel(const Params P)
{
    __shared__ float2 turn[ROT_MAX / 2];
    const int tid = threadIdx.x, t = blockIdx.x;
    grid_dependency_wait();
    const int slot = __ldg(P.slots + t);
    if (slot < 0 || slot >= P.n_slots) return;
    const int heads = P.Hq + 2 * P.Hkv, group = tid / P.lanes, l = tid % P.lanes, groups = NT / P.lanes;
    const bool on = l * 8 < P.D;
    const int pos = __ldg(P.positions + t);
    for (int i = tid; i < P.rot / 2; i += NT) {
        const double turns = (double)pos * (double)__ldg(P.inv_freq + i) * 0.15915494309189533577;      // 1 / 2 pi
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        turn[i] = make_float2(c, s);
    }
    __syncthreads();
    const long long at_block = slot / P.block, at_slot = slot % P.block;
    for (int h0 = 0; h0 < heads; h0 += groups) {
        const int h = h0 + group;
        const int kind = h < P.Hq ? 0 : h < P.Hq + P.Hkv ? 1 : 2, head = kind == 0 ? h : kind == 1 ? h - P.Hq : h - P.Hq - P.Hkv;
        const bool live = on && h < heads;
        Eight<T> e;
        if (live) e = load8<T, VEC>((const T *)P.x[kind] + t * P.x_stride[kind][0] + head * P.x_stride[kind][1] + l * 8);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = live ? to_f(e.v[i]) : 0.f;
        const T *weight = kind < 2 ? (const T *)P.weight[kind] : nullptr;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
        for (int o = P.lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (weight && live) {
            const float r = 1.f / sqrtf(sum / (float)P.D + P.eps);
            const Eight<T> w = load8<T, false>(weight + l * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = y[i] * r * to_f(w.v[i]);
        }
        const int half = P.rot / 16;                               // threads of half a rotated part
        if (P.pairs == 0) {
            // the pair's other entry lies rot / 2 further on or back, with the same place in another thread
            const int lane = tid & 31, other = l < half ? lane + half : lane - half;
            const bool turned = l < 2 * half;
            const int i0 = (l < half ? l : l - half) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = __shfl_sync(0xffffffffu, y[i], turned ? other & 31 : lane);
                if (turned && kind < 2) {
                    const float2 cs = turn[i0 + i];
                    y[i] = l < half ? y[i] * cs.x - z * cs.y : y[i] * cs.x + z * cs.y;
                }
            }
        } else if (l < 2 * half && kind < 2) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 cs = turn[l * 4 + i / 2];
                const float a = y[i], b = y[i + 1];
                y[i] = a * cs.x - b * cs.y;
                y[i + 1] = b * cs.x + a * cs.y;
            }
        }
        if (!live) continue;
        if (kind < 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) e.v[i] = from_f<T>(y[i]);
        }
        T *to = kind == 0 ? (T *)P.q_out + t * P.q_out_stride[0] + head * P.q_out_stride[1]
                          : (T *)P.cache[kind - 1] + at_block * P.cache_stride[kind - 1][0] + at_slot * P.cache_stride[kind - 1][1]
                                + head * P.cache_stride[kind - 1][2];
        store8<T, VEC>(to + l * 8, e);
    }
}

}  // namespace rope
}  // namespace specv
