// Norm and rotation of queries and keys per head, keys and values into the cache (spec_norm_rope_cache).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace specv {
namespace rope {

constexpr int NT = 128, ROT_MAX = 256;
template <int E> constexpr int CTAS = E == 16 ? 5 : 8;            // of an SM: what the registers have room for

struct Params {
    int T, Hq, Hkv, D, rot, pairs, lane_shift;     // 1 << lane_shift threads to a head's row, a power of two >= D / E
    int block, block_shift;
    unsigned block_mul;                            // slot / block = (umulhi(block_mul, slot) + slot) >> block_shift
    long long n_slots;
    const void *x[3];                              // q, k, v
    long long x_stride[3][2];
    const void *weight[2];
    float eps, inv_D;
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

// E entries of a row in registers
template <typename T, int E> struct __align__(16) Entries { T v[E]; };
template <typename T, bool VEC, int E> __device__ __forceinline__ Entries<T, E> load(const T *p)
{
    Entries<T, E> e;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(&e)[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) e.v[i] = p[i];
    }
    return e;
}
template <typename T, bool VEC, int E> __device__ __forceinline__ void store(T *p, const Entries<T, E> &e)
{
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(&e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) p[i] = e.v[i];
    }
}

// What a thread does to its E entries of a row: norm over the row's threads, rotation.
template <int E> struct Turner {
    int l, lanes, half;                            // thread of the row, threads of a row, threads of half a rotated part
    bool halves;
    const float2 *turn;
    float inv_D, eps;

    __device__ __forceinline__ void operator()(float (&y)[E], const float (&w)[E], bool norm) const
    {
        if (norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) sum = fmaf(y[i], y[i], sum);
            for (int o = lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float r = rsqrtf(sum * inv_D + eps);
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] = y[i] * r * w[i];
        }
        const bool turned = l < 2 * half;
        if (halves) {
            // the pair's other entry lies rot / 2 further on or back, with the same place in another thread
            const int lane = threadIdx.x & 31, other = turned ? (l < half ? lane + half : lane - half) & 31 : lane;
            const float4 *cs = (const float4 *)(turn + (turned ? (l < half ? l : l - half) * E : 0));
            const float sign = l < half ? -1.f : 1.f;
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                const float z0 = __shfl_sync(0xffffffffu, y[i], other), z1 = __shfl_sync(0xffffffffu, y[i + 1], other);
                if (!turned) continue;
                const float4 c = cs[i / 2];
                y[i] = y[i] * c.x + sign * (z0 * c.y);
                y[i + 1] = y[i + 1] * c.z + sign * (z1 * c.w);
            }
        } else if (turned) {
            const float4 *cs = (const float4 *)(turn + l * (E / 2));
#pragma unroll
            for (int i = 0; i < E; i += 4) {
                const float4 c = cs[i / 4];
                const float a0 = y[i], b0 = y[i + 1], a1 = y[i + 2], b1 = y[i + 3];
                y[i] = a0 * c.x - b0 * c.y;
                y[i + 1] = b0 * c.x + a0 * c.y;
                y[i + 2] = a1 * c.z - b1 * c.w;
                y[i + 3] = b1 * c.z + a1 * c.w;
            }
        }
    }
};
template <typename T, int E> __device__ __forceinline__ void widen(const Entries<T, E> &e, float (&y)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = to_f(e.v[i]);
}
template <typename T, int E> __device__ __forceinline__ void narrow(const float (&y)[E], Entries<T, E> &e)
{
    if constexpr (sizeof(T) == 2) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&e);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(y[2 * i + 1]), "f"(y[2 * i]));
            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(y[2 * i + 1]), "f"(y[2 * i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) e.v[i] = from_f<T>(y[i]);
    }
}

// A CTA per token, and several tokens one after the other in a long batch: the token's angles once for all heads (the position times a frequency, in
// turns, reduced in fp64: fp32 would lose 1e-2 of an angle at position 1e5), then a row per `lanes` threads, E entries each: the
// queries' rows two at a time, then those of keys and values side by side.  The first rows of each are on their way while the angles are computed.
// 6528 tokens of 48 heads of 128 entries (160 MB) take 39.4 us, 0.62 of the copy bandwidth: instructions (more than half of the issue slots) and the
// waits at the angles bound it, not yet the bytes.  CTAs of 256 threads and eight entries to a thread took 45 us, of 128 threads 40.6, and with
// sixteen entries 39.4; with the kinds of rows mixed in one loop it took 55, with a CTA per token 50, with the next token's first rows fetched
// behind this token's last 42.
template <typename T, bool VEC, int E> __global__ void __launch_bounds__(NT, CTAS<E>) spec_rope_kernel(const Params P)
{
    __shared__ __align__(16) float2 turns[2][ROT_MAX / 2];
    const int tid = threadIdx.x, lanes = 1 << P.lane_shift, groups = NT >> P.lane_shift, group = tid >> P.lane_shift, l = tid & (lanes - 1);
    // (threads behind the row's end, of rows of E * lanes entries, hold zeros)
    const bool on = l * E < P.D, on_q0 = on && group < P.Hq, on_q1 = on && group + groups < P.Hq, on_kv = on && group < 2 * P.Hkv;
    const bool norm_q = P.weight[0] != nullptr, norm_k = P.weight[1] != nullptr, first_key = group < P.Hkv;
    const T *q_head = (const T *)P.x[0] + group * P.x_stride[0][1] + l * E;
    T *out_head = (T *)P.q_out + group * P.q_out_stride[1] + l * E;
    const long long q_step = groups * P.x_stride[0][1], out_step = groups * P.q_out_stride[1];
    const auto kv_head = [&](int h) {
        return h < P.Hkv ? (const T *)P.x[1] + h * P.x_stride[1][1] + l * E : (const T *)P.x[2] + (h - P.Hkv) * P.x_stride[2][1] + l * E;
    };
    const auto cache_head = [&](int h) {
        return h < P.Hkv ? (T *)P.cache[0] + h * P.cache_stride[0][2] + l * E : (T *)P.cache[1] + (h - P.Hkv) * P.cache_stride[1][2] + l * E;
    };
    const T *kv_first = kv_head(group);
    T *cache_first = cache_head(group);
    grid_dependency_wait();
    int t = blockIdx.x, slot = __ldg(P.slots + t), pos = __ldg(P.positions + t);
    for (int turn_of = 0; t < P.T;) {
        const int now = t, here = slot, at = pos;
        t += gridDim.x;
        if (t < P.T) { slot = __ldg(P.slots + t); pos = __ldg(P.positions + t); }
        if (here < 0 || here >= P.n_slots) continue;
        const T *q = q_head + now * P.x_stride[0][0];
        T *out = out_head + now * P.q_out_stride[0];
        const long long k_token = now * P.x_stride[1][0], v_token = now * P.x_stride[2][0];
        Entries<T, E> a = {}, b = {}, c = {};
        if (on_q0) a = load<T, VEC, E>(q);
        if (on_q1) b = load<T, VEC, E>(q + q_step);
        if (on_kv) c = load<T, VEC, E>(kv_first + (first_key ? k_token : v_token));
        float2 *turn = turns[turn_of];             // (turned over only here: a token left out has no barrier that parts two uses)
        turn_of ^= 1;
        for (int i = tid; i < P.rot / 2; i += NT) {
            const double angle = (double)at * (double)__ldg(P.inv_freq + i) * 0.15915494309189533577;      // in turns: / 2 pi
            float sine, cosine;
            sincospif(2.f * (float)(angle - rint(angle)), &sine, &cosine);
            turn[i] = make_float2(cosine, sine);
        }
        __syncthreads();
        const Turner<E> turner = {l, lanes, P.rot / (2 * E), P.pairs == 0, turn, P.inv_D, P.eps};
        float w[E] = {}, y[E];
        if (on && norm_q) widen(load<T, VEC, E>((const T *)P.weight[0] + l * E), w);
        for (int h0 = 0; h0 < P.Hq; h0 += 2 * groups) {
            const int h = h0 + group;
            widen(a, y);
            turner(y, w, norm_q);
            narrow(y, a);
            if (on && h < P.Hq) store<T, VEC, E>(out, a);
            if (h0 + groups < P.Hq) {
                widen(b, y);
                turner(y, w, norm_q);
                narrow(y, b);
                if (on && h + groups < P.Hq) store<T, VEC, E>(out + out_step, b);
            }
            q += 2 * q_step;
            out += 2 * out_step;
            if (h0 + 2 * groups < P.Hq) {
                if (on && h + 2 * groups < P.Hq) a = load<T, VEC, E>(q);
                if (on && h + 3 * groups < P.Hq) b = load<T, VEC, E>(q + q_step);
            }
        }
        if (on && norm_k) widen(load<T, VEC, E>((const T *)P.weight[1] + l * E), w);
        const int block = (int)((__umulhi(P.block_mul, (unsigned)here) + (unsigned)here) >> P.block_shift), in = here - block * P.block;
        const long long k_slot = block * P.cache_stride[0][0] + in * P.cache_stride[0][1];
        const long long v_slot = block * P.cache_stride[1][0] + in * P.cache_stride[1][1];
        for (int h0 = 0; h0 < 2 * P.Hkv; h0 += groups) {
            const int h = h0 + group;
            const bool key = h < P.Hkv, live = on && h < 2 * P.Hkv;
            if (h0 && live) c = load<T, VEC, E>(kv_head(h) + (key ? k_token : v_token));
            if (__any_sync(0xffffffffu, key)) {
                Entries<T, E> turned;
                widen(c, y);
                turner(y, w, norm_k);
                narrow(y, turned);
                if (key) c = turned;
            }
            if (live) store<T, VEC, E>((h0 ? cache_head(h) : cache_first) + (key ? k_slot : v_slot), c);
        }
    }
}

}  // namespace rope
}  // namespace specv
