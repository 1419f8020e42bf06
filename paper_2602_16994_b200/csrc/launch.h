// Host side shared by the sources of the operators around a verification: launches, attributes of kernels, tensor maps, checks of shapes.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include "host.h"
#include "specverify.h"
#include "tree.cuh"

namespace specv {
namespace {

// A kernel that waits by itself for the one before it in the stream (so its CTAs may be placed while that one's last CTAs
// work), in clusters of C CTAs where C > 0.
template <typename P>
int launch(void (*kernel)(P), dim3 grid, int threads, int smem, int C, cudaStream_t st, const P &params)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (C > 0) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)C;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    void *args[1] = {const_cast<P *>(&params)};
    if (cudaLaunchKernelExC(&cfg, (const void *)kernel, args) != cudaSuccess) { cudaGetLastError(); return SPEC_ERR_CUDA; }
    count_launch();
    return SPEC_OK;
}

// Attributes of a kernel that its launch needs, set once per device: dynamic shared memory, clusters above 8 CTAs, and as much of an SM's L1 as can be as
// shared memory, for all kernels alike: CTAs of one that starts early find room beside those of the one before, and no SM is emptied
// to be divided anew between them.
std::mutex g_mutex;
template <typename K> int prepare(K kernel, int smem, bool big_clusters)
{
    struct Entry { const void *k; int dev; };
    static Entry cache[256];
    static int used = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return SPEC_ERR_CUDA; }
    std::lock_guard<std::mutex> lock(g_mutex);
    for (int i = 0; i < used; ++i)
        if (cache[i].k == (const void *)kernel && cache[i].dev == dev) return SPEC_OK;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        cudaGetLastError();
        return SPEC_ERR_CUDA;
    }
    if (big_clusters && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        return SPEC_ERR_CUDA;
    }
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess)
        cudaGetLastError();
    if (used < 256) cache[used++] = Entry{(const void *)kernel, dev};
    return SPEC_OK;
}

// Tensor map of 16-bit entries in four dimensions (sizes and strides in entries from the innermost, whose entries are contiguous), boxes 64 entries
// wide, 128-byte swizzle; false where it has no map.  The driver's function is asked for once.
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
bool tensor_map(CUtensorMap *map, const void *base, bool half, const int64_t (&size)[4], const int64_t (&stride)[3], const int (&box)[3])
{
    static const EncodeTiled encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess) {
            cudaGetLastError();
            return (EncodeTiled) nullptr;
        }
        return found == cudaDriverEntryPointSuccess ? (EncodeTiled)f : nullptr;
    }();
    if (!encode) return false;
    cuuint64_t dims[4], strides[3];
    for (int i = 0; i < 4; ++i) dims[i] = (cuuint64_t)size[i];
    for (int i = 0; i < 3; ++i) {
        const int64_t s = stride[i] * 2;                        // (nothing steps along a dimension of one entry)
        if (s < 0 || (s == 0 && size[i + 1] > 1) || s >= (1ll << 40)) return false;
        strides[i] = s ? (cuuint64_t)s : 16;
    }
    const cuuint32_t shape[4] = {64, (cuuint32_t)box[0], (cuuint32_t)box[1], (cuuint32_t)box[2]}, each[4] = {1, 1, 1, 1};
    return encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, shape,
                  each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTAs of a kernel that has one per SM
constexpr int CTAS_MAX = 160;
int sm_ctas()
{
    static std::atomic<int> cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return 148; }
    int n = cached[dev].load(std::memory_order_relaxed);
    if (n) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) { cudaGetLastError(); n = 148; }
    n = std::min(n, CTAS_MAX);
    cached[dev].store(n, std::memory_order_relaxed);
    return n;
}

TreeArgs tree_args(int N, const int32_t *lengths, const int32_t *n_nodes, const int32_t *parent, int64_t stride)
{
    return TreeArgs{N, lengths, n_nodes, parent, stride};
}
bool bad_tree_shape(int B, int N, int64_t topo_seq_stride)
{
    return B < 1 || B > 65535 || N < 1 || N > SPEC_MAX_NODES || (topo_seq_stride != 0 && topo_seq_stride < N);
}
bool bad_pages(int num_blocks, int block, int width)
{
    return num_blocks < 1 || block < 1 || width < 1 || (int64_t)num_blocks * block > 0x7FFFFFFF;
}
// floor(n / d) for n < 2^31 and 2^(s-1) < d <= 2^s: (n + umulhi(m, n)) >> s with m = floor(2^32 (2^s - d) / d) + 1
void divisor(uint64_t d, unsigned *mul, int *shift)
{
    *shift = 0;
    while ((1ull << *shift) < d) ++*shift;
    *mul = (unsigned)((((uint64_t)1 << 32) * ((1ull << *shift) - d)) / d + 1);
}
bool aligned(const void *p, int64_t n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) == 0; }

}  // namespace
}  // namespace specv
