// What the dense operators share: element types, vectors of them, reductions
// over a warp, launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mlkv_dense.h"
#include "mlkv_internal.cuh"

#ifndef MLKV_NVTX
#define MLKV_NVTX 1
#endif
#if MLKV_NVTX
#include <nvtx3/nvToolsExt.h>
namespace mlkv {
struct DenseRange {
    explicit DenseRange(const char* name) { nvtxRangePushA(name); }
    ~DenseRange() { nvtxRangePop(); }
    DenseRange(const DenseRange&) = delete;
    DenseRange& operator=(const DenseRange&) = delete;
};
}  // namespace mlkv
#define MLKV_DENSE_RANGE(name) mlkv::DenseRange mlkv_dense_range_(name)
#else
#define MLKV_DENSE_RANGE(name) ((void)0)
#endif

namespace mlkv {

inline bool dense_type_ok(int32_t type) { return type >= MLKV_TYPE_FLOAT && type <= MLKV_TYPE_HALF; }
inline int dense_type_size(int32_t type) { return type == MLKV_TYPE_FLOAT ? 4 : 2; }

// SMs of the current device (0: the call failed).
inline int dense_sms() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms;
}

// V consecutive elements of T, moved by one load or store of V * sizeof(T) bytes.
template <class T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// An element of a vector whose type is known at run time (weights and biases:
// few, and read again by every row, so they come from L1).
__device__ __forceinline__ float load_as_float(const void* p, int32_t type, int64_t i) {
    if (type == MLKV_TYPE_FLOAT) return static_cast<const float*>(p)[i];
    if (type == MLKV_TYPE_BFLOAT) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int32_t type, int64_t i, float x) {
    if (type == MLKV_TYPE_FLOAT) static_cast<float*>(p)[i] = x;
    else if (type == MLKV_TYPE_BFLOAT) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
    else static_cast<__half*>(p)[i] = __float2half_rn(x);
}

// Sum over groups of G lanes (a power of two): every lane gets its group's.
__device__ __forceinline__ float group_sum(float x, int G) {
    for (int o = G >> 1; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace mlkv
