// What the dense operators share: element types, vectors of them, reductions
// over a warp, launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

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

// Most dynamic shared memory that any kernel here asks for (of 227 KB with what they declare).
constexpr int kDenseSmem = 226 << 10;

// SMs of the current device (0: the call failed); asked once per device.
inline int dense_sms() {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 0;
    if ((sms = known[dev].load(std::memory_order_relaxed)) != 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// Room for `bytes` of dynamic shared memory, asked for once per kernel and device.
template <class K>
inline bool dense_smem(K* kernel, size_t bytes) {
    if (bytes <= 32 << 10) return true;  // (what the kernel declares itself counts towards the 48 KB too)
    constexpr int kDevices = 64, kKernels = 256;
    static std::atomic<const void*> known[kDevices][kKernels];
    const void* id = reinterpret_cast<const void*>(kernel);
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return false;
    for (int i = 0; i < kKernels; ++i) {
        const void* k = known[dev][i].load(std::memory_order_acquire);
        if (k == id) return true;
        if (k) continue;
        // (whatever a launch may ask for, at once: a later one may ask for more)
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDenseSmem) != cudaSuccess) return false;
        known[dev][i].compare_exchange_strong(k, id);
        return true;
    }
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDenseSmem) == cudaSuccess;
}

// Working memory as the calls take it.
inline bool workspace_ok(const void* p, int64_t given, int64_t need) {
    return need == 0 || (p && given >= need && reinterpret_cast<uintptr_t>(p) % 256 == 0);
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

// Two 16-bit values in a word.
template <class T> __device__ __forceinline__ float2 pair_of_word(uint32_t w);
template <> __device__ __forceinline__ float2 pair_of_word<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 pair_of_word<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<__half2*>(&w));
}
template <class T> __device__ __forceinline__ uint32_t word_of_pair(float2 x);
template <> __device__ __forceinline__ uint32_t word_of_pair<__nv_bfloat16>(float2 x) {
    const __nv_bfloat162 r = __float22bfloat162_rn(x);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t word_of_pair<__half>(float2 x) {
    const __half2 r = __float22half2_rn(x);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Two fp32 operations at once.
__device__ __forceinline__ uint64_t as_x2(float2 v) { return *reinterpret_cast<uint64_t*>(&v); }
__device__ __forceinline__ float2 of_x2(uint64_t v) { return *reinterpret_cast<float2*>(&v); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(as_x2(a)), "l"(as_x2(b)));
    return of_x2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(as_x2(a)), "l"(as_x2(b)));
    return of_x2(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(as_x2(a)), "l"(as_x2(b)), "l"(as_x2(c)));
    return of_x2(r);
}

// N bytes (4, 8 or 16, aligned) on their way into shared memory.
template <int N>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(N) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sum over groups of G lanes (a power of two): every lane gets its group's.
__device__ __forceinline__ float group_sum(float x, int G) {
    for (int o = G >> 1; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace mlkv
