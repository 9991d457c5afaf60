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

// A launch in clusters of blocks; an error stays in cudaGetLastError().
template <typename... Params, typename... Args>
inline void launch_clusters(void (*kernel)(Params...), dim3 cluster, dim3 grid, int threads, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster.x;
    attr[0].val.clusterDim.y = cluster.y;
    attr[0].val.clusterDim.z = cluster.z;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = MLKV_PDL ? 2 : 1;
    cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
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

// The memory that a matrix spans, from its first value to its last.
struct Span {
    uintptr_t from, to;
    template <class T>
    __device__ __forceinline__ Span(const T* p, int64_t rows, int64_t stride, int dim)
        : from(reinterpret_cast<uintptr_t>(p)), to(reinterpret_cast<uintptr_t>(p + (rows - 1) * stride + dim)) {}
};

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

// V values as they lie in memory, read and written in pairs, kept in 32-bit words
// (16-bit values apart would take a register each).  ALIGNED: on 16 bytes (of x;
// 8 of a 16-bit y beside an fp32 x), and a row is whole vectors.  Else read as the
// two aligned pieces of that size around them, which are then shifted: nothing
// waits for the loads before that.  Written as wide as the row's place allows (the
// same for all its vectors): 8 bytes, 4, or, two bytes off, a half, words, a half.
template <class T, int V, bool ALIGNED> struct Values {
    static constexpr int W = sizeof(T) * V / 4, kBytes = sizeof(T) * V, kPieces = ALIGNED ? 1 : 2;
    uint32_t w[W];
    struct Around { uint32_t v[kPieces * W]; };

    static __device__ __forceinline__ const uint8_t* piece(const T* p) {
        return reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)(kBytes - 1));
    }
    static __device__ __forceinline__ bool inside(const uint8_t* at, int bytes, const Span& span) {
        return reinterpret_cast<uintptr_t>(at) >= span.from && reinterpret_cast<uintptr_t>(at) + bytes <= span.to;
    }
    // Of pieces that are not all the matrix's: the values that are, as words.
    static __device__ __forceinline__ uint32_t edge(const uint8_t* at, int i, const Span& span) {
        uint32_t r = 0;
#pragma unroll
        for (int h = 0; h < 4; h += sizeof(T)) {
            const uint8_t* q = at + i * 4 + h;
            if (reinterpret_cast<uintptr_t>(q) < span.from || reinterpret_cast<uintptr_t>(q) >= span.to) continue;
            if constexpr (sizeof(T) == 4) r = *reinterpret_cast<const uint32_t*>(q);
            else r |= (uint32_t)*reinterpret_cast<const uint16_t*>(q) << (8 * h);
        }
        return r;
    }
    static __device__ __forceinline__ void read(const void* p, uint32_t* to) {
        const Pack<uint32_t, W> q = *reinterpret_cast<const Pack<uint32_t, W>*>(p);
#pragma unroll
        for (int i = 0; i < W; ++i) to[i] = q.v[i];
    }
    // In two steps: what holds the values, ...
    static __device__ __forceinline__ Around around(const T* p, const Span& span) {
        Around r;
        if constexpr (ALIGNED) {
            read(p, r.v);
        } else {
            const uint8_t* at = piece(p);
            if (inside(at, 2 * kBytes, span)) {
                read(at, r.v);
                read(at + kBytes, r.v + W);
            } else {
#pragma unroll
                for (int i = 0; i < 2 * W; ++i) r.v[i] = edge(at, i, span);
            }
        }
        return r;
    }
    // ... and the first n of them (the rest 0), `by` bytes after a boundary.
    __device__ __forceinline__ void settle(Around r, uint32_t by, int n) {
        if constexpr (!ALIGNED) {
#pragma unroll
            for (int step = W / 2; step; step /= 2)
#pragma unroll
                for (int i = 0; i + step < 2 * W; ++i) r.v[i] = by & (4 * step) ? r.v[i + step] : r.v[i];
            if (sizeof(T) == 2)
#pragma unroll
                for (int i = 0; i < W; ++i) r.v[i] = __funnelshift_r(r.v[i], r.v[i + 1], (by & 2) * 8);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = r.v[i];
        if (!ALIGNED && n < V)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if constexpr (sizeof(T) == 4) w[i] = i < n ? w[i] : 0u;
                else w[i] = 2 * i + 1 < n ? w[i] : 2 * i < n ? w[i] & 0xFFFFu : 0u;
            }
    }
    static __device__ __forceinline__ uint32_t place(const T* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & (kBytes - 1); }
    __device__ __forceinline__ void load(const T* p, int n, const Span& span) { settle(around(p, span), place(p), n); }

    // From shared memory, where a matrix's pieces lie as they do in memory: the first n values from `at` on.
    __device__ __forceinline__ void take(const uint8_t* from, uint32_t at, int n) {
        Around r;
        if constexpr (ALIGNED) {
            read(from + at, r.v);
        } else {
            read(from + (at & ~(uint32_t)(kBytes - 1)), r.v);
            read(from + (at & ~(uint32_t)(kBytes - 1)) + kBytes, r.v + W);
        }
        settle(r, at & (kBytes - 1), n);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    // What was computed of the values is not to be kept for later: it takes more registers than they do.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int i = 0; i < W; ++i) asm volatile("" : "+r"(w[i]));
    }
    __device__ __forceinline__ float2 pair(int k) const {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
        else return pair_of_word<T>(w[k]);
    }
    __device__ __forceinline__ void set(int k, float2 x) {
        if constexpr (sizeof(T) == 4) {
            w[2 * k] = __float_as_uint(x.x);
            w[2 * k + 1] = __float_as_uint(x.y);
        } else {
            w[k] = word_of_pair<T>(x);
        }
    }
    // The first n values: as wide as the row's place allows (the same for all its vectors).
    __device__ __forceinline__ void store(T* p, int n) const {
        const uint32_t by = (uint32_t)reinterpret_cast<uintptr_t>(p);
        uint32_t* p32 = reinterpret_cast<uint32_t*>(p);
        uint16_t* p16 = reinterpret_cast<uint16_t*>(p);
        if (ALIGNED || (n >= V && !(by & (kBytes - 1)))) {
            Pack<uint32_t, W> q;
#pragma unroll
            for (int i = 0; i < W; ++i) q.v[i] = w[i];
            *reinterpret_cast<Pack<uint32_t, W>*>(p) = q;
        } else if (n >= V && !(by & 7)) {
#pragma unroll
            for (int i = 0; i < W; i += 2) *reinterpret_cast<uint2*>(p32 + i) = make_uint2(w[i], w[i + 1]);
        } else if (n >= V && !(by & 3)) {
#pragma unroll
            for (int i = 0; i < W; ++i) p32[i] = w[i];
        } else if constexpr (sizeof(T) == 2) {
            if (n >= V) {  // two bytes off a word: a half, the words between, a half
                p16[0] = (uint16_t)w[0];
#pragma unroll
                for (int i = 0; i + 1 < W; ++i) *reinterpret_cast<uint32_t*>(p16 + 1 + 2 * i) = __funnelshift_r(w[i], w[i + 1], 16);
                p16[V - 1] = (uint16_t)(w[W - 1] >> 16);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < n) p16[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (i < n) p32[i] = w[i];
        }
    }
};

// --- clusters of blocks ---------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address of the same place in block `rank` of the cluster.
__device__ __forceinline__ uint32_t place_in(uint32_t at, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
// (The threads of a warp arrive together.)
__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Sum over groups of G lanes (a power of two): every lane gets its group's.
__device__ __forceinline__ float group_sum(float x, int G) {
    for (int o = G >> 1; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

}  // namespace mlkv
