// Layer norm of rows and its gradients: what the two passes share.
//
// A row is held in registers by a team of L lanes (part of a warp, a warp, or
// several), vectors of V values dealt out in turn, so that it is read once.
#pragma once

#include <algorithm>
#include <initializer_list>
#include <utility>

#include "dense_common.cuh"

namespace mlkv {

constexpr int64_t kNormMaxDim = (int64_t)1 << 20;
constexpr int kNormLanes = 512;       // most lanes of a team: 128 registers a thread
constexpr int kNormLongLanes = 1024;  // lanes of the kernels of rows too long for registers

struct NormArgs {
    const void* x;
    const void* dy;
    void* out;       // y, or dx (may be null)
    const void* w;
    const void* b;
    float* stats;    // forward: out (may be null); backward: in
    float* part;     // backward: [blocks][2][dim] sums of each block, null: dweight and dbias at once
    void* dweight;
    void* dbias;
    int64_t x_stride, dy_stride, out_stride, rows;
    int32_t dim, w_type;
    float eps;
    int32_t lanes;   // L: lanes per row, a power of two below 32 or a multiple of 32
};

// Weights, held as fp32 in shared memory: in order, or, for vectors of 8, the
// first four values of every vector, then the last four (16-byte reads of
// neighbouring lanes then lie side by side).
template <int V>
__device__ __forceinline__ int weight_place(int c, int dim) {
    return V == 8 ? (((c >> 2) & 1) * (dim / 8) + (c >> 3)) * 4 + (c & 3) : c;
}
template <int V>
__device__ __forceinline__ void stage_weights(float* to, const void* p, int32_t type, int dim) {
    for (int c = threadIdx.x; c < dim; c += blockDim.x) to[weight_place<V>(c, dim)] = load_as_float(p, type, c);
}

// A vector of V values as it lies in memory, read and written in pairs (of one
// value: it and 0).  Kept in 32-bit words: 16-bit values apart would take a
// register each.
template <int V> constexpr int kPairs = (V + 1) / 2;
template <class T, int V> struct Values {
    static constexpr int kWords = sizeof(T) * V / 4;
    Pack<uint32_t, kWords> q;
    __device__ __forceinline__ void load(const T* p) { q = *reinterpret_cast<const Pack<uint32_t, kWords>*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Pack<uint32_t, kWords>*>(p) = q; }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) q.v[i] = 0;
    }
    __device__ __forceinline__ float2 pair(int k) const {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(q.v[2 * k]), V > 1 ? __uint_as_float(q.v[V > 1 ? 2 * k + 1 : 0]) : 0.f);
        else return pair_of_word<T>(q.v[k]);
    }
    __device__ __forceinline__ void set(int k, float2 x) {
        if constexpr (sizeof(T) == 4) {
            q.v[2 * k] = __float_as_uint(x.x);
            if (V > 1) q.v[V > 1 ? 2 * k + 1 : 0] = __float_as_uint(x.y);
        } else {
            q.v[k] = word_of_pair<T>(x);
        }
    }
};
template <class T> struct Half1 {
    uint16_t q;
    __device__ __forceinline__ void load(const T* p) { q = *reinterpret_cast<const uint16_t*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint16_t*>(p) = q; }
    __device__ __forceinline__ void zero() { q = 0; }
    __device__ __forceinline__ float2 pair(int) const { return make_float2(pair_of_word<T>(q).x, 0.f); }
    __device__ __forceinline__ void set(int, float2 x) { q = (uint16_t)word_of_pair<T>(make_float2(x.x, 0.f)); }
};
template <> struct Values<__nv_bfloat16, 1> : Half1<__nv_bfloat16> {};
template <> struct Values<__half, 1> : Half1<__half> {};

template <int V>
__device__ __forceinline__ void weight_pairs(const float* w, int j, int dim, float2 (&o)[kPairs<V>]) {
    if constexpr (V == 1) {
        o[0] = make_float2(w[j], 0.f);
    } else {
        constexpr int H = V > 4 ? 4 : V;
#pragma unroll
        for (int c = 0; c < V; c += H) {
            const Pack<float, H> q = *reinterpret_cast<const Pack<float, H>*>(w + weight_place<V>(j * V + c, dim));
#pragma unroll
            for (int k = 0; k < H / 2; ++k) o[c / 2 + k] = make_float2(q.v[2 * k], q.v[2 * k + 1]);
        }
    }
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Where a thread stands in its block's teams.
struct Team {
    int L, lane, index, count, warps, warp;  // lanes a row; this lane; this team; teams a block; warps a team; this warp of it
    __device__ explicit Team(int lanes)
        : L(lanes), lane(threadIdx.x % lanes), index(threadIdx.x / lanes), count(blockDim.x / lanes),
          warps(lanes / 32), warp((threadIdx.x % lanes) / 32) {}
    // The sums of a and b over the team.  buf: 2 x 32 pairs of the block, used in turn (turn: 0, 1, 0, ...), so
    // that one barrier a sum is enough: who writes a buffer again has seen all of its team past the next sum.
    __device__ __forceinline__ void sum(float& a, float& b, float2* buf, int turn) const {
        const int G = L < 32 ? L : 32;
        for (int o = G >> 1; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (L <= 32) return;
        float2* mine = buf + turn * 32 + index * warps;
        if ((threadIdx.x & 31) == 0) mine[warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(L) : "memory");  // (at most 4 teams of several warps)
        a = b = 0.f;
        for (int i = 0; i < warps; ++i) {
            const float2 q = mine[i];
            a += q.x;
            b += q.y;
        }
    }
    __device__ __forceinline__ float sum(float a, float2* buf, int turn) const {
        float none = 0.f;
        sum(a, none, buf, turn);
        return a;
    }
};

// Values per vector: 16 bytes of the wider type, or as many as every row and
// weight vector is aligned to.
inline int norm_vector_width(int64_t dim, std::initializer_list<std::pair<const void*, int>> bases,
                 std::initializer_list<int64_t> strides, int most) {
    int v = most;
    auto fits = [&](int n) {
        if (dim % n) return false;
        for (int64_t s : strides)
            if (s % n) return false;
        for (auto& b : bases)
            if (reinterpret_cast<uintptr_t>(b.first) % (uintptr_t)std::min(16, n * b.second)) return false;
        return true;
    };
    while (v > 1 && !fits(v)) v /= 2;
    return v;
}

struct NormShape {
    int V, NV, lanes;  // lanes == 0: the row does not fit
};
// The vectors a lane holds: as few lanes as hold the row with at most `most` values each.
inline NormShape norm_shape(int64_t dim, int V, int most) {
    const int64_t nvec = dim / V;
    int nv = 1;
    while (nv < 16 && nv * 2 * V <= most && nvec > (int64_t)32 * nv) nv *= 2;
    int64_t lanes = (nvec + nv - 1) / nv;
    if (lanes <= 32) {
        int p = 1;
        while (p < lanes) p *= 2;
        lanes = p;
    } else {
        lanes = (lanes + 31) / 32 * 32;
    }
    return {V, nv, lanes > kNormLanes ? 0 : (int)lanes};
}

template <class F>
bool by_types(int32_t x_type, int32_t y_type, F f) {
    using B = __nv_bfloat16;
    using H = __half;
    if (x_type == MLKV_TYPE_FLOAT && y_type == MLKV_TYPE_FLOAT) return f(float{}, float{}), true;
    if (x_type == MLKV_TYPE_FLOAT && y_type == MLKV_TYPE_BFLOAT) return f(float{}, B{}), true;
    if (x_type == MLKV_TYPE_FLOAT && y_type == MLKV_TYPE_HALF) return f(float{}, H{}), true;
    if (x_type == MLKV_TYPE_BFLOAT && y_type == MLKV_TYPE_BFLOAT) return f(B{}, B{}), true;
    if (x_type == MLKV_TYPE_HALF && y_type == MLKV_TYPE_HALF) return f(H{}, H{}), true;
    return false;
}
template <int N> struct Int { static constexpr int value = N; };
// f(values a vector, vectors a lane), of which a lane holds at most MOST values.
template <class T, int MOST, class F>
void by_width(int V, int NV, F f) {
    auto nv = [&](auto v) {
        constexpr int w = decltype(v)::value;
        if (NV == 1) f(v, Int<1>{});
        else if (NV == 2) f(v, Int<2>{});
        else if constexpr (4 * w <= MOST) {
            if (NV == 4) f(v, Int<4>{});
            else if constexpr (8 * w <= MOST) {
                if (NV == 8) f(v, Int<8>{});
                else if constexpr (16 * w <= MOST) f(v, Int<16>{});
            }
        }
    };
    if constexpr (sizeof(T) == 2)
        if (V == 8) return nv(Int<8>{});
    if (V >= 4) nv(Int<4>{});
    else if (V == 2) nv(Int<2>{});
    else nv(Int<1>{});
}

inline bool norm_ok(const void* x, int64_t x_stride, int32_t x_type, int32_t y_type, int32_t w_type, int64_t rows, int64_t dim) {
    if (rows < 0 || rows >= (int64_t)1 << 31 || dim < 1 || dim >= kNormMaxDim) return false;
    if (!dense_type_ok(x_type) || !dense_type_ok(y_type) || !dense_type_ok(w_type)) return false;
    if (x_type != y_type && x_type != MLKV_TYPE_FLOAT) return false;
    return rows == 0 || (x && x_stride >= dim);
}

inline int norm_team_threads(int lanes) { return lanes >= 256 ? lanes : 256 / lanes * lanes; }

}  // namespace mlkv
