// Log probabilities of given tokens, entropy and the likeliest alternatives
// (mlkv_token_logprobs), and the gradient of the logits
// (mlkv_token_logprobs_backward).
//
// With c = scale, m = max x, S = sum exp(c (x - m)), P = sum c (x - m) exp(c (x - m)):
//   log p_i = c (x_i - m) - log S,   H = log S - P / S
//   dx_i = c (g [i = t] - p_i (g + h (log p_i + H)))      (g, h: gradients of log p_t and H)
//
// Bound by HBM: the logits are read once (the backward pass reads and writes
// them once).  A block holds a chunk of a row in registers, finds its maximum,
// then its sums; a row of several chunks is joined by a second kernel.  The
// alternatives come out of the same registers: the k-th largest of the maxima
// of 32 disjoint parts of the chunk is at most the chunk's k-th largest value,
// and few other values reach it (about 30 for k = 20 where order and value have
// nothing to do with each other), so only those are sorted.
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "dense_common.cuh"

using namespace mlkv;

namespace {

constexpr int kMostThreads = 256;
constexpr int kCandidates = 512;       // values a chunk's alternatives are sorted from
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -200.f;       // 2^kLeast is 0 in fp32: what lies below (-inf too) need not be told apart

struct ProbArgs {
    const void* x;
    int64_t stride, n;
    const int64_t* targets;
    float scale;
    int32_t vocab, top, chunks, per_chunk;  // 16-byte pieces of a chunk
    float* logprob;
    float* entropy;
    float* stats;
    float* top_logprobs;
    int64_t* top_ids;
    float4* part;                // [n][chunks]: m, S, P of each chunk
    unsigned long long* keys;    // [n][chunks][top]
};

// A 16-byte piece of a row, which holds N values.
template <class T> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kMinusInf = 0xFF800000u;
    static __device__ __forceinline__ float2 pair(const uint4& q, int i) {
        return i == 0 ? make_float2(__uint_as_float(q.x), __uint_as_float(q.y)) : make_float2(__uint_as_float(q.z), __uint_as_float(q.w));
    }
    // The largest value, NaN where there is one.
    static __device__ __forceinline__ float max2(float a, float b) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
        return r;
    }
    static __device__ __forceinline__ float most(const uint4& q) {
        return max2(max2(__uint_as_float(q.x), __uint_as_float(q.y)), max2(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
};
template <> struct Piece<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    static __device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
    static __device__ __forceinline__ float2 pair(const uint4& q, int i) {
        const uint32_t w = word(q, i);
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ __nv_bfloat162 as2(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
    static __device__ __forceinline__ float most(const uint4& q) {
        const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(as2(q.x), as2(q.y)), __hmax2_nan(as2(q.z), as2(q.w)));
        return __bfloat162float(__hmax_nan(m.x, m.y));
    }
};
template <> struct Piece<__half> {
    static constexpr int N = 8;
    static constexpr uint32_t kMinusInf = 0xFC00FC00u;
    static __device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
    static __device__ __forceinline__ __half2 as2(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
    static __device__ __forceinline__ float2 pair(const uint4& q, int i) { return __half22float2(as2(word(q, i))); }
    static __device__ __forceinline__ float most(const uint4& q) {
        const __half2 m = __hmax2_nan(__hmax2_nan(as2(q.x), as2(q.y)), __hmax2_nan(as2(q.z), as2(q.w)));
        return __half2float(__hmax_nan(m.x, m.y));
    }
};

__device__ __forceinline__ float max_nan(float a, float b) { return Piece<float>::max2(a, b); }

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
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A row's values in 16-byte pieces: the first begins at or before the row's
// first value, on a 16-byte boundary; the values outside the row are not read.
template <class T>
struct RowPieces {
    const T* first;  // the first piece's place
    int before;      // its values that lie before the row
    int vocab, count;
    __device__ __forceinline__ RowPieces(const void* base, int64_t offset, int vocab_) : vocab(vocab_) {
        const T* row = static_cast<const T*>(base) + offset;
        before = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        first = row - before;
        count = (before + vocab + Piece<T>::N - 1) / Piece<T>::N;
    }
    __device__ __forceinline__ int index(int piece) const { return piece * Piece<T>::N - before; }  // of its first value
    __device__ __forceinline__ bool whole(int piece) const { return index(piece) >= 0 && index(piece) + Piece<T>::N <= vocab; }
    __device__ __forceinline__ uint4 load(int piece) const {
        constexpr int N = Piece<T>::N;
        if (whole(piece)) return *reinterpret_cast<const uint4*>(first + (int64_t)piece * N);
        constexpr uint32_t f = Piece<T>::kMinusInf;
        uint32_t w[4] = {f, f, f, f};
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int i = index(piece) + e;
            if (i < 0 || i >= vocab) continue;
            if constexpr (sizeof(T) == 4) {
                w[e] = *reinterpret_cast<const uint32_t*>(first + (int64_t)piece * N + e);
            } else {
                const uint32_t v = *reinterpret_cast<const uint16_t*>(first + (int64_t)piece * N + e);
                w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | v << 16 : (w[e / 2] & 0xFFFF0000u) | v;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// fp32 values in their order as unsigned numbers, NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (isnan(x)) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    if (o == 0xFFFFFFFFu) return CUDART_NAN_F;
    return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o);
}
// A candidate: its order, then the lowest index.  0: none; ~0: above all.
using Key = unsigned long long;
__device__ __forceinline__ Key key_of(float x, int index) { return (Key)order_of(x) << 32 | (0xFFFFFFFEu - (uint32_t)index); }

// The 32 lanes' values in falling order (bitonic sort; `from` = 32: of a bitonic sequence).
template <class K>
__device__ __forceinline__ K sort_lanes(K x, int lane, int from = 2) {
    for (int size = from; size <= 32; size <<= 1)
        for (int o = size >> 1; o; o >>= 1) {
            const K y = __shfl_xor_sync(0xffffffffu, x, o);
            const bool want_max = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
            x = want_max ? (x > y ? x : y) : (x < y ? x : y);
        }
    return x;
}
// The 32 largest of `count` keys, lane i holding the i-th (the warp).
__device__ __forceinline__ Key best_of(const Key* keys, int count, int lane) {
    Key best = sort_lanes<Key>(lane < count ? keys[lane] : 0ull, lane);
    for (int b = 32; b < count; b += 32) {
        const Key k = sort_lanes<Key>(b + lane < count ? keys[b + lane] : 0ull, lane);
        const Key other = __shfl_sync(0xffffffffu, k, 31 - lane);
        best = sort_lanes<Key>(best > other ? best : other, lane, 32);
    }
    return best;
}

// A row's results from its sums (the warp; lane i with its i-th alternative).
template <class T>
__device__ __forceinline__ void finish_row(const ProbArgs& a, int64_t r, float m, float s, float p, Key best, int lane) {
    const bool empty = m == -CUDART_INF_F, bad = isnan(m) || m == CUDART_INF_F;
    const float logs = bad ? CUDART_NAN_F : empty ? 0.f : logf(s);
    if (lane == 0) {
        const int64_t t = a.targets[r];
        float lp = 0.f;
        if (t >= a.vocab) lp = CUDART_NAN_F;
        else if (t >= 0) {
            const float x = to_float(static_cast<const T*>(a.x)[r * a.stride + t]);
            lp = empty ? -CUDART_INF_F : (x - m) * a.scale - logs;
        }
        a.logprob[r] = lp;
        a.entropy[r] = bad ? CUDART_NAN_F : empty ? 0.f : logs - kLn2 * p / s;
        a.stats[2 * r] = m;
        a.stats[2 * r + 1] = logs;
    }
    if (lane < a.top) {
        a.top_ids[r * a.top + lane] = best ? (int64_t)(0xFFFFFFFEu - (uint32_t)best) : -1;
        a.top_logprobs[r * a.top + lane] = best ? (value_of((uint32_t)(best >> 32)) - m) * a.scale - logs : -CUDART_INF_F;
    }
}

template <class T, int NV, bool TOP>
__global__ void __launch_bounds__(kMostThreads) k_logprobs(ProbArgs a) {
    pdl_enter();
    using P = Piece<T>;
    __shared__ float maxima[32];
    __shared__ float2 sums[kMostThreads / 32];
    __shared__ Key found[TOP ? kCandidates : 1];
    __shared__ int count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t r = blockIdx.x / (unsigned)a.chunks;
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks);
    const RowPieces<T> row(a.x, r * a.stride, a.vocab);
    const int p0 = chunk * a.per_chunk, p1 = min(row.count, p0 + a.per_chunk);
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = p0 + i * (int)blockDim.x + (int)threadIdx.x;
        constexpr uint32_t f = P::kMinusInf;
        q[i] = p < p1 ? row.load(p) : make_uint4(f, f, f, f);
    }
    if (TOP && threadIdx.x == 0) count = 0;
    float m = P::most(q[0]);
#pragma unroll
    for (int i = 1; i < NV; ++i) m = max_nan(m, P::most(q[i]));
    // the 32 parts' maxima: each that of as many lanes as there are warps
    for (int o = warps >> 1; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane % warps == 0) maxima[warp * (32 / warps) + lane / warps] = m;
    __syncthreads();
    m = maxima[lane];
    float least = 0.f;  // the smallest value that may be an alternative
    if (TOP) {
        const uint32_t sorted = sort_lanes<uint32_t>(order_of(m), lane);
        m = value_of(__shfl_sync(0xffffffffu, sorted, 0));
        least = value_of(__shfl_sync(0xffffffffu, sorted, a.top - 1));
        least = fmaxf(least, -3.4028234663852886e38f);  // (also where it is NaN: -inf is no alternative)
    } else {
        for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    const float base = m == -CUDART_INF_F ? 0.f : m, c = a.scale * kLog2e;
    const float2 minus = make_float2(-base, -base), c2 = make_float2(c, c);
    float2 s2 = make_float2(0.f, 0.f), t2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int k = 0; k < P::N / 2; ++k) {
            float2 d = mul2(add2(P::pair(q[i], k), minus), c2);
            d = make_float2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast));
            const float2 e = make_float2(exp2_fast(d.x), exp2_fast(d.y));
            s2 = add2(s2, e);
            t2 = fma2(d, e, t2);
        }
        if (TOP && P::most(q[i]) >= least) {
            const int at = row.index(p0 + i * (int)blockDim.x + (int)threadIdx.x);
#pragma unroll
            for (int k = 0; k < P::N / 2; ++k) {
                const float2 x = P::pair(q[i], k);
                if (x.x >= least) {
                    const int to = atomicAdd(&count, 1);
                    if (to < kCandidates) found[to] = key_of(x.x, at + 2 * k);
                }
                if (x.y >= least) {
                    const int to = atomicAdd(&count, 1);
                    if (to < kCandidates) found[to] = key_of(x.y, at + 2 * k + 1);
                }
            }
        }
    }
    float s = group_sum(s2.x + s2.y, 32), t = group_sum(t2.x + t2.y, 32);
    if (lane == 0) sums[warp] = make_float2(s, t);
    __syncthreads();
    int n = 0;
    if (TOP) {
        n = count;
        // More values than there is room for reach the bound (equal ones, as a rule), or NaN is among them: the
        // alternatives one by one.
        if (n > kCandidates || isnan(m)) {
            __syncthreads();
            n = a.top;
            Key mine = 0, last = ~0ull;
            bool look = true;
            for (int k = 0; k < a.top; ++k) {
                if (look) {
                    mine = 0;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int at = row.index(p0 + i * (int)blockDim.x + (int)threadIdx.x);
#pragma unroll
                        for (int e = 0; e < P::N / 2; ++e) {
                            const float2 x = P::pair(q[i], e);
                            const Key k0 = key_of(x.x, at + 2 * e), k1 = key_of(x.y, at + 2 * e + 1);
                            if (x.x != -CUDART_INF_F && k0 < last && k0 > mine) mine = k0;
                            if (x.y != -CUDART_INF_F && k1 < last && k1 > mine) mine = k1;
                        }
                    }
                }
                Key b = mine;
                for (int o = 16; o; o >>= 1) {
                    const Key y = __shfl_xor_sync(0xffffffffu, b, o);
                    b = b > y ? b : y;
                }
                if (lane == 0) found[32 + 8 * (k & 1) + warp] = b;
                __syncthreads();
                for (int w = 0; w < warps; ++w) {
                    const Key y = found[32 + 8 * (k & 1) + w];
                    b = b > y ? b : y;
                }
                if (threadIdx.x == 0) found[k] = b;
                look = b == mine;
                last = b;
            }
            __syncthreads();
        }
    }
    if (warp != 0) return;
    const float2 w = lane < warps ? sums[lane] : make_float2(0.f, 0.f);
    s = group_sum(w.x, 32);
    t = group_sum(w.y, 32);
    const Key best = TOP ? best_of(found, n, lane) : 0ull;
    if (a.chunks == 1) {
        finish_row<T>(a, r, m, s, t, best, lane);
        return;
    }
    if (lane == 0) a.part[blockIdx.x] = make_float4(m, s, t, 0.f);
    if (TOP && lane < a.top) a.keys[(int64_t)blockIdx.x * a.top + lane] = best;
}

// A row's chunks joined (a warp a row).
template <class T>
__global__ void __launch_bounds__(128) k_logprobs_join(ProbArgs a) {
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (r >= a.n) return;
    const float4* part = a.part + r * a.chunks;
    const float c = a.scale * kLog2e;
    float m = -CUDART_INF_F;
    for (int i = lane; i < a.chunks; i += 32) m = max_nan(m, part[i].x);
    for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = 0.f, t = 0.f;
    for (int i = lane; i < a.chunks; i += 32) {
        const float4 q = part[i];
        if (q.x == -CUDART_INF_F) continue;  // (its sums are of nothing)
        const float d = fmaxf((q.x - m) * c, kLeast), e = exp2f(d);
        s += q.y * e;
        t += (q.z + d * q.y) * e;
    }
    s = group_sum(s, 32);
    t = group_sum(t, 32);
    const Key best = a.top ? best_of(a.keys + r * a.chunks * a.top, a.chunks * a.top, lane) : 0ull;
    finish_row<T>(a, r, m, s, t, best, lane);
}

struct GradArgs {
    const void* x;
    void* dx;
    int64_t stride, dx_stride;
    const int64_t* targets;
    const float *entropy, *stats, *dlogprob, *dentropy;
    float scale;
    int32_t vocab, chunks, per_chunk;
};

template <class T>
__device__ __forceinline__ uint32_t pack2(float2 v) {
    if constexpr (sizeof(T) == 2) {
        T lo = from_float<T>(v.x), hi = from_float<T>(v.y);
        return (uint32_t)*reinterpret_cast<uint16_t*>(&lo) | (uint32_t)*reinterpret_cast<uint16_t*>(&hi) << 16;
    } else {
        return 0;
    }
}

template <class T, int NV>
__global__ void __launch_bounds__(kMostThreads) k_logprobs_backward(GradArgs a) {
    pdl_enter();
    using P = Piece<T>;
    constexpr int N = P::N;
    const int64_t r = blockIdx.x / (unsigned)a.chunks;
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks);
    const RowPieces<T> row(a.x, r * a.stride, a.vocab);
    T* out = static_cast<T*>(a.dx) + r * a.dx_stride - row.before;  // the piece's values' places
    const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
    const int p0 = chunk * a.per_chunk, p1 = min(row.count, p0 + a.per_chunk);
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = p0 + i * (int)blockDim.x + (int)threadIdx.x;
        if (p < p1) q[i] = row.load(p);
    }
    const float m = a.stats[2 * r], logs = a.stats[2 * r + 1];
    const int64_t target = a.targets[r];
    const float g = target >= 0 && a.dlogprob ? a.dlogprob[r] : 0.f, h = a.dentropy ? a.dentropy[r] : 0.f;
    // dx = p (A + B u) with u = log2 p, and scale g more at the target
    const float c = a.scale * kLog2e, base = m == -CUDART_INF_F ? 0.f : m;
    float A = -a.scale * (g + (h != 0.f ? h * a.entropy[r] : 0.f));
    const float B = -a.scale * h * kLn2, at_target = a.scale * g;
    if (isnan(m) || m == CUDART_INF_F || target >= a.vocab) A = CUDART_NAN_F;
    const float2 minus = make_float2(-base, -base), c2 = make_float2(c, c), A2 = make_float2(A, A), B2 = make_float2(B, B),
                 l2 = make_float2(-logs * kLog2e, -logs * kLog2e);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = p0 + i * (int)blockDim.x + (int)threadIdx.x;
        if (p >= p1) continue;
        const int at = row.index(p);
        float v[N];
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
            float2 u = fma2(add2(P::pair(q[i], k), minus), c2, l2);
            u = make_float2(fmaxf(u.x, kLeast), fmaxf(u.y, kLeast));
            const float2 d = mul2(make_float2(exp2_fast(u.x), exp2_fast(u.y)), fma2(B2, u, A2));
            v[2 * k] = d.x;
            v[2 * k + 1] = d.y;
        }
        if (target >= at && target < at + N) {
            // (a masked token has no gradient)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at + e == target && (e & 1 ? P::pair(q[i], e / 2).y : P::pair(q[i], e / 2).x) != -CUDART_INF_F) v[e] += at_target;
        }
        if (aligned && row.whole(p)) {
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float4*>(out + (int64_t)p * N) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                *reinterpret_cast<uint4*>(out + (int64_t)p * N) =
                    make_uint4(pack2<T>(make_float2(v[0], v[1])), pack2<T>(make_float2(v[2], v[3])),
                               pack2<T>(make_float2(v[N - 4], v[N - 3])), pack2<T>(make_float2(v[N - 2], v[N - 1])));
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at + e >= 0 && at + e < a.vocab) out[(int64_t)p * N + e] = from_float<T>(v[e]);
        }
    }
}

struct Split {
    int threads, NV, chunks, per_chunk;
};

// How a row of so many 16-byte pieces is cut: one chunk where a block's
// registers hold it, in as few threads as hold 4 pieces each; longer rows in
// equal chunks, smaller ones where there are too few rows to fill the GPU.
Split split_of(int64_t n, int64_t vocab, int size, int sms) {
    const int64_t pieces = (vocab * size + 15 + 15) / 16;  // wherever the row begins
    for (int t = 32; t <= kMostThreads; t *= 2)
        for (int nv = 1; nv <= 4; nv *= 2)
            if (pieces <= (int64_t)t * nv) return {t, nv, 1, (int)pieces};
    int nv = 8;
    while (nv > 2 && n * ((pieces + kMostThreads * nv - 1) / (kMostThreads * nv)) < 2 * sms) nv /= 2;
    const int64_t chunks = (pieces + kMostThreads * nv - 1) / (kMostThreads * nv);
    return {kMostThreads, nv, (int)chunks, (int)((pieces + chunks - 1) / chunks)};
}

template <class F>
bool by_type(int32_t type, F f) {
    if (type == MLKV_TYPE_FLOAT) f(float{});
    else if (type == MLKV_TYPE_BFLOAT) f(__nv_bfloat16{});
    else f(__half{});
    return true;
}
template <int N> struct Int { static constexpr int value = N; };
template <class F>
void by_pieces(int nv, F f) {
    if (nv == 1) f(Int<1>{});
    else if (nv == 2) f(Int<2>{});
    else if (nv == 4) f(Int<4>{});
    else f(Int<8>{});
}

bool probs_ok(int64_t n, int64_t vocab, int32_t type, float scale) {
    return n >= 0 && n < (int64_t)1 << 31 && vocab >= 1 && vocab < (int64_t)1 << 30 && dense_type_ok(type) && scale > 0.f && std::isfinite(scale);
}

// Blocks of a launch, at most 2^31 - 1 of them.
bool grid_ok(int64_t n, const Split& s) { return n * s.chunks < (int64_t)1 << 31; }

}  // namespace

extern "C" int64_t mlkv_token_logprobs_workspace(int64_t n, int64_t vocab, int32_t type, int32_t top) {
    if (!probs_ok(n, vocab, type, 1.f) || top < 0 || top > MLKV_MAX_TOP) return -1;
    if (n == 0) return 0;
    const int sms = dense_sms();
    if (!sms) return -1;
    const Split s = split_of(n, vocab, dense_type_size(type), sms);
    return s.chunks == 1 ? 0 : n * s.chunks * (16 + 8 * (int64_t)top);
}

extern "C" int mlkv_token_logprobs(const void* d_logits, int64_t stride, int32_t type, int64_t n, int64_t vocab,
                                   const int64_t* d_targets, float scale, int32_t top, float* d_logprob,
                                   float* d_entropy, float* d_stats, float* d_top_logprobs, int64_t* d_top_ids,
                                   void* d_workspace, int64_t workspace_bytes, void* stream) {
    MLKV_DENSE_RANGE("mlkv_token_logprobs");
    if (!probs_ok(n, vocab, type, scale) || top < 0 || top > MLKV_MAX_TOP) return MLKV_ERR_INVALID;
    if (n == 0) return MLKV_OK;
    if (!d_logits || stride < vocab || !d_targets || !d_logprob || !d_entropy || !d_stats) return MLKV_ERR_INVALID;
    if (top > 0 && (!d_top_logprobs || !d_top_ids)) return MLKV_ERR_INVALID;
    const int sms = dense_sms();
    if (!sms) return MLKV_ERR_CUDA;
    const Split s = split_of(n, vocab, dense_type_size(type), sms);
    if (!grid_ok(n, s)) return MLKV_ERR_UNSUPPORTED;
    if (s.chunks > 1 && (!d_workspace || workspace_bytes < n * s.chunks * (16 + 8 * (int64_t)top))) return MLKV_ERR_INVALID;
    ProbArgs a = {};
    a.x = d_logits; a.stride = stride; a.n = n; a.targets = d_targets; a.scale = scale; a.vocab = (int32_t)vocab;
    a.top = top; a.chunks = s.chunks; a.per_chunk = s.per_chunk; a.logprob = d_logprob; a.entropy = d_entropy;
    a.stats = d_stats; a.top_logprobs = d_top_logprobs; a.top_ids = d_top_ids;
    a.part = static_cast<float4*>(d_workspace);
    a.keys = reinterpret_cast<Key*>(a.part + n * s.chunks);
    cudaStream_t st = (cudaStream_t)stream;
    by_type(type, [&](auto t) {
        using T = decltype(t);
        by_pieces(s.NV, [&](auto nv) {
            constexpr int NV = decltype(nv)::value;
            const dim3 grid((unsigned)(n * s.chunks)), block(s.threads);
            if (top) launch_kernel(true, k_logprobs<T, NV, true>, grid, block, 0, st, a);
            else launch_kernel(true, k_logprobs<T, NV, false>, grid, block, 0, st, a);
        });
        if (s.chunks > 1) launch_kernel(true, k_logprobs_join<T>, dim3((unsigned)((n + 3) / 4)), dim3(128), 0, st, a);
    });
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

extern "C" int mlkv_token_logprobs_backward(const void* d_logits, int64_t stride, int32_t type, int64_t n, int64_t vocab,
                                            const int64_t* d_targets, float scale, const float* d_entropy,
                                            const float* d_stats, const float* d_dlogprob, const float* d_dentropy,
                                            void* d_dlogits, int64_t dlogits_stride, void* stream) {
    MLKV_DENSE_RANGE("mlkv_token_logprobs_backward");
    if (!probs_ok(n, vocab, type, scale)) return MLKV_ERR_INVALID;
    if (n == 0) return MLKV_OK;
    if (!d_logits || stride < vocab || !d_targets || !d_stats || (d_dentropy && !d_entropy) || !d_dlogits ||
        dlogits_stride < vocab || (d_dlogits == d_logits && dlogits_stride != stride)) return MLKV_ERR_INVALID;
    const int sms = dense_sms();
    if (!sms) return MLKV_ERR_CUDA;
    const Split s = split_of(n, vocab, dense_type_size(type), sms);
    if (!grid_ok(n, s)) return MLKV_ERR_UNSUPPORTED;
    GradArgs a = {};
    a.x = d_logits; a.dx = d_dlogits; a.stride = stride; a.dx_stride = dlogits_stride; a.targets = d_targets;
    a.entropy = d_entropy; a.stats = d_stats; a.dlogprob = d_dlogprob; a.dentropy = d_dentropy; a.scale = scale;
    a.vocab = (int32_t)vocab; a.chunks = s.chunks; a.per_chunk = s.per_chunk;
    cudaStream_t st = (cudaStream_t)stream;
    by_type(type, [&](auto t) {
        using T = decltype(t);
        by_pieces(s.NV, [&](auto nv) {
            launch_kernel(true, k_logprobs_backward<T, decltype(nv)::value>, dim3((unsigned)(n * s.chunks)), dim3(s.threads), 0, st, a);
        });
    });
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}
