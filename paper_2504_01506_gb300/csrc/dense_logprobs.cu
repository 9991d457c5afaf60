// Log probabilities of given tokens, entropy and the likeliest alternatives
// (mlkv_token_logprobs), and the gradient of the logits
// (mlkv_token_logprobs_backward).
//
// With c = scale, m = max x, S = sum exp(c (x - m)), P = sum c (x - m) exp(c (x - m)):
//   log p_i = c (x_i - m) - log S,   H = log S - P / S
//   dx_i = c (g [i = t] - p_i (g + h (log p_i + H)))      (g, h: gradients of log p_t and H)
//
// Bound by HBM: the logits are read once (the backward pass reads and writes
// them once).  A block streams a row, or a span of one where rows are few (a
// second kernel joins the spans).  At 16 bits the stream is as near to the rate
// of instructions as to that of memory, so it is kept short: every thread has
// sums of its own against a reference of its own, which it moves only when a
// value is 2^8 above it (nothing is rescaled, no barrier), and the exponent is
// one fused multiply-add, c x - reference.  Values that far below that their
// exponential is 0 are raised to a floor first, so that -inf times 0 cannot be.
//
// The alternatives come out of the same stream.  Every thread knows the largest
// value it has seen, and in which batch first.  Of 32 disjoint parts of the
// block, take the k-th largest of the parts' largest values: a thread's batch
// whose largest value is below this bar holds none of the k best (nor one that
// equals it, in a later batch than those k).  The few batches that reach the bar
// (of a thread: about 30 while the values seen double, for k = 20) are listed in
// shared memory; at the end the block reads them again and sorts what of them
// reaches the last bar.  The bar is raised after 1, 3, 5, 9, 17 ... batches, by one
// warp and without a barrier but for the first time.
//
// 8,192 x 131,072 bf16 values with 20 alternatives: 398 us (5.4 TB/s; 17
// instructions a value), 2,048 rows without 86 (6.3; 9.5); one such row, 8 spans of a
// cluster, 11 us (latency: a stream of 2 batches, a sort of what was listed).  515
// x 50,001 fp32, 5 alternatives: 29 us.
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "dense_common.cuh"

using namespace mlkv;

namespace {

constexpr int kMostThreads = 256;
constexpr int kBatch = 4;              // 16-byte pieces a thread works on at a time ...
constexpr int kStages = 2;             // ... of a ring of so many batches
constexpr int kMostSpans = 64;         // of a row
constexpr int kListed = 8;             // batches, of a thread each, that the list has room for: so many a thread
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -200.f;       // 2^kLeast is 0 in fp32: what lies below (-inf too) need not be told apart

struct ProbArgs {
    const void* x;
    int64_t stride, n;
    const int64_t* targets;
    float scale;
    int32_t vocab, top, spans, per_span;  // 16-byte pieces of a span
    int32_t joined;               // a row's spans are a cluster, which joins them itself
    float* logprob;
    float* entropy;
    float* stats;
    float* top_logprobs;
    int64_t* top_ids;
    float4* part;                // [n][spans]: m, S, P of each
    unsigned long long* keys;    // [n][spans][top]
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
    template <int B> static __device__ __forceinline__ float most(const uint4 (&q)[B]) {
        float m = __uint_as_float(q[0].x);
#pragma unroll
        for (int i = 0; i < B; ++i) m = max2(max2(max2(m, __uint_as_float(q[i].x)), max2(__uint_as_float(q[i].y), __uint_as_float(q[i].z))), __uint_as_float(q[i].w));
        return m;
    }
    // The floor, as the exponent has it.
    struct Floor {};
    static __device__ __forceinline__ Floor floor_of(float, float) { return {}; }
    static __device__ __forceinline__ float2 raised(const uint4& q, int i, Floor) { return pair(q, i); }
    static __device__ __forceinline__ float2 clamp(float2 d) { return make_float2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast)); }
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
    template <int B> static __device__ __forceinline__ float most(const uint4 (&q)[B]) {
        __nv_bfloat162 m = as2(q[0].x);
#pragma unroll
        for (int i = 0; i < B; ++i) m = __hmax2_nan(__hmax2_nan(__hmax2_nan(m, as2(q[i].x)), __hmax2_nan(as2(q[i].y), as2(q[i].z))), as2(q[i].w));
        return __bfloat162float(__hmax_nan(m.x, m.y));
    }
    // The floor, on the values themselves, two at a time: so far below `at` that the exponential is 0, whatever
    // bf16 makes of it (its range is fp32's, so there is such a value).
    using Floor = __nv_bfloat162;
    static __device__ __forceinline__ Floor floor_of(float at, float c) {
        const __nv_bfloat16 v = __float2bfloat16_rd(at - fmaxf(-kLeast / c, fabsf(at) * 0x1p-6f));
        return __nv_bfloat162(v, v);
    }
    static __device__ __forceinline__ float2 raised(const uint4& q, int i, Floor f) {
        const __nv_bfloat162 v = __hmax2(as2(word(q, i)), f);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(&v);
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ float2 clamp(float2 d) { return d; }
};
template <> struct Piece<__half> {
    static constexpr int N = 8;
    static constexpr uint32_t kMinusInf = 0xFC00FC00u;
    static __device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
    static __device__ __forceinline__ __half2 as2(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
    static __device__ __forceinline__ float2 pair(const uint4& q, int i) { return __half22float2(as2(word(q, i))); }
    template <int B> static __device__ __forceinline__ float most(const uint4 (&q)[B]) {
        __half2 m = as2(q[0].x);
#pragma unroll
        for (int i = 0; i < B; ++i) m = __hmax2_nan(__hmax2_nan(__hmax2_nan(m, as2(q[i].x)), __hmax2_nan(as2(q[i].y), as2(q[i].z))), as2(q[i].w));
        return __half2float(__hmax_nan(m.x, m.y));
    }
    // The floor, as the exponent has it (fp16 need not have a value that low).
    struct Floor {};
    static __device__ __forceinline__ Floor floor_of(float, float) { return {}; }
    static __device__ __forceinline__ float2 raised(const uint4& q, int i, Floor) { return pair(q, i); }
    static __device__ __forceinline__ float2 clamp(float2 d) { return make_float2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast)); }
};

__device__ __forceinline__ float max_nan(float a, float b) { return Piece<float>::max2(a, b); }

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The scale of exponents of 2.  (Not infinite, whose product with 0 is not 0.)
__device__ __forceinline__ float of_log2(float scale) { return fminf(scale * kLog2e, 3.4028234663852886e38f); }

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
#pragma unroll 1
    for (int size = from; size <= 32; size <<= 1)
#pragma unroll 1
        for (int o = size >> 1; o; o >>= 1) {
            const K y = __shfl_xor_sync(0xffffffffu, x, o);
            const bool want_max = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
            x = want_max ? (x > y ? x : y) : (x < y ? x : y);
        }
    return x;
}
// The 32 largest of `count` keys, lane i holding the i-th (the warp).
__device__ __forceinline__ Key best_of(const Key* keys, int count, int lane) {
    Key best = 0;
    for (int b = 0; b < count; b += 32) {
        const Key k = sort_lanes<Key>(b + lane < count ? keys[b + lane] : 0ull, lane);
        const Key other = __shfl_sync(0xffffffffu, k, 31 - lane);
        best = sort_lanes<Key>(best > other ? best : other, lane, 32);
    }
    return best;
}
// Leaves the `top` best of list[0 .. count) in list[0 .. top), in order, 0 where
// there are fewer (the block, whose threads may just have written the list; keys
// are distinct).  Each warp cuts its share of a long list to 32; what is left is
// placed by counting the better ones.
template <int THREADS>
__device__ __noinline__ void select(Key* list, int count, int top) {
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (count > THREADS) {
        const int share = (count + kWarps - 1) / kWarps, from = warp * share;
        const Key k = best_of(list + from, max(0, min(share, count - from)), lane);
        __syncthreads();
        list[threadIdx.x] = k;
        count = THREADS;
        __syncthreads();
    }
    const Key mine = (int)threadIdx.x < count ? list[threadIdx.x] : 0;
    int rank = 0;
#pragma unroll 4
    for (int i = 0; i < count; ++i) rank += list[i] > mine;
    __syncthreads();
    if ((int)threadIdx.x < top) list[threadIdx.x] = 0;
    __syncthreads();
    if (mine && rank < top) list[rank] = mine;
    __syncthreads();
}

// A row's results from its sums (a warp; lane i with its i-th alternative).
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

// Sums of what a thread has seen: s = sum 2^(c x - at), p = sum (c x - at) 2^(c x - at).
struct Sums {
    float at, s, p;
    // Against a reference lower by d.
    __device__ __forceinline__ void move(float to, float d) {
        at = to;
        if (s == 0.f) return;  // of nothing that counts
        d = fmaxf(d, kLeast);
        const float e = exp2f(d);
        p = (p + d * s) * e;
        s *= e;
    }
};
// Whether c x - c max can be formed as c x - reference: neither overflows, and a
// floor lies below the maximum.  (Not with a row of nothing but the lowest fp32.)
__device__ __forceinline__ bool fused_ok(float most, float c) {
    return most == -CUDART_INF_F || (fabsf(most) <= 1e30f && fabsf(most) * c <= 1e30f && c <= 1e30f && c >= 1e-30f);
}

template <class T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprobs(ProbArgs a) {
    pdl_enter();
    using P = Piece<T>;
    constexpr uint32_t f = P::kMinusInf;
    constexpr int kWarps = THREADS / 32, kRoom = kListed * THREADS, kStep = kBatch * THREADS;
    extern __shared__ __align__(16) uint8_t shared[];  // the ring; then [kRoom] listed batches
    __shared__ float2 sums[kWarps];
    __shared__ Key parts[32];        // the parts' largest values, with the batch that has it first
    __shared__ volatile unsigned long long bar;  // (value, last batch), raised by one warp or another
    __shared__ int count, values;
    __shared__ __align__(16) float4 told;  // to the cluster
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint4* ring = reinterpret_cast<uint4*>(shared) + threadIdx.x;  // (a thread reads what it copied itself)
    int* listed = reinterpret_cast<int*>(shared + kStages * kStep * sizeof(uint4));
    Key* list = reinterpret_cast<Key*>(shared);  // at the end, where the ring was
    static_assert(kStages * kBatch * sizeof(uint4) >= (kListed + 2) * sizeof(Key), "the list fits the ring");
    const int64_t r = blockIdx.x / (unsigned)a.spans;
    const int span = (int)(blockIdx.x % (unsigned)a.spans);
    const RowPieces<T> row(a.x, r * a.stride, a.vocab);
    const int p0 = span * a.per_span, p1 = min(row.count, p0 + a.per_span);
    const float c = of_log2(a.scale);
    const float2 c2 = make_float2(c, c);
    auto fetch = [&](int base, int stage) {
        uint4* to = ring + stage * kStep;
        if (base > 0 && base + kStep <= min(p1, row.count - 1)) {
            const uint4* from = reinterpret_cast<const uint4*>(row.first) + base + threadIdx.x;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) copy_async<16>(to + i * THREADS, from + i * THREADS);
        } else {
#pragma unroll 1
            for (int i = 0; i < kBatch; ++i) {
                const int p = base + i * THREADS + (int)threadIdx.x;
                if (p < p1 && row.whole(p)) copy_async<16>(to + i * THREADS, reinterpret_cast<const uint4*>(row.first) + p);
                else to[i * THREADS] = p < p1 ? row.load(p) : make_uint4(f, f, f, f);
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(p0 + i * kStep, i);
    if (TOP && threadIdx.x == 0) {
        count = values = 0;
        bar = 0xFF7FFFFF7FFFFFFFull;  // everything
    }
    Sums sum = {0.f, 0.f, 0.f};
    typename P::Floor floor = P::floor_of(0.f, c);
    float most = -CUDART_INF_F;  // the largest value this thread has seen (NaN where there is one) ...
    int first = 0;               // ... and the first batch that holds it
    float least = 0.f;           // the bar: batches whose largest value is above this, or equal up to batch `last`
    int last = 0;
    auto tell = [&] {  // the best of this warp's parts
        Key mine = most == -CUDART_INF_F ? 0ull : key_of(most, first);
#pragma unroll
        for (int o = kWarps >> 1; o; o >>= 1) {
            const Key y = __shfl_xor_sync(0xffffffffu, mine, o);
            mine = mine > y ? mine : y;
        }
        if (lane % kWarps == 0) *const_cast<volatile Key*>(&parts[warp * (32 / kWarps) + lane / kWarps]) = mine;
    };
    // The bar of what the parts have told (a warp): of the k-th largest value the last batch that has it.  What
    // other warps have seen since, or tell meanwhile, makes the bar lower than it could be, and as good.
    auto raise = [&] {
        const Key mine = *const_cast<volatile Key*>(&parts[lane]);
        const uint32_t value = (uint32_t)(mine >> 32);
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < 32; ++i) above += __shfl_sync(0xffffffffu, value, i) > value;
        const uint32_t kth = __reduce_min_sync(0xffffffffu, above < a.top ? value : 0xFFFFFFFFu);
        const uint32_t batch = __reduce_min_sync(0xffffffffu, value == kth ? (uint32_t)mine : 0xFFFFFFFFu);
        least = kth ? value_of(kth) : -3.4028234663852886e38f;  // (0: fewer parts with a value than k)
        last = kth ? (int)(0xFFFFFFFEu - batch) : 0x7FFFFFFF;
        return __reduce_max_sync(0xffffffffu, value);
    };
    int batch = 0, stage = 0;
    for (int base = p0; base < p1; base += kStep, ++batch) {
        fetch(base + (kStages - 1) * kStep, stage == 0 ? kStages - 1 : stage - 1);
        copy_wait<kStages - 1>();
        uint4 q[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) q[i] = ring[stage * kStep + i * THREADS];
        stage = stage == kStages - 1 ? 0 : stage + 1;
        const float now = P::most(q);
        if (now > most) first = batch;
        most = max_nan(most, now);
        if (TOP) {
            if ((batch & (batch - 1)) == 0) {
                tell();
                if (batch == 0) {
                    __syncthreads();
                    raise();
                }
            } else if ((batch & (batch - 2)) == 1 && warp == __popc(batch) % kWarps) {
                raise();  // (a batch later, when the other warps have told too, as a rule)
                if (lane == 0) bar = (unsigned long long)__float_as_uint(least) << 32 | (uint32_t)last;
            } else {
                const unsigned long long told = bar;
                const float value = __uint_as_float((uint32_t)(told >> 32));
                const int since = (int)(uint32_t)told;
                if (value > least || (value == least && since < last)) least = value, last = since;
            }
            if (now >= least && (now > least || batch <= last)) {
                const int to = atomicAdd(&count, 1);
                if (to < kRoom) listed[to] = base + (int)threadIdx.x;
            }
        }
        const float to = now * c;
        if (to - sum.at > 8.f || (sum.s == 0.f && to > -1e30f)) {  // (what is lower counts nothing against 0 either)
            sum.move(to, sum.at - to);
            floor = P::floor_of(now, c);
        }
        const float2 minus = make_float2(-sum.at, -sum.at);
        float2 s2 = make_float2(sum.s, 0.f), t2 = make_float2(sum.p, 0.f);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int k = 0; k < P::N / 2; ++k) {
                const float2 d = P::clamp(fma2(P::raised(q[i], k, floor), c2, minus));
                const float2 e = make_float2(exp2_fast(d.x), exp2_fast(d.y));
                s2 = add2(s2, e);
                t2 = fma2(d, e, t2);
            }
        sum.s = s2.x + s2.y;
        sum.p = t2.x + t2.y;
    }
    copy_wait<0>();
    // the block's largest value, and its sums against it
    tell();
    __syncthreads();
    {
        const uint32_t top = TOP ? raise() : __reduce_max_sync(0xffffffffu, (uint32_t)(parts[lane] >> 32));
        most = top ? value_of(top) : -CUDART_INF_F;
    }
    if (fused_ok(most, c)) {
        sum.move(0.f, most == -CUDART_INF_F ? 0.f : fmaf(-most, c, sum.at));
    } else {
        sum.s = sum.p = 0.f;
        for (int p = p0 + (int)threadIdx.x; p < p1; p += THREADS) {
            const uint4 w = row.load(p);
#pragma unroll 1
            for (int e = 0; e < P::N / 2; ++e) {
                const float2 x = P::pair(w, e);
                const float d0 = fmaxf((x.x - most) * c, kLeast), d1 = fmaxf((x.y - most) * c, kLeast);
                sum.s += exp2_fast(d0) + exp2_fast(d1);
                sum.p += d0 * exp2_fast(d0) + d1 * exp2_fast(d1);
            }
        }
    }
    const float s = group_sum(sum.s, 32), t = group_sum(sum.p, 32);
    if (lane == 0) sums[warp] = make_float2(s, t);
    if (TOP) {
        if (count <= kRoom && !isnan(most)) {
            // the listed batches' pieces, a thread one at a time; what reaches the bar is cut to the k best when
            // there is much of it
            const int n = count * kBatch;
            Key least_key = 0;
            for (int i0 = 0; i0 < n; i0 += THREADS) {
                const int i = i0 + (int)threadIdx.x, p = i < n ? listed[i / kBatch] + (i % kBatch) * THREADS : p1;
                if (p < p1) {
                    const int at = row.index(p);
                    const uint4 w = row.load(p);
#pragma unroll
                    for (int e = 0; e < P::N; ++e) {
                        const float2 two = P::pair(w, e / 2);
                        const float x = e & 1 ? two.y : two.x;
                        if (!(x >= least)) continue;
                        const Key key = key_of(x, at + e);
                        if (key > least_key) list[atomicAdd(&values, 1)] = key;
                    }
                }
                __syncthreads();
                const int have = values;
                __syncthreads();
                if (have > THREADS) {
                    select<THREADS>(list, have, a.top);
                    least_key = list[a.top - 1];
                    if (threadIdx.x == 0) values = a.top;
                    __syncthreads();
                }
            }
            select<THREADS>(list, values, a.top);
        } else {
            // The list ran over, or NaN is among the values: one alternative after another, from the row itself, of
            // which the thread that held the last one reads its share again while the others wait.  (Scores that rise
            // along the row get here: 8,192 x 50,000 bf16, 20 alternatives, 194 us of random ones, 3,523 of sorted
            // rows, 5,026 with a NaN in each.)
            Key mine = 0, below = ~0ull;
            bool look = true;
            __syncthreads();
            for (int k = 0; k < a.top; ++k) {
                if (look) {
                    mine = 0;
                    for (int p = p0 + (int)threadIdx.x; p < p1; p += THREADS) {
                        const uint4 w = row.load(p);
                        const int at = row.index(p);
#pragma unroll 1
                        for (int e = 0; e < P::N / 2; ++e) {
                            const float2 x = P::pair(w, e);
                            const Key k0 = key_of(x.x, at + 2 * e), k1 = key_of(x.y, at + 2 * e + 1);
                            if (x.x != -CUDART_INF_F && k0 < below && k0 > mine) mine = k0;
                            if (x.y != -CUDART_INF_F && k1 < below && k1 > mine) mine = k1;
                        }
                    }
                }
                Key b = mine;
                for (int o = 16; o; o >>= 1) {
                    const Key y = __shfl_xor_sync(0xffffffffu, b, o);
                    b = b > y ? b : y;
                }
                if (lane == 0) parts[8 * (k & 1) + warp] = b;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) {
                    const Key y = parts[8 * (k & 1) + w];
                    b = b > y ? b : y;
                }
                if (threadIdx.x == 0) list[k] = b;
                look = b == mine;
                below = b;
            }
            __syncthreads();
        }
    } else {
        __syncthreads();
    }
    if (warp == 0) {
        const float2 w = lane < kWarps ? sums[lane] : make_float2(0.f, 0.f);
        sum.s = group_sum(w.x, 32);
        sum.p = group_sum(w.y, 32);
        const Key mine = TOP && lane < a.top ? list[lane] : 0ull;
        if (a.spans == 1) {
            finish_row<T>(a, r, most, sum.s, sum.p, mine, lane);
        } else if (a.joined) {
            if (lane == 0) told = make_float4(most, sum.s, sum.p, 0.f);
            if (TOP) parts[lane] = mine;
        } else {
            if (lane == 0) a.part[blockIdx.x] = make_float4(most, sum.s, sum.p, 0.f);
            if (TOP && lane < a.top) a.keys[(int64_t)blockIdx.x * a.top + lane] = mine;
        }
    }
    if (!a.joined) return;
    cluster_sync();
    if (span == 0) {  // the cluster's first block: what the others have told
        if (TOP) {
            for (int i = threadIdx.x; i < a.spans * a.top; i += THREADS)
                asm volatile("ld.shared::cluster.b64 %0, [%1];" : "=l"(list[i]) : "r"(place_in(smem_of(&parts[i % a.top]), i / a.top)) : "memory");
            select<THREADS>(list, a.spans * a.top, a.top);
        }
        if (warp == 0) {
            float4 its = make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
            if (lane < a.spans)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(its.x), "=f"(its.y), "=f"(its.z), "=f"(its.w)
                             : "r"(place_in(smem_of(&told), lane))
                             : "memory");
            float m = its.x;
            for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            Sums one = {0.f, its.y, its.z};
            if (its.x != -CUDART_INF_F) one.move(0.f, (its.x - m) * c);
            const float s = group_sum(one.s, 32), p = group_sum(one.p, 32);
            finish_row<T>(a, r, m, s, p, TOP && lane < a.top ? list[lane] : 0ull, lane);
        }
    }
    cluster_sync();  // (nothing of a block's memory is wanted by another any more)
}

// A row's spans joined (a block a row).
template <class T>
__global__ void __launch_bounds__(kMostThreads) k_logprobs_join(ProbArgs a) {
    pdl_enter();
    __shared__ Key list[kMostSpans * MLKV_MAX_TOP];
    __shared__ Key bars[kMostThreads / 32];
    __shared__ int count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r = blockIdx.x;
    const float4* part = a.part + r * a.spans;
    if (a.top) {
        // no alternative is below any span's last, and few others are not
        const Key* keys = a.keys + r * a.spans * a.top;
        Key bar = 0;
        for (int i = threadIdx.x; i < a.spans; i += kMostThreads) bar = max(bar, keys[i * a.top + a.top - 1]);
        for (int o = 16; o; o >>= 1) bar = max(bar, __shfl_xor_sync(0xffffffffu, bar, o));
        if (lane == 0) bars[warp] = bar;
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        for (int w = 0; w < kMostThreads / 32; ++w) bar = max(bar, bars[w]);
        for (int i = threadIdx.x; i < a.spans * a.top; i += kMostThreads) {
            const Key k = keys[i];
            if (k && k >= bar) list[atomicAdd(&count, 1)] = k;
        }
        __syncthreads();
        select<kMostThreads>(list, count, a.top);
    }
    if (warp != 0) return;
    const float c = of_log2(a.scale);
    float m = -CUDART_INF_F;
    for (int i = lane; i < a.spans; i += 32) m = max_nan(m, part[i].x);
    for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = 0.f, t = 0.f;
    for (int i = lane; i < a.spans; i += 32) {
        const float4 q = part[i];
        Sums one = {0.f, q.y, q.z};
        if (q.x != -CUDART_INF_F) one.move(0.f, (q.x - m) * c);
        s += one.s;
        t += one.p;
    }
    s = group_sum(s, 32);
    t = group_sum(t, 32);
    finish_row<T>(a, r, m, s, t, a.top && lane < a.top ? list[lane] : 0ull, lane);
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

// Every piece once in and once out, all of a block's loads on their way at once: 8,192 x 131,072 bf16 values 608 us,
// 7.1 TB/s (a plain copy: 6.8); 16,384 x 15,000 fp16 157, 6.3.
template <class T, int NV>
__global__ void __launch_bounds__(kMostThreads, 4) k_logprobs_backward(GradArgs a) {
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
    // dx = p (A + B u) with u = log2 p, and scale g more at the target.  A scale so large that A and B would not be
    // finite comes last (of what is often 0 then).
    const bool large = a.scale > 0x1p64f;
    const float c = of_log2(a.scale), base = m == -CUDART_INF_F ? 0.f : m, by = large ? 1.f : a.scale;
    float A = -by * (g + (h != 0.f ? h * a.entropy[r] : 0.f));
    const float B = -by * h * kLn2, at_target = by * g;
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
        if (large)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] *= a.scale;
        if (aligned && row.whole(p)) {
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float4*>(out + (int64_t)p * N) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                *reinterpret_cast<uint4*>(out + (int64_t)p * N) =
                    make_uint4(pack2<T>(make_float2(v[0], v[1])), pack2<T>(make_float2(v[2], v[3])),
                               pack2<T>(make_float2(v[N - 4], v[N - 3])), pack2<T>(make_float2(v[N - 2], v[N - 1])));
            }
        } else {  // (of rows that lie otherwise than the logits' a value at a time: 8,192 x 50,001 bf16 out of rows 5 wider
                  // 956 us, 8 wider 264)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at + e >= 0 && at + e < a.vocab) out[(int64_t)p * N + e] = from_float<T>(v[e]);
        }
    }
}

struct Split {
    int threads, NV, parts, per_part;
    bool joined;
};

// 16-byte pieces of the longest row: one more where rows may begin within one.
int64_t pieces_of(int64_t vocab, int size, bool aligned) { return (vocab * size + (aligned ? 15 : 30)) / 16; }
bool pieces_aligned(const void* p, int64_t stride, int size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0;
}

// The forward pass: threads a block, and spans a row.  As many blocks run at a
// time as hold 1,024 threads an SM; the spans are what makes the last of these
// waves end soonest, a block costing about 1,700 pieces beside its own (2.4 us
// of latencies at 1.4 ns a piece).
// Threads a block: as few as give a thread no more than 16 pieces, or, where rows
// are many, as few as still make 4 waves: what a block does besides streaming
// (its first loads, the sums over it, the alternatives' sort) is then done by fewer
// warps, beside more blocks that stream.  (At most 8 to 16 pieces a thread / this,
// us: 16,384 x 15,000 fp16 91 / 81; 15,000 x 8,000 bf16, 5 alternatives, 104 / 82;
// 16,384 x 50,000 bf16 263 / 233; 8,192 x 50,000, 20 alternatives, 233 / 193; 3 waves
// instead: 8,192 x 131,072, 20 alternatives, 497, 398 with 4.)
constexpr int64_t kWaves = 4;
Split spans_of(int64_t n, int64_t pieces, int sms) {
    int threads = kMostThreads;
    for (int t = 32; t < kMostThreads; t *= 2)
        if (pieces <= (int64_t)t * 16 || (n >= kWaves * sms * (1024 / t) && pieces <= (int64_t)t * 256)) {
            threads = t;
            break;
        }
    const int64_t wave = (int64_t)sms * (1024 / threads);
    // Few rows: up to 8 spans of at least 256 pieces, a cluster, which saves a launch; where they stay short
    // beside the time that takes.
    if (n * 8 <= wave && pieces >= 512 && pieces <= 8 * 8192) {
        const int64_t s = std::min<int64_t>(8, pieces / 256);
        return {threads, 0, (int)s, (int)((pieces + s - 1) / s), true};
    }
    int64_t best = 1, cost = INT64_MAX;
    for (int64_t s = 1; s <= kMostSpans && (s == 1 || pieces / s >= 256); ++s) {
        const int64_t now = (n * s + wave - 1) / wave * (pieces / s + 1700);
        if (now < cost) cost = now, best = s;
        if (n > 4 * wave) break;
    }
    return {threads, 0, (int)best, (int)((pieces + best - 1) / best), false};
}

// The backward pass: a block holds what it loads at once, up to 8 pieces a thread.
Split parts_of(int64_t n, int64_t pieces, int sms) {
    for (int t = 32; t <= kMostThreads; t *= 2)
        for (int nv = 1; nv <= 4; nv *= 2)
            if (pieces <= (int64_t)t * nv) return {t, nv, 1, (int)pieces, false};
    int nv = 8;
    while (nv > 2 && n * ((pieces + kMostThreads * nv - 1) / (kMostThreads * nv)) < 2 * sms) nv /= 2;
    const int64_t parts = (pieces + kMostThreads * nv - 1) / (kMostThreads * nv);
    return {kMostThreads, nv, (int)parts, (int)((pieces + parts - 1) / parts), false};
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

template <class F>
void by_threads(int threads, F f) {
    if (threads == 32) f(Int<32>{});
    else if (threads == 64) f(Int<64>{});
    else if (threads == 128) f(Int<128>{});
    else f(Int<256>{});
}

bool probs_ok(int64_t n, int64_t vocab, int32_t type, float scale) {
    return n >= 0 && n < (int64_t)1 << 31 && vocab >= 1 && vocab < (int64_t)1 << 30 && dense_type_ok(type) && scale > 0.f && std::isfinite(scale);
}

// Blocks of a launch, at most 2^31 - 1 of them.
bool grid_ok(int64_t n, const Split& s) { return n * s.parts < (int64_t)1 << 31; }

}  // namespace

extern "C" int64_t mlkv_token_logprobs_workspace(int64_t n, int64_t vocab, int32_t type, int32_t top) {
    if (!probs_ok(n, vocab, type, 1.f) || top < 0 || top > MLKV_MAX_TOP) return -1;
    if (n == 0) return 0;
    const int sms = dense_sms();
    if (!sms) return -1;
    int64_t most = 0;  // wherever the rows begin
    for (bool aligned : {false, true}) {
        const Split s = spans_of(n, pieces_of(vocab, dense_type_size(type), aligned), sms);
        if (s.parts > 1 && !s.joined) most = std::max(most, n * s.parts * (16 + 8 * (int64_t)top));
    }
    return most;
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
    const int size = dense_type_size(type);
    const Split s = spans_of(n, pieces_of(vocab, size, pieces_aligned(d_logits, stride, size)), sms);
    if (!grid_ok(n, s)) return MLKV_ERR_UNSUPPORTED;
    if (!workspace_ok(d_workspace, workspace_bytes, s.parts > 1 && !s.joined ? n * s.parts * (16 + 8 * (int64_t)top) : 0)) return MLKV_ERR_INVALID;
    ProbArgs a = {};
    a.x = d_logits; a.stride = stride; a.n = n; a.targets = d_targets; a.scale = scale; a.vocab = (int32_t)vocab;
    a.top = top; a.spans = s.parts; a.per_span = s.per_part; a.joined = s.joined; a.logprob = d_logprob; a.entropy = d_entropy;
    a.stats = d_stats; a.top_logprobs = d_top_logprobs; a.top_ids = d_top_ids;
    a.part = static_cast<float4*>(d_workspace);
    a.keys = reinterpret_cast<Key*>(a.part + n * s.parts);
    cudaStream_t st = (cudaStream_t)stream;
    bool ok = true;
    by_type(type, [&](auto t) {
        using T = decltype(t);
        const dim3 grid((unsigned)(n * s.parts)), block(s.threads);
        auto launch = [&](auto kernel, bool listed) {
            const size_t bytes = (size_t)s.threads * (kStages * kBatch * sizeof(uint4) + (listed ? kListed * sizeof(int) : 0));
            ok = dense_smem(kernel, bytes);
            if (!ok) return;
            if (s.joined) launch_clusters(kernel, s.parts, n * s.parts, s.threads, bytes, st, a);
            else launch_kernel(true, kernel, grid, block, bytes, st, a);
        };
        by_threads(s.threads, [&](auto n) {
            constexpr int N = decltype(n)::value;
            if (top) launch(k_logprobs<T, true, N>, true);
            else launch(k_logprobs<T, false, N>, false);
        });
        if (ok && s.parts > 1 && !s.joined) launch_kernel(true, k_logprobs_join<T>, dim3((unsigned)n), dim3(kMostThreads), 0, st, a);
    });
    return ok && cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
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
    const int size = dense_type_size(type);
    const Split s = parts_of(n, pieces_of(vocab, size, pieces_aligned(d_logits, stride, size)), sms);
    if (!grid_ok(n, s)) return MLKV_ERR_UNSUPPORTED;
    GradArgs a = {};
    a.x = d_logits; a.dx = d_dlogits; a.stride = stride; a.dx_stride = dlogits_stride; a.targets = d_targets;
    a.entropy = d_entropy; a.stats = d_stats; a.dlogprob = d_dlogprob; a.dentropy = d_dentropy; a.scale = scale;
    a.vocab = (int32_t)vocab; a.chunks = s.parts; a.per_chunk = s.per_part;
    cudaStream_t st = (cudaStream_t)stream;
    by_type(type, [&](auto t) {
        using T = decltype(t);
        by_pieces(s.NV, [&](auto nv) {
            launch_kernel(true, k_logprobs_backward<T, decltype(nv)::value>, dim3((unsigned)(n * s.parts)), dim3(s.threads), 0, st, a);
        });
    });
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}
