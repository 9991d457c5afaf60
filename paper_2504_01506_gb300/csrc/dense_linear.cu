// The matrix product with bias, activation and residual, and its gradients
// (mlkv_linear, mlkv_linear_backward).
//
//   forward   y = act(x W^T + b) + r
//   backward  p = dy act'(z),  dx = p W,  dW = p^T x,  db = column sums of p
//
// All three products are D[i][j] = sum_k A[i][k] B[j][k] for operands whose rows
// in memory run along k, or along i or j (dx: W's; dW: both), which the matrix
// unit takes as they lie.  One kernel computes them (k_product): TMA brings
// tiles into a ring in shared memory, one thread issues tcgen05.mma into one of
// two accumulators in tensor memory, and 4 to 16 warps take the other one out
// through the epilogue, whose blocks leave by TMA too.
//
// Sums are fp32 all the way; what is rounded to 16 bits is z (`pre`, which the
// slopes are taken at, while y goes by z itself), y, p and the gradients, once each.
#include <cudaTypedefs.h>

#include <algorithm>

#include "dense_mma.cuh"

using namespace mlkv;

namespace {

constexpr int kBM = 128;      // rows (i) of a tile
constexpr int kBK = 64;       // values along k of a stage: 128 bytes

__device__ uint32_t g_timeouts;  // blocks in which a wait ran out (never set back: what has been told of is the host's)

struct Epilogue {
    const void* bias;
    const void* residual;
    void* pre;
    void* out;
    int64_t residual_stride, pre_stride, out_stride;
    int32_t type, act;
    int32_t wide;       // rows of out, pre and residual can be moved 16 bytes at a time
};

struct Product {
    int32_t I, J, blocks;            // extents; 64-value blocks along k
    int32_t tiles_i, tiles_j;
    int32_t whole;                   // tiles that are computed whole; of the others, in shares of k, ...
    int32_t shares, blocks_per_share;
    float* part;                     // ... the sums: [share][tile][rows of a tile][columns of a tile]
    int32_t joined;                  // a tile's shares are a cluster, which adds them up itself
    int32_t injected;                // (mlkv_debug_fail) no operands are brought
    int32_t beside;                  // needs nothing of the launch before it, which needs nothing of its outputs
    uint32_t idesc;
    // The operands (rows of k values), where sums near 0 are computed again (relu's): below `doubt` of the
    // largest beside them.
    const void *a, *b;
    int64_t a_stride, b_stride;
    int32_t k;
    float doubt;
    Epilogue e;
};

__device__ __forceinline__ float widen(int32_t type, uint16_t v) {
    return type == MLKV_TYPE_BFLOAT ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
}
__device__ __forceinline__ uint16_t narrow(int32_t type, float v) {
    return type == MLKV_TYPE_BFLOAT ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

// 1 / (1 + 2^u), two at a time, to a few units of 2^-22: what follows is rounded to 16 bits.
__device__ __forceinline__ float2 squash(float2 u) {
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(u.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(u.y));
    e = add2(e, make_float2(1.f, 1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return r;
}
__device__ __forceinline__ float2 splat2(float x) { return make_float2(x, x); }
__device__ __forceinline__ float at_least(float x, float least) {  // NaN stays NaN
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(least));
    return r;
}
__device__ __forceinline__ float at_most(float x, float most) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(most));
    return r;
}
// sigmoid(z) = squash(kSilu z);  (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 = squash(z (kGelu + kGelu3 z^2))
constexpr float kLog2e = 1.4426950408889634f, kSilu = -kLog2e, kGeluSlope = 1.5957691216057308f, kCube = 0.044715f;
constexpr float kGelu = -kLog2e * kGeluSlope, kGelu3 = kGelu * kCube;
// Of two values.  (Far below 0 the value is 0, not the product of -inf and 0.)
template <int ACT>
__device__ __forceinline__ float2 activate(float2 z) {
    if (ACT == MLKV_ACT_NONE) return z;
    if (ACT == MLKV_ACT_RELU) return make_float2(at_least(z.x, 0.f), at_least(z.y, 0.f));
    const float2 low = make_float2(at_least(z.x, -1e4f), at_least(z.y, -1e4f));
    if (ACT == MLKV_ACT_SILU) return mul2(low, squash(mul2(low, splat2(kSilu))));
    return mul2(low, squash(mul2(low, fma2(mul2(low, low), splat2(kGelu3), splat2(kGelu)))));
}
// The slope there.  (Far from 0 it is 0 or 1, not a product with an infinite factor.)
template <int ACT>
__device__ __forceinline__ float2 slope(float2 z) {
    if (ACT == MLKV_ACT_NONE) return splat2(1.f);
    if (ACT == MLKV_ACT_RELU) return make_float2(z.x > 0.f ? 1.f : z.x != z.x ? z.x : 0.f, z.y > 0.f ? 1.f : z.y != z.y ? z.y : 0.f);
    z = make_float2(at_most(at_least(z.x, -100.f), 100.f), at_most(at_least(z.y, -100.f), 100.f));
    const float2 one = splat2(1.f), z2 = mul2(z, z);
    // q + z q (1 - q) u', u the argument of the sigmoid
    const float2 q = squash(ACT == MLKV_ACT_SILU ? mul2(z, splat2(kSilu)) : mul2(z, fma2(z2, splat2(kGelu3), splat2(kGelu))));
    const float2 rest = mul2(mul2(z, q), fma2(q, splat2(-1.f), one));
    return ACT == MLKV_ACT_SILU ? add2(rest, q) : fma2(rest, fma2(z2, splat2(3.f * kGeluSlope * kCube), splat2(kGeluSlope)), q);
}
template <int N> struct Act { static constexpr int value = N; };
template <class F>
__device__ __forceinline__ void by_act(int32_t act, F f) {
    if (act == MLKV_ACT_RELU) f(Act<MLKV_ACT_RELU>{});
    else if (act == MLKV_ACT_GELU_TANH) f(Act<MLKV_ACT_GELU_TANH>{});
    else if (act == MLKV_ACT_SILU) f(Act<MLKV_ACT_SILU>{});
}

// What becomes of the sum at (row, col) of the output.
__device__ __forceinline__ float finish(const Epilogue& e, float v, int64_t row, int64_t col) {
    if (e.bias) v += widen(e.type, static_cast<const uint16_t*>(e.bias)[col]);
    if (e.pre) static_cast<uint16_t*>(e.pre)[row * e.pre_stride + col] = narrow(e.type, v);
    by_act(e.act, [&](auto act) { v = activate<decltype(act)::value>(splat2(v)).x; });
    if (e.residual) v += widen(e.type, static_cast<const uint16_t*>(e.residual)[row * e.residual_stride + col]);
    return v;
}

// A tile: groups of 8 tiles along i by all along j, so that tiles that run at the same time share operands in L2.
__device__ __forceinline__ void tile_at(const Product& p, int t, int& i, int& j) {
    const int group = t / (8 * p.tiles_j), first = group * 8, size = min(8, p.tiles_i - first);
    t -= group * 8 * p.tiles_j;
    i = first + t % size;
    j = t / size;
}
// What a block does t-th: a tile, or a share of one.
struct Work {
    int i, j, share, k0, k1;
    int64_t part;  // which of the tiles' shares
    __device__ __forceinline__ Work(const Product& p, int t, bool joined, int mine) {
        share = joined ? mine : 0;
        part = -1;
        if (!joined && t >= p.whole) {
            const int rest = p.tiles_i * p.tiles_j - p.whole;
            part = t - p.whole;
            share = (t - p.whole) / rest;
            t = p.whole + (t - p.whole) % rest;
        }
        tile_at(p, t, i, j);
        k0 = joined || part >= 0 ? share * p.blocks_per_share : 0;
        k1 = joined || part >= 0 ? min(p.blocks, k0 + p.blocks_per_share) : p.blocks;
    }
};

// 16 sums of a tile whose rows run along the output's columns: this lane's
// column i of the output, from row j0 on.  A warp writes 32 columns of a row at a time.
template <class T>
__device__ __forceinline__ void put_columns(const Product& p, const uint32_t (&r)[16], int64_t i, int64_t j0) {
    const Epilogue& e = p.e;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        if (j0 + q >= p.J) break;
        static_cast<T*>(e.out)[(j0 + q) * e.out_stride + i] = from_float<T>(finish(e, __uint_as_float(r[q]), j0 + q, i));
    }
}

// Four sums of one row of the output, from col on, through the epilogue.
template <class T>
__device__ __forceinline__ void put_four(const Epilogue& e, const float4& sum, int64_t row, int64_t col, int64_t cols) {
    if (e.wide && col + 4 <= cols) {
        float2 v[2] = {make_float2(sum.x, sum.y), make_float2(sum.z, sum.w)};
        uint2 x = make_uint2(0, 0);
        if (e.residual) x = *reinterpret_cast<const uint2*>(static_cast<const T*>(e.residual) + row * e.residual_stride + col);
        if (e.bias) {
            const T* b = static_cast<const T*>(e.bias) + col;
            v[0] = add2(v[0], make_float2(to_float(b[0]), to_float(b[1])));
            v[1] = add2(v[1], make_float2(to_float(b[2]), to_float(b[3])));
        }
        if (e.pre)
            *reinterpret_cast<uint2*>(static_cast<T*>(e.pre) + row * e.pre_stride + col) = make_uint2(word_of_pair<T>(v[0]), word_of_pair<T>(v[1]));
        by_act(e.act, [&](auto act) {
            v[0] = activate<decltype(act)::value>(v[0]);
            v[1] = activate<decltype(act)::value>(v[1]);
        });
        if (e.residual) {
            v[0] = add2(v[0], pair_of_word<T>(x.x));
            v[1] = add2(v[1], pair_of_word<T>(x.y));
        }
        *reinterpret_cast<uint2*>(static_cast<T*>(e.out) + row * e.out_stride + col) = make_uint2(word_of_pair<T>(v[0]), word_of_pair<T>(v[1]));
        return;
    }
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (col + k < cols) static_cast<T*>(e.out)[row * e.out_stride + col + k] = from_float<T>(finish(e, v[k], row, col + k));
}

// The shares of a tile whose rows run along the output's columns, [column j][128
// rows i] of sums at `at` in the shared memory of each block of the cluster, added
// up in order: this block's part of the rows, four of one column a thread (of 128) at a time.
template <class T, int BN>
__device__ __forceinline__ void join_columns(const Product& p, uint32_t at, int i, int j, uint32_t rank) {
    const int rows = kBM / p.shares / 4, columns = min(BN, p.J - j * BN);
    for (int q = threadIdx.x; q < rows * columns; q += 128) {
        const int c = q / rows, r = ((int)rank * rows + q % rows) * 4;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < p.shares; ++s) {
            float4 x;
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                         : "r"(place_in(at + (c * kBM + r) * 4, s))
                         : "memory");
            sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
        }
        put_four<T>(p.e, sum, (int64_t)j * BN + c, (int64_t)i * kBM + r, p.I);
    }
}

// A warp's corner of shared memory: two halves of 32 rows by 32 values (64 bytes a
// row, 16-byte pieces in the 64-byte swizzle: piece c of a row at c ^ (row / 2 & 3)),
// or 32 rows by 32 sums (128 bytes a row, piece c at c ^ (row & 7)).  The lane that
// has a row writes and reads it here without bank conflicts, TMA or, for rows that
// it does not take, the lanes side by side move it to memory and from it.
struct Half {
    uint8_t* at;
    __device__ __forceinline__ uint4& piece(int row, int c) const { return *reinterpret_cast<uint4*>(at + row * 64 + ((c ^ (row >> 1 & 3)) << 4)); }
    __device__ __forceinline__ uint16_t& value(int row, int c) const {
        return *reinterpret_cast<uint16_t*>(at + row * 64 + (((c >> 3) ^ (row >> 1 & 3)) << 4) + (c & 7) * 2);
    }
};
constexpr int kHalf = 2048, kCorner = 2 * kHalf, kBias = 128;

// A block of 32 rows by 32 columns of a matrix of 16-bit values.
struct Place {
    int r0, c0, rows, cols, lane;  // (from r0, c0 on; of the matrix)
    bool whole;                    // all its columns are there, and 16 bytes of a row can be moved at a time
};
template <class T>
__device__ __forceinline__ void put_values(Half s, T* m, int64_t stride, const Place& q) {
    if (q.c0 + q.lane >= q.cols) return;
    uint16_t* at = reinterpret_cast<uint16_t*>(m) + q.r0 * stride + q.c0 + q.lane;
    const int n = min(32, q.rows - q.r0);
#pragma unroll 8
    for (int r = 0; r < n; ++r, at += stride) *at = s.value(r, q.lane);
}
// A block of the residual: loaded ahead of its use, then put into a half.
template <class T>
struct Ahead {
    uint4 v[4];
    __device__ __forceinline__ void load(const T* m, int64_t stride, const Place& q) {
        if (!q.whole) return;
        const int row = q.r0 + (q.lane >> 2);
        const T* at = m + row * stride + q.c0 + (q.lane & 3) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row + i * 8 < q.rows) v[i] = *reinterpret_cast<const uint4*>(at + i * 8 * stride);
    }
    __device__ __forceinline__ void settle(Half s, const T* m, int64_t stride, const Place& q) const {
        if (q.whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s.piece(i * 8 + (q.lane >> 2), q.lane & 3) = v[i];
        } else if (q.c0 + q.lane < q.cols) {
            const uint16_t* at = reinterpret_cast<const uint16_t*>(m) + q.r0 * stride + q.c0 + q.lane;
            const int n = min(32, q.rows - q.r0);
#pragma unroll 8
            for (int r = 0; r < n; ++r, at += stride) s.value(r, q.lane) = *at;
        }
    }
};

// relu's slope jumps at 0, where the matrix unit's rounding (about 2^-24 of the
// sums on the way, every 16 values of k) decides it at random: one such value moves
// a whole row of dx.  So of a lane's 32 values the smallest, where it is that near
// 0, is computed again by the warp, in 64 bits.  (65,536 x 416 by 512: about 90 of
// 33.5 million.  Of sums that go out as shares, or of 64 rows or fewer, it is not:
// they are a few million at the most.  A column alone in its block of 32 has none
// to be small beside, and stays as it is.  A sum of exactly 0 beside others that
// are not always comes here, so that a weight row of zeros sends every row round:
// 304 us with one, 2,797 with one in each 32 columns, 37 without.)
template <class T>
__device__ __forceinline__ void doubtful(const Product& p, float2 (&v)[16], int r0, int c0, int lane) {
    const int columns = p.J - c0;  // (the sums past the last are 0)
    float least = INFINITY, most = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        least = fminf(least, fminf(2 * k < columns ? fabsf(v[k].x) : INFINITY, 2 * k + 1 < columns ? fabsf(v[k].y) : INFINITY));
        most = fmaxf(most, fmaxf(fabsf(v[k].x), fabsf(v[k].y)));
    }
    uint32_t again = __ballot_sync(0xffffffffu, r0 + lane < p.I && least < most * p.doubt && most < 1e30f);
    if (!again) return;
    int at = 32;  // this lane's smallest (the first one)
#pragma unroll
    for (int k = 15; k >= 0; --k) {
        if (fabsf(v[k].y) == least) at = 2 * k + 1;
        if (fabsf(v[k].x) == least) at = 2 * k;
    }
    for (; again; again &= again - 1) {
        const int from = __ffs(again) - 1, c = __shfl_sync(0xffffffffu, at, from), col = c0 + c;
        if (c == 32) continue;
        const T *a = static_cast<const T*>(p.a) + (r0 + from) * p.a_stride, *b = static_cast<const T*>(p.b) + col * p.b_stride;
        double sum = 0;
#pragma unroll 4
        for (int k = lane * 8; k + 8 <= p.k; k += 256) {  // (rows that TMA takes: on 16 bytes)
            const uint4 x = *reinterpret_cast<const uint4*>(a + k), y = *reinterpret_cast<const uint4*>(b + k);
            auto add = [&](uint32_t u, uint32_t w) {
                const float2 m = mul2(pair_of_word<T>(u), pair_of_word<T>(w));  // (exact)
                sum += (double)m.x + (double)m.y;
            };
            add(x.x, y.x);
            add(x.y, y.y);
            add(x.z, y.z);
            add(x.w, y.w);
        }
        if (lane < (p.k & 7)) sum += (double)to_float(a[(p.k & ~7) + lane]) * (double)to_float(b[(p.k & ~7) + lane]);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (p.e.bias) sum += (double)to_float(static_cast<const T*>(p.e.bias)[col]);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            if (lane == from && c == 2 * k) v[k].x = (float)sum;
            if (lane == from && c == 2 * k + 1) v[k].y = (float)sum;
        }
    }
}

// A warp's 32 rows of a tile's sums, from column c0 on, 32 columns at a time: out
// of tensor memory and through the epilogue.  `wait` returns when the sums are
// there; the residual's first block is on its way before that, each other while
// the one before it is worked on.  `part`: where the sums of a share go as they
// are, this warp's part of it (rows of `stride`).
template <class T, bool DOUBT, class W>
__device__ __forceinline__ bool put_blocks(const Product& p, const CUtensorMap* out_map, const CUtensorMap* pre_map, uint32_t tmem,
                                           uint8_t* corner, float* bias_at, int r0, int c0, int blocks, float* part, int stride, int lane,
                                           uint32_t& turn, W wait) {
    const Epilogue& e = p.e;
    const T* residual = part ? nullptr : static_cast<const T*>(e.residual);
    const bool biased = e.bias && !part;
    auto place = [&](int b) { return Place{r0, c0 + b * 32, p.I, p.J, lane, e.wide && c0 + b * 32 + 32 <= p.J}; };
    auto bias_of = [&](int b) {
        const int c = c0 + b * 32 + lane;
        return c < p.J ? to_float(static_cast<const T*>(e.bias)[c]) : 0.f;
    };
    Ahead<T> ahead;
    float bias = 0.f;
    if (biased) bias = bias_of(0);
    if (residual) ahead.load(residual, e.residual_stride, place(0));
    if (!wait()) return false;
    const bool two = e.pre || residual;  // both halves have a use of their own; else they take turns, from tile to tile
#pragma unroll 1
    for (int b = 0; b < blocks && c0 + b * 32 < p.J; ++b) {
        const Place q = place(b);
        uint32_t acc[32];
        __syncwarp();
        tmem_ld32(tmem + b * 32, acc);
        if (part) {  // (a corner's 4 KB as 32 rows of 128 bytes)
            if (b == 0) {  // what an earlier tile has left there is still on its way
                if (e.wide && lane == 0) tma_store_read<0>();
                __syncwarp();
            }
            tmem_wait_ld();
            auto sums = [&](int row, int c) -> uint4& { return *reinterpret_cast<uint4*>(corner + row * 128 + ((c ^ (row & 7)) << 4)); };
#pragma unroll
            for (int c = 0; c < 8; ++c) sums(lane, c) = make_uint4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
            __syncwarp();
            float* to = part + (lane >> 3) * stride + b * 32 + (lane & 7) * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(to + i * 4 * stride) = sums(i * 4 + (lane >> 3), lane & 7);
            continue;
        }
        if (biased) {
            bias_at[lane] = bias;
            if (b + 1 < blocks) bias = bias_of(b + 1);
        }
        __syncwarp();
        tmem_wait_ld();
        float2 v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = make_float2(__uint_as_float(acc[2 * k]), __uint_as_float(acc[2 * k + 1]));
        if (biased) {
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
                const float4 x = reinterpret_cast<const float4*>(bias_at)[k / 2];
                v[k] = add2(v[k], make_float2(x.x, x.y));
                v[k + 1] = add2(v[k + 1], make_float2(x.z, x.w));
            }
        }
        if (DOUBT && p.a) doubtful<T>(p, v, r0, q.c0, lane);
        // What a half holds goes to memory; whoever fills it next waits until it has been read.
        auto put = [&](Half s, const CUtensorMap* map, void* m, int64_t stride) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                s.piece(lane, c) = make_uint4(word_of_pair<T>(v[4 * c]), word_of_pair<T>(v[4 * c + 1]), word_of_pair<T>(v[4 * c + 2]), word_of_pair<T>(v[4 * c + 3]));
            if (e.wide) fence_async();
            __syncwarp();
            if (!e.wide) put_values(s, static_cast<T*>(m), stride, q);
            else if (lane == 0) tma_store(map, q.c0, q.r0, smem_of(s.at));
        };
        auto free_half = [&](bool all) {  // all stores have read theirs, or all but the last
            if (e.wide && lane == 0) {
                if (all) tma_store_read<0>();
                else tma_store_read<1>();
            }
            __syncwarp();
        };
        const Half first = {corner}, second = {corner + kHalf};
        if (e.pre) {
            free_half(false);
            put(first, pre_map, e.pre, e.pre_stride);
        }
        if (residual) {
            free_half(!e.pre);
            ahead.settle(second, residual, e.residual_stride, q);
            if (b + 1 < blocks) ahead.load(residual, e.residual_stride, place(b + 1));
        }
        by_act(e.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = activate<decltype(act)::value>(v[k]);
        });
        if (residual) {
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 x = second.piece(lane, c);
                v[4 * c] = add2(v[4 * c], pair_of_word<T>(x.x));
                v[4 * c + 1] = add2(v[4 * c + 1], pair_of_word<T>(x.y));
                v[4 * c + 2] = add2(v[4 * c + 2], pair_of_word<T>(x.z));
                v[4 * c + 3] = add2(v[4 * c + 3], pair_of_word<T>(x.w));
            }
            __syncwarp();
        } else {
            free_half(false);
        }
        put(two || (turn++ & 1) ? second : first, out_map, e.out, e.out_stride);
    }
    return true;
}

// The shared memory of a block: the ring of operand tiles, and a corner and 32
// bias values for every epilogue warp.
// A pair of blocks has a tile of 256 rows between them, and half of its columns' operand each.
template <int BN, bool SWAP, bool PAIR> struct Ring {
    // Epilogue warps.  A tile's sums take 8 warps 2.8 us to take out, 16 of them 2.1 (65,536 x 512 by k = 64: 21.3 and
    // 17.2 us): 16 where single blocks have short k, 8 where pairs have the shared memory in more stages.
    static constexpr int kEpilogue = SWAP || BN < 128 ? 4 : BN == 128 || PAIR ? 8 : 16;
    static constexpr int kThreads = (kEpilogue + 2) * 32;       // ... and the TMA warp, and the MMA warp
    static constexpr int kA = kBM * kBK * 2, kB = (PAIR ? BN / 2 : BN) * kBK * 2, kStage = kA + kB;
    static constexpr int kCorners = SWAP ? 0 : kEpilogue * (kCorner + kBias);
    static constexpr int kFit = (kDenseSmem - 1024 - kCorners) / kStage;
    static constexpr int kStages = kFit < 12 ? kFit : 12;
    static constexpr int kBytes = kStages * kStage + kCorners + 1024;  // (aligned to 1,024 within)
    static constexpr uint32_t kColumns = 2 * BN < 32 ? 32 : 2 * BN;
};

// Bound by the matrix unit where k is long: 16,384 x 4,096 by k = 4,096 (pairs) 284 us, 1.94 PFLOP/s, its pipe active
// 81 to 87% of the time.  By what L2 hands to the SMs (48 KB a block of k and tile) and the epilogue's bytes where k is
// short: 65,536 x 512 by 416, relu and pre 41 us, 189 MB of them to HBM at 4.6 TB/s.  By the weight's bytes where rows are few: one
// row by a weight of 4,096 x 4,096 8.3 us, 4.0 TB/s.
//
// A_MN, B_MN: the operand's rows run along i (j), not k.  SWAP: i runs along
// the output's columns (few rows: the weight is the operand of 128 rows a tile).
// PAIR: two blocks on neighbouring SMs share a tile of 256 rows.  Each holds its
// own 128 rows of A, half of B's and its rows' sums; the first issues the
// products of both, so that B crosses each SM's shared memory half as often.
template <int BN, bool A_MN, bool B_MN, bool SWAP, bool PAIR, class T>
__global__ void __launch_bounds__(Ring<BN, SWAP, PAIR>::kThreads, 1)
    k_product(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
              const __grid_constant__ CUtensorMap out_map, const __grid_constant__ CUtensorMap pre_map, const Product p) {
    using R = Ring<BN, SWAP, PAIR>;
    constexpr int S = R::kStages, kTma = R::kEpilogue, kMma = kTma + 1, kBlocks = PAIR ? 2 : 1, kCols = BN / kBlocks;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * S + 5];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    const uint32_t ring = (smem_of(raw) + 1023u) & ~1023u;
    const uint32_t full = smem_of(bars), empty = full + 8 * S, done = empty + 8 * S, drained = done + 16, ended = drained + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0;
    const bool joined = SWAP && p.joined;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(done + 8 * s, 1);
            mbar_init(drained + 8 * s, kBlocks * R::kEpilogue);
        }
        mbar_init(ended, 1);
        stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch(&ma);
        tma_prefetch(&mb);
    }
    if (warp == kMma) tmem_alloc<PAIR>(smem_of(&tmem_at), R::kColumns);
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    // Beside the product before it: by the time this is placed, that one's blocks have all seen what is before it
    // complete, and this reads by TMA alone (L1 holds nothing of it).
    if (p.beside) pdl_next();
    else pdl_enter();

    // joined shares: one tile a block, its share by its place in the cluster
    const int tiles = p.tiles_i * p.tiles_j, mine = joined ? (int)cluster_rank() : 0;
    const int total = joined ? tiles : p.whole + (tiles - p.whole) * p.shares, first = joined ? blockIdx.x / p.shares : blockIdx.x / kBlocks;
    const int step = joined ? tiles : gridDim.x / kBlocks;
    if (warp == kTma) {
        if (lane == 0 && !p.injected) {
            uint32_t n = 0;  // stages filled
            bool ok = true;
            for (int t = first; t < total && ok; t += step) {
                const Work w(p, t, joined, mine);
                const int row = (w.i * kBlocks + (int)rank) * kBM, col = w.j * BN + (int)rank * kCols;
                for (int k = w.k0; k < w.k1; ++k, ++n) {
                    const uint32_t s = n % S, at = ring + s * R::kStage;
                    if (n >= S && !(ok = mbar_wait(empty + 8 * s, (n / S - 1) & 1, &stop))) break;
                    if (rank == 0) mbar_expect(full + 8 * s, kBlocks * R::kStage);
                    const uint32_t bar = PAIR ? place_in(full + 8 * s, 0) : full + 8 * s;
                    auto load = [&](uint32_t to, const CUtensorMap* m, int x, int y) {
                        if (PAIR) tma_load_pair(to, m, x, y, bar);
                        else tma_load(to, m, x, y, bar);
                    };
                    if (A_MN)
                        for (int b = 0; b < kBM / 64; ++b) load(at + b * 8192, &ma, row + b * 64, k * kBK);
                    else
                        load(at, &ma, k * kBK, row);
                    if (B_MN)
                        for (int b = 0; b < kCols / 64; ++b) load(at + R::kA + b * 8192, &mb, col + b * 64, k * kBK);
                    else
                        load(at + R::kA, &mb, k * kBK, col);
                }
            }
            // (all have been brought: until the last has been read, the products may give up)
            if (ok && n) ok = mbar_wait(empty + 8 * ((n - 1) % S), ((n - 1) / S) & 1, &stop);
            if (!ok && rank == 0) {  // given up: the copies in flight still write into shared memory
                Waited waited;
                for (uint32_t b = n > S ? n - S : 0; b < n; ++b) mbar_drain(full + 8 * (b % S), (b / S) & 1, waited);
            }
        }
    } else if (warp == kMma) {
        if (lane == 0 && rank == 0) {
            uint32_t n = 0, u = 0;  // stages read, accumulators used
            bool ok = true;
            for (int t = first; t < total && ok; t += step, ++u) {
                const Work w(p, t, joined, mine);
                const uint32_t acc = u & 1, d = tmem + acc * BN;
                if (u >= 2 && !(ok = mbar_wait(drained + 8 * acc, (u / 2 - 1) & 1, &stop))) break;
                tc_fence_after();
                for (int k = w.k0; k < w.k1; ++k, ++n) {
                    const uint32_t s = n % S, at = ring + s * R::kStage;
                    if (!(ok = mbar_wait(full + 8 * s, (n / S) & 1, &stop))) break;
                    tc_fence_after();
                    const uint64_t da = smem_desc(at, A_MN ? 8192 : 16), db = smem_desc(at + R::kA, B_MN ? 8192 : 16);
#pragma unroll
                    for (int q = 0; q < kBK / 16; ++q)  // 16 values along k: 32 bytes of a row, or 16 rows
                        tc_mma<PAIR>(d, da + q * (A_MN ? 128 : 2), db + q * (B_MN ? 128 : 2), p.idesc, k > w.k0 || q > 0);
                    tc_commit<PAIR>(empty + 8 * s);
                }
                if (ok) tc_commit<PAIR>(done + 8 * acc);
            }
            if (!ok) {  // given up: products in flight still write into tensor memory
                tc_commit<PAIR>(ended);
                Waited waited;
                mbar_drain(ended, 0, waited);
            }
        }
    } else {
        uint32_t u = 0, turn = 0;
        const uint32_t told = PAIR ? place_in(drained, 0) : drained;
        for (int t = first; t < total; t += step, ++u) {
            const Work w(p, t, joined, mine);
            const uint32_t acc = u & 1, at = tmem + acc * BN + ((uint32_t)(warp & 3) << 21);
            auto wait = [&] {
                const bool ok = __all_sync(0xffffffffu, mbar_wait(done + 8 * acc, (u / 2) & 1, &stop));
                tc_fence_after();
                return ok;
            };
            const int in_tile = (int)rank * kBM + (warp & 3) * 32, r0 = w.i * kBlocks * kBM + in_tile;
            if constexpr (SWAP) {
                if (!wait()) break;
#pragma unroll 1
                for (int c = 0; c < BN; c += 16) {
                    uint32_t r[16];
                    __syncwarp();
                    tmem_ld16(at + c, r);
                    tmem_wait_ld();
                    if (joined) {  // where the ring was: all of it has been read
                        const bool any = w.k0 < w.k1;
#pragma unroll
                        for (int q = 0; q < 16; ++q)
                            reinterpret_cast<uint32_t*>(raw + (ring - smem_of(raw)))[(c + q) * kBM + warp * 32 + lane] = any ? r[q] : 0u;
                    } else if (r0 + lane < p.I) {
                        put_columns<T>(p, r, r0 + lane, (int64_t)w.j * BN + c);
                    }
                }
            } else {
                const int cols = BN * 4 / R::kEpilogue, c = (warp >> 2) * cols;  // this warp's
                uint8_t* corners = raw + (ring - smem_of(raw)) + S * R::kStage;
                float* part = w.part < 0 ? nullptr : p.part + (w.part * kBlocks * kBM + in_tile) * BN + c;
                if (!put_blocks<T, !A_MN && !B_MN>(p, &out_map, &pre_map, at + c, corners + warp * kCorner,
                                   reinterpret_cast<float*>(corners + R::kEpilogue * kCorner + warp * kBias), r0, w.j * BN + c,
                                   r0 < p.I ? cols / 32 : 0, part, BN, lane, turn, wait)) break;
            }
            __syncwarp();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_in(told + 8 * acc);
                else mbar_arrive(told + 8 * acc);
            }
        }
    }
    if (!SWAP && warp < R::kEpilogue && lane == 0) tma_store_done();
    tc_fence_before();
    __syncthreads();
    if (joined) {
        const Work w(p, first, true, mine);
        cluster_sync();
        if (warp < 4) join_columns<T, BN>(p, ring, w.i, w.j, mine);
    }
    if (PAIR || joined) cluster_sync();  // nothing of this block's memory is wanted by another any more
    tc_fence_after();
    if (threadIdx.x == 0 && stop) atomicAdd(&g_timeouts, 1u);
    if (warp == kMma) tmem_free<PAIR>(tmem, R::kColumns);
    if (p.beside) pdl_enter_last();  // whoever waits for this grid waits for those before it
}

// The shares of the tiles that are not whole, added up in a fixed order, and the epilogue: four columns a thread, or,
// where there are many shares, four threads (GROUPS), each with every fourth share; 2^blocks_per_tile blocks a tile of
// 2^(wide + 2) columns.  (No shares: of zeros.  With one thread / four, us: 64 shares of a 64 x 64 gradient 12.2 / 5.2, 9 of
// 512 x 512 5.7 / 5.2, 4 of 1,000 x 776 6.2 / 8.1.)
template <class T, int GROUPS>
__global__ void __launch_bounds__(256) k_product_finish(const Product p, int blocks_per_tile, int wide) {
    pdl_enter();
    constexpr int kOf = 256 / GROUPS;
    __shared__ float4 sums[GROUPS][kOf];
    const int mine = threadIdx.x % kOf, group = threadIdx.x / kOf;
    const int64_t all = gridDim.x * (int64_t)kOf;
    const float4* part = reinterpret_cast<const float4*>(p.part) + blockIdx.x * (int64_t)kOf + mine;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& x) { sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w); };
#pragma unroll 8
    for (int s = group; s < p.shares; s += GROUPS) add(part[s * all]);
    if (GROUPS > 1) {
        sums[group][mine] = sum;
        __syncthreads();
        if (group) return;
        for (int g = 1; g < GROUPS; ++g) add(sums[g][mine]);
    }
    const int q = (int)(blockIdx.x & ((1u << blocks_per_tile) - 1)) * kOf + mine;
    int i, j;
    tile_at(p, p.whole + (int)(blockIdx.x >> blocks_per_tile), i, j);
    const int64_t row = (int64_t)i * ((kOf << blocks_per_tile) >> wide) + (q >> wide);
    const int64_t col = ((int64_t)j << (wide + 2)) + (q & ((1 << wide) - 1)) * 4;
    if (row < p.I && col < p.J) put_four<T>(p.e, sum, row, col, p.J);
}

// Rows whose stride or place TMA does not take (multiples of 16 bytes), laid out anew: up to two matrices at a time.
// Bound by latency at the sizes met (4,099 x 777 and 1,001 x 777: 6 us, 16 MB), by HBM above.
struct Align {
    const uint16_t* in;
    uint16_t* out;
    int64_t stride, out_stride, rows, cols;
};
__global__ void __launch_bounds__(256) k_align(Align a, Align b) {
    pdl_enter();
    const Align m = blockIdx.y ? b : a;
    const Span span(m.in, m.rows, m.stride, (int)m.cols);
    const int64_t per = m.out_stride / 8, step = gridDim.x * 256ll;
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < m.rows * per; at += step) {
        const int64_t r = at / per, c = (at - r * per) * 8;
        Values<uint16_t, 8, false> v;
        v.load(m.in + r * m.stride + c, (int)(m.cols - c), span);
        *reinterpret_cast<uint4*>(m.out + r * m.out_stride + c) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    }
}

// p = dy act'(z), and the sums of its columns over a block's rows.  A thread
// takes 8 columns, a block 256 columns of a share of the rows: one round of
// blocks, four an SM, of two rows a warp at a time.  Bound by HBM: 65,536 x 512
// bf16, relu, 29 us (6.8 TB/s, some of it from L2; with two blocks an SM, four rows
// and two rounds 36), 16,384 x 4,096, gelu, 63 (75).
constexpr int kSlopeBlocks = 4;
struct Slope {
    const void* dy;
    const void* pre;
    void* p;           // null: not wanted (p is dy)
    float* part;       // [shares][cols], null with one share, joined ones or no sums
    void* dbias;
    int64_t dy_stride, pre_stride, p_stride, rows, cols, share;
    int32_t act, joined;  // (the blocks of a column are a cluster)
};
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(256, ALIGNED ? kSlopeBlocks : 2) k_slope(Slope a) {
    pdl_enter();
    __shared__ float sums[8][256], mine[256];
    using Row = Values<T, 8, ALIGNED>;
    constexpr int kRows = 2;  // on their way at a time
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (blockIdx.x * 32ll + lane) * 8;
    const int n = (int)min((int64_t)8, a.cols - c);
    const int64_t r0 = blockIdx.y * a.share, r1 = min(a.rows, r0 + a.share);
    const T *dy = static_cast<const T*>(a.dy), *pre = static_cast<const T*>(a.pre);
    const Span dy_span(dy, a.rows, a.dy_stride, (int)a.cols), pre_span(pre, a.rows, a.pre_stride, (int)a.cols);
    float2 s[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] = splat2(0.f);
    if (n > 0)
        for (int64_t r = r0 + warp; r < r1; r += 8 * kRows) {
            Row d[kRows], z[kRows];
            typename Row::Around d_at[kRows], z_at[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (r + 8 * i >= r1) continue;
                d_at[i] = Row::around(dy + (r + 8 * i) * a.dy_stride + c, dy_span);
                if (a.act != MLKV_ACT_NONE) z_at[i] = Row::around(pre + (r + 8 * i) * a.pre_stride + c, pre_span);
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (r + 8 * i >= r1) continue;
                d[i].settle(d_at[i], Row::place(dy + (r + 8 * i) * a.dy_stride), n);
                if (a.act != MLKV_ACT_NONE) z[i].settle(z_at[i], Row::place(pre + (r + 8 * i) * a.pre_stride), n);
                if (a.act == MLKV_ACT_NONE) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) s[q] = add2(s[q], d[i].pair(q));
                }
                by_act(a.act, [&](auto act) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float2 v = mul2(d[i].pair(q), slope<decltype(act)::value>(z[i].pair(q)));
                        s[q] = add2(s[q], v);
                        d[i].set(q, v);
                    }
                });
                if (a.p)  // (rows of whole vectors)
                    *reinterpret_cast<uint4*>(static_cast<T*>(a.p) + (r + 8 * i) * a.p_stride + c) = make_uint4(d[i].w[0], d[i].w[1], d[i].w[2], d[i].w[3]);
            }
        }
    if (!a.dbias) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<float2*>(&sums[warp][lane * 8 + 2 * q]) = s[q];
    __syncthreads();
    const int64_t col = blockIdx.x * 256ll + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sums[w][threadIdx.x];
    if (a.joined) {  // the first block adds the others' sums up, in order
        mine[threadIdx.x] = t;
        cluster_sync();
        if (blockIdx.y == 0) {
            t = 0.f;
            for (int b = 0; b < (int)gridDim.y; ++b) {
                float x;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(place_in(smem_of(&mine[threadIdx.x]), b)) : "memory");
                t += x;
            }
        }
        cluster_sync();
        if (blockIdx.y) return;
    }
    if (col >= a.cols) return;
    if (a.part) a.part[blockIdx.y * a.cols + col] = t;
    else static_cast<T*>(a.dbias)[col] = from_float<T>(t);
}

// The shares' sums of 32 columns, added up by 32 warps of which each takes every 32nd share, then over the warps (608
// shares of 512 columns: 6 us with the launch, from L2).
// beside: as in k_product (the shares are complete, and read from L2).
__global__ void __launch_bounds__(1024) k_column_sums(const float* part, int shares, int64_t cols, void* out, int32_t type, int beside) {
    if (beside) pdl_next();
    else pdl_enter();
    __shared__ float s[32][33];
    const int64_t c = blockIdx.x * 32ll + (threadIdx.x & 31);
    const int w = threadIdx.x >> 5;
    float t = 0.f;
    if (c < cols)
        for (int b = w; b < shares; b += 32) t += __ldcg(part + b * cols + c);
    s[w][threadIdx.x & 31] = t;
    __syncthreads();
    t = group_sum(s[threadIdx.x & 31][w], 32);  // warp w: column w of the block's
    const int64_t o = blockIdx.x * 32ll + w;
    if ((threadIdx.x & 31) == 0 && o < cols) static_cast<uint16_t*>(out)[o] = narrow(type, t);
    if (beside) pdl_enter_last();
}

// --- host ----------------------------------------------------------------------

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encode() {
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (PFN_cuTensorMapEncodeTiled_v12000)f;
    }();
    return fn;
}

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
constexpr int64_t kAlign = 256;

// Working memory handed out in order; with base == nullptr only counted.
struct Arena {
    char* base;
    int64_t used = 0;
    void* take(int64_t bytes) {
        void* p = base ? base + used : nullptr;
        used += round_up(bytes, kAlign);
        return p;
    }
};

struct Matrix {
    const uint16_t* p;
    int64_t stride, rows, cols;
    bool aligned() const { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; }
};

struct Caller {
    cudaStream_t st;
    int sms;
    bool run;        // false: only count the working memory
    int32_t type;
    Arena arena;
    int rc = MLKV_OK;
    unsigned blocks_for(int64_t items) const { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 16ll * sms)); }

    // Two matrices as TMA takes them.
    void align(Matrix& a, Matrix& b) {
        Align to[2] = {};
        int n = 0;
        for (Matrix* m : {&a, &b}) {
            if (m->rows == 1) m->stride = round_up(m->cols, 8);  // (the one row's end is its end)
            if (m->aligned() || !m->rows || !m->cols) continue;
            const int64_t stride = round_up(m->cols, 8);
            uint16_t* p = static_cast<uint16_t*>(arena.take(m->rows * stride * 2));
            to[n++] = {m->p, p, m->stride, stride, m->rows, m->cols};
            *m = {p, stride, m->rows, m->cols};
        }
        if (!run || !n) return;
        const int64_t vectors = std::max(to[0].rows * to[0].out_stride, to[1].rows * to[1].out_stride) / 8;
        launch_kernel(true, k_align, dim3(blocks_for(vectors), n), dim3(256), 0, st, to[0], to[1]);
    }

    bool encode(CUtensorMap* map, const Matrix& m, bool mn, int rows) {
        return encode(map, m, 64, mn ? kBK : rows, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    bool encode(CUtensorMap* map, const Matrix& m, int across, int down, CUtensorMapSwizzle swizzle) {
        const auto fn = tensor_map_encode();
        if (!fn) return false;
        const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows}, strides[1] = {(cuuint64_t)m.stride * 2};
        const cuuint32_t box[2] = {(cuuint32_t)across, (cuuint32_t)down}, step[2] = {1, 1};
        return fn(map, type == MLKV_TYPE_BFLOAT ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                  const_cast<uint16_t*>(m.p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }

    template <int BN, bool A_MN, bool B_MN, bool SWAP, bool PAIR = false>
    void launch(const Matrix& a, const Matrix& b, Product p) {
        using R = Ring<BN, SWAP, PAIR>;
        CUtensorMap ma, mb;
        if (!encode(&ma, a, A_MN, kBM) || !encode(&mb, b, B_MN, PAIR ? BN / 2 : BN)) {
            rc = MLKV_ERR_CUDA;
            return;
        }
        CUtensorMap out = ma, pre = ma;  // (not looked at where the epilogue does not store by TMA)
        if (!SWAP && p.e.wide) {
            if (!encode(&out, {static_cast<const uint16_t*>(p.e.out), p.e.out_stride, p.I, p.J}, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B) ||
                (p.e.pre && !encode(&pre, {static_cast<const uint16_t*>(p.e.pre), p.e.pre_stride, p.I, p.J}, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B))) {
                rc = MLKV_ERR_CUDA;
                return;
            }
        }
        p.injected = take_injected_product();
        p.idesc = mma_desc(type == MLKV_TYPE_BFLOAT, A_MN, B_MN, PAIR ? 2 * kBM : kBM, BN);
        const int64_t all = (int64_t)p.tiles_i * p.tiles_j, tiles = p.joined ? all * p.shares : p.whole + (all - p.whole) * p.shares;
        auto go = [&](auto kernel) {
            if (!dense_smem(kernel, R::kBytes)) rc = MLKV_ERR_CUDA;
            else if (PAIR) launch_clusters(kernel, 2, 2 * std::min<int64_t>(tiles, sms / 2), R::kThreads, R::kBytes, st, ma, mb, out, pre, p);
            else if (p.joined) launch_clusters(kernel, p.shares, tiles, R::kThreads, R::kBytes, st, ma, mb, out, pre, p);
            else launch_kernel(true, kernel, dim3((unsigned)std::min<int64_t>(tiles, sms)), dim3(R::kThreads), R::kBytes, st, ma, mb, out, pre, p);
        };
        if (type == MLKV_TYPE_BFLOAT) go(k_product<BN, A_MN, B_MN, SWAP, PAIR, __nv_bfloat16>);
        else go(k_product<BN, A_MN, B_MN, SWAP, PAIR, __half>);
    }
    void finish_shares(const Product& p, int high, int bn) {
        if (!run) return;
        const int groups = p.shares >= 8 ? 4 : 1, blocks = high * bn / 1024 * groups, wide = bn == 64 ? 4 : bn == 128 ? 5 : 6;
        int per = 0;
        while (1 << per < blocks) ++per;
        const dim3 grid((unsigned)((int64_t)(p.tiles_i * p.tiles_j - p.whole) * blocks));
        const bool b = type == MLKV_TYPE_BFLOAT;
        const auto kernel = groups == 4 ? (b ? k_product_finish<__nv_bfloat16, 4> : k_product_finish<__half, 4>)
                                        : (b ? k_product_finish<__nv_bfloat16, 1> : k_product_finish<__half, 1>);
        launch_kernel(true, kernel, grid, dim3(256), 0, st, p, per, wide);
    }
    // Whether pairs of blocks take the tiles of 256 columns: where there are enough for every pair, and k is long
    // enough for the products to count beside the epilogue.  (Single blocks / pairs, us: 16,384 x 4,096 by k = 4,096
    // 331 / 298; 8,192 x 1,024 by 8,192 102 / 86; 4,096 x 4,096 by 1,024 32 / 29; 65,536 x 512 by 416 37 / 42.)
    bool pair_pays(int64_t tiles_i, int64_t tiles_j, int64_t blocks) const {
        return blocks >= 12 && (tiles_i + 1) / 2 * tiles_j * (blocks / 12) >= sms / 2;
    }

    // The time, in us, of `rounds` of work after one another, each of a tile of bn columns (and 128 rows a block) and
    // `blocks` blocks of k, on `busy` SMs: what a width takes besides k, once; a block of k, by its operands' latency,
    // their bytes through L2 on all those SMs, or the matrix unit's rate.
    static float time_of(int64_t rounds, int bn, int64_t blocks, int64_t busy, bool pair) {
        constexpr float kLatency = 0.25f, kL2 = 15e6f;
        const float fixed = bn == 64 ? 5.f : bn == 128 ? 6.5f : 8.5f, bytes = (float)(kBM + (pair ? bn / 2 : bn)) * kBK * 2;
        const float block = std::max(rounds > 1 ? 0.f : kLatency, std::max((float)busy * bytes / kL2, 0.34f * bn / 256));
        return fixed + (float)(rounds * blocks) * block;
    }
    // The launch that adds shares of tiles up.
    static float time_to_finish(int64_t tiles, int64_t shares, int high, int bn) {
        constexpr float kLaunch = 4.f, kBytes = 6e6f;
        return kLaunch + (float)((shares + 1) * tiles * high * bn) * 4 / kBytes;
    }
    // Tiles (the last ones) whose k is shared out, and their shares, of at least 4 blocks: where the tiles do not fill
    // the GPU, or its last round.  (Gradients of a 4,096 x 4,096 weight over 16,384 rows: 256 tiles on 76 pairs of SMs.)
    struct Split { int64_t tiles, shares; float time; };
    Split split(int64_t tiles, int high, int bn, int64_t blocks) const {
        const bool pair = high > kBM;
        const int64_t places = pair ? sms / 2 : sms, full = tiles / places, rest = tiles % places;
        const int64_t busy = full ? sms : rest * (pair ? 2 : 1);
        Split best = {0, 1, time_of(full + (rest > 0), bn, blocks, busy, pair)};
        const float before = full ? time_of(full, bn, blocks, busy, pair) : 0.f;
        if (!rest) return best;
        auto look = [&](int64_t s) {
            const int64_t rounds = (rest * s + places - 1) / places;
            if (s < 2 || s * 4 > blocks || rounds >= s) return;
            const float t = before + time_of(rounds, bn, (blocks + s - 1) / s, std::min(rest * s, places) * (pair ? 2 : 1), pair) + time_to_finish(rest, s, high, bn);
            if (t < best.time) best = {rest, s, t};
        };
        for (int64_t s = std::min(places / rest, blocks / 4); s > 1; s /= 2) look(s);  // within a round
        for (int64_t r = 2; r <= 4 && full; ++r) look(r * places / rest);               // the most in r short ones
        return best;
    }
    // The width of single blocks' tiles, where the narrower ones fit on the GPU at once.  (Widths of 256 / 128 / 64 at
    // their best, us: 300 x 1,000 by k = 520 9.7 / 7.8 / 7.2; 1,000 x 1,000 by 1,000 12.8 / 9.9 / 8.3; 200 x 512 by 8,192
    // 12.3 / 10.5 / 10.3; 512 x 512 by 8,000 13.1 / 12.4 / 14.6; 4,096 x 1,000 by 776 14.6 / 16.0 / 21.0.)
    int width(int64_t rows, int64_t cols, int64_t blocks) const {
        int best = cols <= 64 ? 64 : cols <= 128 ? 128 : 256;
        float least = 3e38f;
        for (int bn = 64; bn <= 256; bn *= 2) {
            const int64_t tiles = (rows + kBM - 1) / kBM * ((cols + bn - 1) / bn);
            if (tiles <= sms) {
                const float t = split(tiles, kBM, bn, blocks).time;
                if (t < least) {
                    least = t;
                    best = bn;
                }
            }
            if (bn >= cols) break;
        }
        return best;
    }

    // What a product leaves to another launch: shares to be added up.
    struct Rest {
        Product p;
        int high, bn;
    };
    void finish(const Rest& r) {
        if (r.p.part) finish_shares(r.p, r.high, r.bn);
    }

    // out = epilogue(A B^T): A [rows][k], B [cols][k]; *_mn: held as [k][rows], [k][cols].
    template <bool A_MN, bool B_MN>
    Rest product(Matrix a, Matrix b, int64_t rows, int64_t cols, int64_t k, Epilogue e, bool beside = false) {
        if (!rows || !cols) return {};
        e.type = type;
        auto wide = [](const void* p, int64_t stride) { return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0); };
        e.wide = wide(e.out, e.out_stride) && wide(e.pre, e.pre_stride) && wide(e.residual, e.residual_stride);
        const bool swap = !A_MN && rows <= 64 && k > 0;  // few rows: the wide operand fills the tiles' 128 rows
        Product p = {};
        p.I = (int32_t)(swap ? cols : rows);
        p.J = (int32_t)(swap ? rows : cols);
        p.blocks = (int32_t)((k + kBK - 1) / kBK);
        p.e = e;
        if (!A_MN && !B_MN && !swap && e.act == MLKV_ACT_RELU) {
            p.a = a.p; p.a_stride = a.stride; p.b = b.p; p.b_stride = b.stride;
            p.k = (int32_t)k;
            p.doubt = (float)p.blocks / (1 << 22);
        }
        const int64_t down = ((int64_t)p.I + kBM - 1) / kBM;
        const bool pair = !swap && cols > 128 && pair_pays(down, (p.J + 255) / 256, p.blocks);
        const int bn = swap ? (rows <= 16 ? 16 : rows <= 32 ? 32 : 64) : pair ? 256 : width(rows, cols, p.blocks);
        const int64_t across = (p.J + bn - 1) / bn, high = pair ? 2 * kBM : kBM, tiles = ((int64_t)p.I + high - 1) / high * across;
        if (tiles >= (int64_t)1 << 30) {
            rc = MLKV_ERR_UNSUPPORTED;
            return {};
        }
        p.tiles_i = (int32_t)(tiles / across);
        p.tiles_j = (int32_t)across;
        p.whole = (int32_t)tiles;
        p.shares = 1;
        if (k == 0) {
            p.whole = p.shares = 0;
            finish_shares(p, (int)high, bn);
            return {};
        }
        if (swap) {
            // few rows: k in shares of at least 4 blocks, those of a tile a cluster (of 2, 4 or 8), one tile a block
            int n = 1;
            while (n < 8 && 2 * n <= std::min<int64_t>(sms / tiles, p.blocks / 4)) n *= 2;
            p.shares = n;
            p.joined = n > 1;
            p.blocks_per_share = (p.blocks + n - 1) / n;  // (the last may be of nothing)
        } else {
            const Split s = split(tiles, (int)high, bn, p.blocks);
            if (s.shares > 1) {
                p.whole = (int32_t)(tiles - s.tiles);
                p.blocks_per_share = (int32_t)((p.blocks + s.shares - 1) / s.shares);
                p.shares = (p.blocks + p.blocks_per_share - 1) / p.blocks_per_share;
                p.part = static_cast<float*>(arena.take(s.tiles * p.shares * high * bn * 4));
            }
        }
        p.beside = beside;
        const Rest rest = {p, (int)high, bn};
        if (!run) return rest;
        if constexpr (!A_MN) {
            if (swap) {
                if (bn == 16) launch<16, B_MN, false, true>(b, a, p);
                else if (bn == 32) launch<32, B_MN, false, true>(b, a, p);
                else launch<64, B_MN, false, true>(b, a, p);
            }
        }
        if (!swap) {
            if (bn == 64) launch<64, A_MN, B_MN, false>(a, b, p);
            else if (bn == 128) launch<128, A_MN, B_MN, false>(a, b, p);
            else if (pair) launch<256, A_MN, B_MN, false, true>(a, b, p);
            else launch<256, A_MN, B_MN, false>(a, b, p);
        }
        return rest;
    }

    void forward(const mlkv_linear_args& g) {
        Epilogue e = {};
        e.bias = g.d_bias; e.residual = g.d_residual; e.residual_stride = g.residual_stride;
        e.pre = g.d_pre; e.pre_stride = g.pre_stride; e.out = g.d_y; e.out_stride = g.y_stride; e.act = g.activation;
        Matrix x = {(const uint16_t*)g.d_x, g.x_stride, g.m, g.k}, w = {(const uint16_t*)g.d_weight, g.weight_stride, g.n, g.k};
        if (g.m && g.n && g.k) align(x, w);
        finish(product<false, false>(x, w, g.m, g.n, g.k, e));
    }

    void backward(const mlkv_linear_args& g) {
        Matrix p = {(const uint16_t*)g.d_dy, g.dy_stride, g.m, g.n};
        const bool act = g.activation != MLKV_ACT_NONE, products = (g.d_dx || g.d_dweight) && g.m && g.n;
        const bool copy = products && (act || !p.aligned());
        const float* part = nullptr;  // of dbias, from `shares` blocks
        int shares = 0;
        if (g.m && g.n && (copy || g.d_dbias)) {
            Slope s = {};
            s.dy = p.p; s.dy_stride = g.dy_stride; s.pre = g.d_pre; s.pre_stride = g.pre_stride;
            s.rows = g.m; s.cols = g.n; s.act = g.activation; s.dbias = g.d_dbias;
            if (copy) {
                s.p_stride = round_up(g.n, 8);
                s.p = arena.take(g.m * s.p_stride * 2);
                p = {static_cast<const uint16_t*>(s.p), s.p_stride, g.m, g.n};
            }
            const Matrix dy = {(const uint16_t*)s.dy, s.dy_stride, 0, 0}, pre = {(const uint16_t*)s.pre, s.pre_stride, 0, 0};
            const bool whole = g.n % 8 == 0 && dy.aligned() && (!act || pre.aligned());
            const int64_t across = (g.n + 255) / 256;
            // a block's warps take 4 rows each at least; up to 1,024 rows no column has more blocks than a cluster
            const int64_t most = g.d_dbias && g.m <= 1024 ? 8 : (int64_t)kSlopeBlocks * sms / across;
            const int64_t wanted = std::max<int64_t>(1, std::min<int64_t>((g.m + 31) / 32, most));
            s.share = (g.m + wanted - 1) / wanted;
            const unsigned down = (unsigned)((g.m + s.share - 1) / s.share);
            s.joined = g.d_dbias && down > 1 && down <= 8;
            if (g.d_dbias && down > 8) s.part = static_cast<float*>(arena.take((int64_t)down * g.n * 4));
            if (run) {
                const dim3 grid((unsigned)across, down);
                auto go = [&](auto kernel) {
                    if (s.joined) launch_clusters(kernel, dim3(1, down), grid, 256, 0, st, s);
                    else launch_kernel(true, kernel, grid, dim3(256), 0, st, s);
                };
                const bool b = type == MLKV_TYPE_BFLOAT;
                if (whole) go(b ? k_slope<__nv_bfloat16, true> : k_slope<__half, true>);
                else go(b ? k_slope<__nv_bfloat16, false> : k_slope<__half, false>);
                part = s.part;
                shares = (int)down;
            }
        } else if (run && g.d_dbias && g.n) {
            if (cudaMemsetAsync(g.d_dbias, 0, g.n * 2, st) != cudaSuccess) rc = MLKV_ERR_CUDA;
        }
        Epilogue e = {};
        Matrix x = {(const uint16_t*)g.d_x, g.x_stride, g.m, g.k}, w = {(const uint16_t*)g.d_weight, g.weight_stride, g.n, g.k}, none = {};
        if (g.m && g.n && g.k) align(g.d_dweight ? x : none, g.d_dx ? w : none);
        // The bias's sums and dW's blocks take the SMs that dx has no work for, at its start or as its last tiles run out.  (A step of 300 x 520
        // to 1,000: 21.3 us on the GPU, one after the other 25.2; of 4,099 x 777 to 1,001 67, 71.)
        Rest dx = {}, dw = {};
        if (g.d_dx) {
            e.out = g.d_dx; e.out_stride = g.dx_stride;
            dx = product<false, true>(p, w, g.m, g.k, g.n, e);
        }
        const bool beside = !MLKV_PDL_TRIGGER_FIRST && rc == MLKV_OK && g.d_dx && g.m && g.n && g.k;  // (dx's blocks have waited first)
        if (part) launch_kernel(true, k_column_sums, dim3((unsigned)((g.n + 31) / 32)), dim3(1024), 0, st, part, shares, g.n, g.d_dbias, type, (int)beside);
        if (g.d_dweight) {
            e.out = g.d_dweight; e.out_stride = g.dweight_stride;
            dw = product<true, true>(p, x, g.n, g.k, g.m, e, beside);
        }
        finish(dx);
        finish(dw);
    }
};

bool rows_ok(const void* p, int64_t stride, int64_t rows, int64_t cols, bool may_be_null) {
    if (!p) return may_be_null || rows == 0 || cols == 0;
    return stride >= cols && stride < (int64_t)1 << 38;  // (TMA's strides have 40 bits)
}
bool linear_ok(const mlkv_linear_args* g) {
    if (!g || g->m < 0 || g->n < 0 || g->k < 0) return false;
    if (std::max(g->m, std::max(g->n, g->k)) >= (int64_t)1 << 30) return false;  // (a tile's rows in 32 bits)
    if (g->type != MLKV_TYPE_BFLOAT && g->type != MLKV_TYPE_HALF) return false;
    if (g->activation < MLKV_ACT_NONE || g->activation > MLKV_ACT_SILU) return false;
    return rows_ok(g->d_x, g->x_stride, g->m, g->k, false) && rows_ok(g->d_weight, g->weight_stride, g->n, g->k, false);
}
bool forward_ok(const mlkv_linear_args* g) {
    return linear_ok(g) && rows_ok(g->d_y, g->y_stride, g->m, g->n, false) && rows_ok(g->d_pre, g->pre_stride, g->m, g->n, true) &&
           rows_ok(g->d_residual, g->residual_stride, g->m, g->n, true);
}
bool backward_ok(const mlkv_linear_args* g) {
    return linear_ok(g) && rows_ok(g->d_dy, g->dy_stride, g->m, g->n, false) &&
           rows_ok(g->d_pre, g->pre_stride, g->m, g->n, g->activation == MLKV_ACT_NONE) &&
           rows_ok(g->d_dx, g->dx_stride, g->m, g->k, true) && rows_ok(g->d_dweight, g->dweight_stride, g->n, g->k, true);
}

int64_t working_memory(const mlkv_linear_args* g, bool backward) {
    Caller c = {nullptr, dense_sms(), false, g->type, {nullptr}};
    if (!c.sms) return -1;
    if (backward) c.backward(*g);
    else c.forward(*g);
    return c.rc == MLKV_OK ? c.arena.used : -2;
}

int run_linear(const mlkv_linear_args* g, bool backward, void* stream) {
    const int64_t need = working_memory(g, backward);
    if (need < 0) return need == -2 ? MLKV_ERR_UNSUPPORTED : MLKV_ERR_CUDA;
    if (!workspace_ok(g->d_workspace, g->workspace_bytes, need)) return MLKV_ERR_INVALID;
    Caller c = {(cudaStream_t)stream, dense_sms(), true, g->type, {static_cast<char*>(g->d_workspace)}};
    if (backward) c.backward(*g);
    else c.forward(*g);
    if (c.rc != MLKV_OK) return c.rc;
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

}  // namespace

extern "C" int64_t mlkv_linear_workspace(const mlkv_linear_args* args) {
    return forward_ok(args) ? working_memory(args, false) : -1;
}
extern "C" int64_t mlkv_linear_backward_workspace(const mlkv_linear_args* args) {
    return backward_ok(args) ? working_memory(args, true) : -1;
}
extern "C" int mlkv_linear(const mlkv_linear_args* args, void* stream) {
    MLKV_DENSE_RANGE("mlkv_linear");
    return forward_ok(args) ? run_linear(args, false, stream) : MLKV_ERR_INVALID;
}
extern "C" int mlkv_linear_backward(const mlkv_linear_args* args, void* stream) {
    MLKV_DENSE_RANGE("mlkv_linear_backward");
    return backward_ok(args) ? run_linear(args, true, stream) : MLKV_ERR_INVALID;
}

extern "C" int mlkv_dense_sync(void* stream) {
    MLKV_DENSE_RANGE("mlkv_dense_sync");
    constexpr int kDevices = 64;
    static std::atomic<uint32_t> told[kDevices];  // of g_timeouts
    int dev = 0;
    uint32_t now = 0;
    // (first the wait, which a stream that is being captured refuses: a copy would be captured)
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices || cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess ||
        cudaMemcpyFromSymbolAsync(&now, g_timeouts, sizeof(now), 0, cudaMemcpyDeviceToHost, (cudaStream_t)stream) != cudaSuccess ||
        cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess)
        return MLKV_ERR_CUDA;
    for (uint32_t before = told[dev].load(); (int32_t)(now - before) > 0;)
        if (told[dev].compare_exchange_weak(before, now)) return MLKV_ERR_TIMEOUT;
    return MLKV_OK;
}
