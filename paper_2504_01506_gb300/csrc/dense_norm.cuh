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

// A lane's vectors are 16 bytes of x: V values.  Weights, held as fp32 in shared
// memory: in order, or, for vectors of 8, the first four values of every vector,
// then the last four (16-byte reads of neighbouring lanes then lie side by side).
// `room` values, a multiple of V and at least dim; those past dim are 0, and
// without a weight it is `none`.
template <int V>
__device__ __forceinline__ int weight_place(int c, int room) {
    return V == 8 ? (((c >> 2) & 1) * (room / 8) + (c >> 3)) * 4 + (c & 3) : c;
}
template <int V>
__device__ __forceinline__ void stage_weights(float* to, const void* p, int32_t type, int dim, int room, float none) {
    for (int c = threadIdx.x; c < room; c += blockDim.x)
        to[weight_place<V>(c, room)] = c >= dim ? 0.f : p ? load_as_float(p, type, c) : none;
}
template <int V>
__device__ __forceinline__ void weight_pairs(const float* w, int j, int room, float2 (&o)[V / 2]) {
#pragma unroll
    for (int c = 0; c < V; c += 4) {
        const float4 q = *reinterpret_cast<const float4*>(w + weight_place<V>(j * V + c, room));
        o[c / 2] = make_float2(q.x, q.y);
        o[c / 2 + 1] = make_float2(q.z, q.w);
    }
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Where a thread stands in its block's teams.
struct Team {
    int L, lane, index, count, warps;  // lanes a row; this lane; this team; teams a block; warps a team
    float2* mine;                      // this team's place for its warps' sums: 2 x (8, or all 32) pairs
    // sums: 64 pairs of the block.  (Followed by a barrier of the block before the first sum.)
    __device__ Team(int lanes, float2* sums)
        : L(lanes), lane(threadIdx.x % lanes), index(threadIdx.x / lanes), count(blockDim.x / lanes), warps(lanes / 32) {
        mine = sums + (warps <= 8 ? index * 16 : 0);  // (at most 4 teams of several warps, one of more than 8)
        for (int i = threadIdx.x; i < 64; i += blockDim.x) sums[i] = make_float2(0.f, 0.f);
    }
    // The sums of a and b over the team.  `turn` goes 0, 1, 0, ..., so that one barrier a sum is enough: who
    // writes a place again has seen all of its team past the next sum.
    __device__ __forceinline__ void sum(float& a, float& b, int turn) const {
        if (L < 32) {
            for (int o = L >> 1; o; o >>= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, o);
                b += __shfl_xor_sync(0xffffffffu, b, o);
            }
            return;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (L == 32) return;
        float2* at = mine + turn * (warps <= 8 ? 8 : 32);
        if ((threadIdx.x & 31) == 0) at[lane >> 5] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(L) : "memory");
        float2 s = make_float2(0.f, 0.f);
        if (warps <= 8) {  // (places without a warp hold 0)
#pragma unroll
            for (int i = 0; i < 4; i += 2) s = pair_sum(s, at + i);
            if (warps > 4)
#pragma unroll
                for (int i = 4; i < 8; i += 2) s = pair_sum(s, at + i);
        } else {
            for (int i = 0; i < warps; ++i) s = add2(s, at[i]);
        }
        a = s.x;
        b = s.y;
    }
    __device__ __forceinline__ void sync() const {
        if (L <= 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(L) : "memory");
    }
    static __device__ __forceinline__ float2 pair_sum(float2 s, const float2* two) {
        const float4 q = *reinterpret_cast<const float4*>(two);
        return add2(add2(s, make_float2(q.x, q.y)), make_float2(q.z, q.w));
    }
    __device__ __forceinline__ float sum(float a, int turn) const {
        float none = 0.f;
        sum(a, none, turn);
        return a;
    }
};

// Whether rows are whole vectors of V values on their boundary.
inline bool norm_aligned(const void* p, int64_t stride, int size, int64_t dim, int V) {
    return !p || (reinterpret_cast<uintptr_t>(p) % (V * size) == 0 && stride % V == 0 && dim % V == 0);
}

constexpr int kNormAhead = 2;  // rows of each team on their way into shared memory

// Bytes of a team's row in shared memory, with what lies around it.
__host__ __device__ constexpr int norm_row(int room, int size) { return (room * size + 47) / 16 * 16; }

// Rows on their way into shared memory.  ALIGNED: each thread has its own vectors, and reads only what it copied
// itself.  Else a team has the row, in the aligned pieces that it lies in, of which a lane's vector is parts of two.
// (20,000 rows of 4,001 bf16 values, forward / backward: each lane's words loaded into registers a row ahead 140 / 272
// us; this way 108 / 193, and, with the row on its way out in shared memory too, to be stored in 16-byte pieces, 124 /
// 185: its barriers and shifts cost what the wider stores save.)
template <class T, int V, int NV, bool ALIGNED> struct RowRing {
    using Row = Values<T, V, ALIGNED>;
    uint8_t* at;
    int apart, slot_bytes;  // bytes from a thread's vector to its next; of a slot
    static __device__ __forceinline__ int bytes(const Team& tm, int room) {
        return kNormAhead * (ALIGNED ? NV * (int)blockDim.x * Row::kBytes : tm.count * norm_row(room, sizeof(T)));
    }
    __device__ __forceinline__ RowRing(uint8_t* from, const Team& tm, int room)
        : at(from + (ALIGNED ? threadIdx.x * Row::kBytes : tm.index * norm_row(room, sizeof(T)))), apart((int)blockDim.x * Row::kBytes),
          slot_bytes(bytes(tm, room) / kNormAhead) {}
    // Of this lane, whose vectors start at columns c.
    __device__ __forceinline__ void fetch(const Team& tm, int slot, const T* row, const int (&c)[NV], int dim, const Span& span) const {
        uint8_t* to = at + slot * slot_bytes;
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < NV; ++i) copy_async<Row::kBytes>(to + i * apart, row + c[i]);
        } else {
            using Piece = Values<T, 16 / sizeof(T), false>;
            const uint8_t* from = Piece::piece(row);
            const int end = (int)Piece::place(row) + dim * (int)sizeof(T);
            for (int p = tm.lane * 16; p < end; p += tm.L * 16) {
                if (Piece::inside(from + p, 16, span)) copy_async<16>(to + p, from + p);
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(to + p)[i] = Piece::edge(from + p, i, span);
            }
        }
    }
    // Vector i, from column c on, of a row `by` bytes after a boundary.
    __device__ __forceinline__ void take(Row& v, int slot, int i, int c, uint32_t by, int dim) const {
        if (ALIGNED) v.take(at + slot * slot_bytes, i * apart, V);
        else v.take(at + slot * slot_bytes, by + c * (int)sizeof(T), dim - c);
    }
};

struct NormShape {
    int NV, lanes;  // lanes == 0: the row does not fit
};
// The vectors a lane holds: as many as `most` values allow, so that as few lanes
// as can be share the sums over a row (their cost is per lane and row: 200,003
// rows of 100 fp32 values take 64 us with one vector a lane, 39 with 2, 30 with
// 4, 26 with 8); fewer where there are too few rows to fill the GPU that way.
inline NormShape norm_shape(int64_t rows, int64_t dim, int V, int most, int most_lanes, int sms) {
    const int64_t nvec = (dim + V - 1) / V;
    auto lanes_of = [&](int nv) {
        const int64_t n = (nvec + nv - 1) / nv;
        int64_t p = 1;
        while (p < n && p < 32) p *= 2;
        return n <= 32 ? p : (n + 31) / 32 * 32;
    };
    int nv = 1;
    while (nv * 2 * V <= most && nv < nvec) nv *= 2;
    while (nv > 1 && lanes_of(nv / 2) <= 32 && rows * lanes_of(nv) < 1024ll * sms) nv /= 2;
    const int64_t lanes = lanes_of(nv);
    return {nv, lanes > most_lanes ? 0 : (int)lanes};
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
// f(vectors a lane, whether rows are aligned).
template <int MOST_NV, class F>
void by_shape(int NV, bool aligned, F f) {
    auto nv = [&](auto al) {
        if (NV == 1) f(Int<1>{}, al);
        else if (NV == 2) f(Int<2>{}, al);
        else if constexpr (MOST_NV >= 4) {
            if (NV == 4) f(Int<4>{}, al);
            else if constexpr (MOST_NV >= 8) f(Int<8>{}, al);
        }
    };
    if (aligned) nv(Int<1>{});
    else nv(Int<0>{});
}

inline bool norm_ok(const void* x, int64_t x_stride, int32_t x_type, int32_t y_type, int32_t w_type, int64_t rows, int64_t dim) {
    if (rows < 0 || rows >= (int64_t)1 << 30 || dim < 1 || dim >= kNormMaxDim) return false;
    if (!dense_type_ok(x_type) || !dense_type_ok(y_type) || !dense_type_ok(w_type)) return false;
    if (x_type != y_type && x_type != MLKV_TYPE_FLOAT) return false;
    return rows == 0 || (x && x_stride >= dim);
}

inline int norm_team_threads(int lanes) { return lanes >= 256 ? lanes : 256 / lanes * lanes; }

}  // namespace mlkv
