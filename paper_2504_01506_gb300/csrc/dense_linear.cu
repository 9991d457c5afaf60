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
// two accumulators in tensor memory, and four warps take the other one out
// through the epilogue.
#include <cudaTypedefs.h>

#include <algorithm>

#include "dense_mma.cuh"

using namespace mlkv;

namespace {

constexpr int kBM = 128;      // rows (i) of a tile
constexpr int kBK = 64;       // values along k of a stage: 128 bytes
constexpr int kThreads = 192; // four epilogue warps, a TMA warp, an MMA warp

__device__ uint32_t g_status;  // MLKV_ERR_TIMEOUT: a wait ran out

struct Epilogue {
    const void* bias;
    const void* residual;
    void* pre;
    void* out;          // rows of 16-bit values ...
    float* part;        // ... or, where not null, fp32 sums of a share of k: [share][rows][part_stride]
    int64_t residual_stride, pre_stride, out_stride, part_stride, part_size;
    int32_t type, act;
    int32_t wide;       // rows of out, pre and residual can be moved 16 bytes at a time
};

struct Product {
    int32_t I, J, blocks;            // extents; 64-value blocks along k
    int32_t tiles_i, tiles_j, shares, blocks_per_share;
    uint32_t idesc;
    Epilogue e;
};

__device__ __forceinline__ float widen(int32_t type, uint16_t v) {
    return type == MLKV_TYPE_BFLOAT ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
}
__device__ __forceinline__ uint16_t narrow(int32_t type, float v) {
    return type == MLKV_TYPE_BFLOAT ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
__device__ __forceinline__ uint32_t narrow2(int32_t type, float lo, float hi) {
    return (uint32_t)narrow(type, lo) | (uint32_t)narrow(type, hi) << 16;
}

__device__ __forceinline__ float sigmoid_fast(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
constexpr float kGelu = 1.5957691216057308f, kGelu3 = 0.044715f;  // 2 sqrt(2/pi): (1 + tanh u) / 2 = sigmoid(2u)
__device__ __forceinline__ float activate(int32_t act, float z) {
    if (act == MLKV_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    if (act == MLKV_ACT_SILU) return z == -INFINITY ? 0.f : z * sigmoid_fast(z);
    if (act == MLKV_ACT_GELU_TANH) return z == -INFINITY ? 0.f : z * sigmoid_fast(kGelu * (z + kGelu3 * z * z * z));
    return z;
}
__device__ __forceinline__ float slope(int32_t act, float z) {
    if (act == MLKV_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    // far from 0 the slopes are 0 and 1; the bound keeps products of a vanished and an infinite factor out
    z = fminf(fmaxf(z, -100.f), 100.f) + (z != z ? z : 0.f);
    if (act == MLKV_ACT_SILU) {
        const float q = sigmoid_fast(z);
        return q * (1.f + z * (1.f - q));
    }
    if (act == MLKV_ACT_GELU_TANH) {
        const float q = sigmoid_fast(kGelu * (z + kGelu3 * z * z * z));
        return q + z * q * (1.f - q) * kGelu * (1.f + 3.f * kGelu3 * z * z);
    }
    return 1.f;
}

// What becomes of the sum at (row, col) of the output.
__device__ __forceinline__ float finish(const Epilogue& e, float v, int64_t row, int64_t col) {
    if (e.bias) v += widen(e.type, static_cast<const uint16_t*>(e.bias)[col]);
    if (e.pre) static_cast<uint16_t*>(e.pre)[row * e.pre_stride + col] = narrow(e.type, v);
    v = activate(e.act, v);
    if (e.residual) v += widen(e.type, static_cast<const uint16_t*>(e.residual)[row * e.residual_stride + col]);
    return v;
}

// The tile (of i, j and k shares) that comes t-th: groups of 8 tiles along i by
// all along j, so that tiles that run at the same time share operands in L2.
__device__ __forceinline__ void tile_at(const Product& p, int t, int& i, int& j, int& share) {
    const int plane = p.tiles_i * p.tiles_j;
    share = t / plane;
    t -= share * plane;
    const int group = t / (8 * p.tiles_j), first = group * 8, size = min(8, p.tiles_i - first);
    t -= group * 8 * p.tiles_j;
    i = first + t % size;
    j = t / size;
}

// 16 sums of row i of the product, from column j0 on.
template <bool SWAP>
__device__ __forceinline__ void put16(const Product& p, const uint32_t (&r)[16], int64_t row_i, int64_t j0, int share) {
    const Epilogue& e = p.e;
    if (e.part) {
        float* o = e.part + share * e.part_size;
#pragma unroll
        for (int q = 0; q < 16; ++q)
            if (j0 + q < p.J) o[SWAP ? (j0 + q) * e.part_stride + row_i : row_i * e.part_stride + j0 + q] = __uint_as_float(r[q]);
    } else if (SWAP) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            if (j0 + q < p.J)
                static_cast<uint16_t*>(e.out)[(j0 + q) * e.out_stride + row_i] =
                    narrow(e.type, finish(e, __uint_as_float(r[q]), j0 + q, row_i));
    } else if (e.wide && j0 + 16 <= p.J) {
        float v[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) v[q] = __uint_as_float(r[q]);
        if (e.bias)
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] += widen(e.type, static_cast<const uint16_t*>(e.bias)[j0 + q]);
        if (e.pre) {
            uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(e.pre) + row_i * e.pre_stride + j0);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                o[h] = make_uint4(narrow2(e.type, v[8 * h], v[8 * h + 1]), narrow2(e.type, v[8 * h + 2], v[8 * h + 3]),
                                  narrow2(e.type, v[8 * h + 4], v[8 * h + 5]), narrow2(e.type, v[8 * h + 6], v[8 * h + 7]));
        }
        if (e.act != MLKV_ACT_NONE)
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = activate(e.act, v[q]);
        if (e.residual) {
            const uint4* o = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(e.residual) + row_i * e.residual_stride + j0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 x = o[h];
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v[8 * h + 2 * q] += widen(e.type, (uint16_t)w[q]);
                    v[8 * h + 2 * q + 1] += widen(e.type, (uint16_t)(w[q] >> 16));
                }
            }
        }
        uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(e.out) + row_i * e.out_stride + j0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            o[h] = make_uint4(narrow2(e.type, v[8 * h], v[8 * h + 1]), narrow2(e.type, v[8 * h + 2], v[8 * h + 3]),
                              narrow2(e.type, v[8 * h + 4], v[8 * h + 5]), narrow2(e.type, v[8 * h + 6], v[8 * h + 7]));
    } else {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            if (j0 + q < p.J)
                static_cast<uint16_t*>(e.out)[row_i * e.out_stride + j0 + q] =
                    narrow(e.type, finish(e, __uint_as_float(r[q]), row_i, j0 + q));
    }
}

template <int BN> struct Ring {
    static constexpr int kA = kBM * kBK * 2, kB = BN * kBK * 2, kStage = kA + kB;
    static constexpr int kStages = (200 * 1024) / kStage < 12 ? (200 * 1024) / kStage : 12;
    static constexpr int kBytes = kStages * kStage + 1024;  // (aligned to 1,024 within)
    static constexpr uint32_t kColumns = 2 * BN < 32 ? 32 : 2 * BN;
};

// A_MN, B_MN: the operand's rows run along i (j), not k.  SWAP: i runs along
// the output's columns (few rows: the weight is the operand of 128 rows a tile).
template <int BN, bool A_MN, bool B_MN, bool SWAP>
__global__ void __launch_bounds__(kThreads, 1)
    k_product(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb, const Product p) {
    using R = Ring<BN>;
    constexpr int S = R::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * S + 4];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    const uint32_t ring = (smem_of(raw) + 1023u) & ~1023u;
    const uint32_t full = smem_of(bars), empty = full + 8 * S, done = empty + 8 * S, drained = done + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(done + 8 * s, 1);
            mbar_init(drained + 8 * s, 128);
        }
        stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch(&ma);
        tma_prefetch(&mb);
    }
    if (warp == 5) tmem_alloc(smem_of(&tmem_at), R::kColumns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_enter();

    const int total = p.tiles_i * p.tiles_j * p.shares;
    if (warp == 4) {
        if (lane == 0) {
            uint32_t n = 0;  // stages filled
            bool ok = true;
            for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                int i, j, share;
                tile_at(p, t, i, j, share);
                const int k0 = share * p.blocks_per_share, k1 = min(p.blocks, k0 + p.blocks_per_share);
                for (int k = k0; k < k1; ++k, ++n) {
                    const uint32_t s = n % S, at = ring + s * R::kStage, bar = full + 8 * s;
                    if (n >= S && !(ok = mbar_wait(empty + 8 * s, (n / S - 1) & 1, &stop))) break;
                    mbar_expect(bar, R::kStage);
                    if (A_MN)
                        for (int b = 0; b < kBM / 64; ++b) tma_load(at + b * 8192, &ma, i * kBM + b * 64, k * kBK, bar);
                    else
                        tma_load(at, &ma, k * kBK, i * kBM, bar);
                    if (B_MN)
                        for (int b = 0; b < BN / 64; ++b) tma_load(at + R::kA + b * 8192, &mb, j * BN + b * 64, k * kBK, bar);
                    else
                        tma_load(at + R::kA, &mb, k * kBK, j * BN, bar);
                }
            }
            if (!ok) {  // given up: the copies in flight still write into this block's shared memory
                for (uint32_t b = n > S ? n - S : 0; b < n; ++b)
                    for (uint32_t tries = 0; tries < 1u << 20 && !mbar_try(full + 8 * (b % S), (b / S) & 1); ++tries) {}
            }
        }
    } else if (warp == 5) {
        if (lane == 0) {
            uint32_t n = 0, u = 0;  // stages read, accumulators used
            bool ok = true;
            for (int t = blockIdx.x; t < total && ok; t += gridDim.x, ++u) {
                int i, j, share;
                tile_at(p, t, i, j, share);
                const int k0 = share * p.blocks_per_share, k1 = min(p.blocks, k0 + p.blocks_per_share);
                const uint32_t acc = u & 1, d = tmem + acc * BN;
                if (u >= 2 && !(ok = mbar_wait(drained + 8 * acc, (u / 2 - 1) & 1, &stop))) break;
                tc_fence_after();
                for (int k = k0; k < k1; ++k, ++n) {
                    const uint32_t s = n % S, at = ring + s * R::kStage;
                    if (!(ok = mbar_wait(full + 8 * s, (n / S) & 1, &stop))) break;
                    tc_fence_after();
                    const uint64_t da = smem_desc(at, A_MN ? 8192 : 16), db = smem_desc(at + R::kA, B_MN ? 8192 : 16);
#pragma unroll
                    for (int q = 0; q < kBK / 16; ++q)  // 16 values along k: 32 bytes of a row, or 16 rows
                        tc_mma(d, da + q * (A_MN ? 128 : 2), db + q * (B_MN ? 128 : 2), p.idesc, k > k0 || q > 0);
                    tc_commit(empty + 8 * s);
                }
                if (ok) tc_commit(done + 8 * acc);
            }
        }
    } else {
        uint32_t u = 0;
        for (int t = blockIdx.x; t < total; t += gridDim.x, ++u) {
            int i, j, share;
            tile_at(p, t, i, j, share);
            const uint32_t acc = u & 1, at = tmem + acc * BN + ((uint32_t)warp << 21);
            if (!__all_sync(0xffffffffu, mbar_wait(done + 8 * acc, (u / 2) & 1, &stop))) break;
            tc_fence_after();
            const int64_t row_i = (int64_t)i * kBM + warp * 32 + lane;
            for (int c = 0; c < BN; c += 16) {
                uint32_t r[16];
                __syncwarp();
                tmem_ld16(at + c, r);
                tmem_wait_ld();
                if (row_i < p.I) put16<SWAP>(p, r, row_i, (int64_t)j * BN + c, share);
            }
            __syncwarp();
            tc_fence_before();
            mbar_arrive(drained + 8 * acc);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && stop) atomicMax(&g_status, (uint32_t)MLKV_ERR_TIMEOUT);
    if (warp == 5) tmem_free(tmem, R::kColumns);
}

// The shares of k added up in order, and the epilogue (shares == 0: of zeros).
__global__ void __launch_bounds__(256) k_product_finish(Epilogue e, int64_t rows, int64_t cols, int shares) {
    pdl_enter();
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < rows * cols; at += gridDim.x * 256ll) {
        const int64_t r = at / cols, c = at - r * cols;
        float v = 0.f;
        for (int s = 0; s < shares; ++s) v += e.part[s * e.part_size + r * e.part_stride + c];
        static_cast<uint16_t*>(e.out)[r * e.out_stride + c] = narrow(e.type, finish(e, v, r, c));
    }
}

// Rows whose stride or place TMA does not take (multiples of 16 bytes), laid out anew.
__global__ void __launch_bounds__(256) k_align(const uint16_t* __restrict__ in, int64_t stride, uint16_t* __restrict__ out,
                                               int64_t out_stride, int64_t rows, int64_t cols) {
    pdl_enter();
    const int64_t per = out_stride / 8;
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < rows * per; at += gridDim.x * 256ll) {
        const int64_t r = at / per, c = (at - r * per) * 8;
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (c + q < cols) w[q / 2] |= (uint32_t)in[r * stride + c + q] << (16 * (q & 1));
        *reinterpret_cast<uint4*>(out + r * out_stride + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// p = dy act'(z), and the sums of its columns over a block's rows.  A thread
// takes V columns, a block 32 V columns of a share of the rows.
struct Slope {
    const uint16_t* dy;
    const uint16_t* pre;
    uint16_t* p;       // null: not wanted (p is dy)
    float* part;       // [shares][cols], null with one share or no sums
    void* dbias;
    int64_t dy_stride, pre_stride, p_stride, rows, cols, share;
    int32_t type, act;
};
template <int V>
__global__ void __launch_bounds__(256) k_slope(Slope a) {
    pdl_enter();
    __shared__ float sums[8][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (blockIdx.x * 32ll + lane) * V;
    const int64_t r0 = blockIdx.y * a.share, r1 = min(a.rows, r0 + a.share);
    float s[V];
#pragma unroll
    for (int q = 0; q < V; ++q) s[q] = 0.f;
    if (c < a.cols)
        for (int64_t r = r0 + warp; r < r1; r += 8) {
            const Pack<uint16_t, V> d = *reinterpret_cast<const Pack<uint16_t, V>*>(a.dy + r * a.dy_stride + c);
            Pack<uint16_t, V> o = d;
            if (a.act != MLKV_ACT_NONE) {
                const Pack<uint16_t, V> z = *reinterpret_cast<const Pack<uint16_t, V>*>(a.pre + r * a.pre_stride + c);
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    const float v = widen(a.type, d.v[q]) * slope(a.act, widen(a.type, z.v[q]));
                    o.v[q] = narrow(a.type, v);
                    s[q] += v;
                }
            } else {
#pragma unroll
                for (int q = 0; q < V; ++q) s[q] += widen(a.type, d.v[q]);
            }
            if (a.p) *reinterpret_cast<Pack<uint16_t, V>*>(a.p + r * a.p_stride + c) = o;
        }
    if (!a.dbias) return;
#pragma unroll
    for (int q = 0; q < V; ++q) sums[warp][lane * V + q] = s[q];
    __syncthreads();
    for (int q = threadIdx.x; q < 32 * V; q += 256) {
        const int64_t col = blockIdx.x * 32ll * V + q;
        if (col >= a.cols) continue;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += sums[w][q];
        if (a.part) a.part[blockIdx.y * a.cols + col] = t;
        else static_cast<uint16_t*>(a.dbias)[col] = narrow(a.type, t);
    }
}
__global__ void __launch_bounds__(256) k_column_sums(const float* __restrict__ part, int shares, int64_t cols, void* out, int32_t type) {
    pdl_enter();
    const int64_t c = blockIdx.x * 256ll + threadIdx.x;
    if (c >= cols) return;
    float t = 0.f;
    for (int s = 0; s < shares; ++s) t += part[s * cols + c];
    static_cast<uint16_t*>(out)[c] = narrow(type, t);
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

    // The matrix as TMA takes it.
    Matrix aligned(const Matrix& m) {
        if (m.aligned()) return m;
        const int64_t stride = round_up(m.cols, 8);
        uint16_t* to = static_cast<uint16_t*>(arena.take(m.rows * stride * 2));
        if (run && m.rows)
            launch_kernel(true, k_align, dim3(blocks_for(m.rows * stride / 8)), dim3(256), 0, st, m.p, m.stride, to, stride, m.rows, m.cols);
        return {to, stride, m.rows, m.cols};
    }

    bool encode(CUtensorMap* map, const Matrix& m, bool mn, int rows) {
        const auto fn = tensor_map_encode();
        if (!fn) return false;
        const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows}, strides[1] = {(cuuint64_t)m.stride * 2};
        const cuuint32_t box[2] = {64, (cuuint32_t)(mn ? kBK : rows)}, step[2] = {1, 1};
        return fn(map, type == MLKV_TYPE_BFLOAT ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                  const_cast<uint16_t*>(m.p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }

    template <int BN, bool A_MN, bool B_MN, bool SWAP>
    void launch(const Matrix& a, const Matrix& b, Product p) {
        CUtensorMap ma, mb;
        auto kernel = k_product<BN, A_MN, B_MN, SWAP>;
        if (!encode(&ma, a, A_MN, kBM) || !encode(&mb, b, B_MN, BN) ||
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<BN>::kBytes) != cudaSuccess) {
            rc = MLKV_ERR_CUDA;
            return;
        }
        p.idesc = mma_desc(type == MLKV_TYPE_BFLOAT, A_MN, B_MN, kBM, BN);
        const int64_t tiles = (int64_t)p.tiles_i * p.tiles_j * p.shares;
        launch_kernel(true, kernel, dim3((unsigned)std::min<int64_t>(tiles, sms)), dim3(kThreads), Ring<BN>::kBytes, st, ma, mb, p);
    }

    // out = epilogue(A B^T): A [rows][k], B [cols][k]; *_mn: held as [k][rows], [k][cols].
    template <bool A_MN, bool B_MN>
    void product(Matrix a, Matrix b, int64_t rows, int64_t cols, int64_t k, Epilogue e) {
        if (!rows || !cols) return;
        e.type = type;
        if (k == 0) {
            if (run) launch_kernel(true, k_product_finish, dim3(blocks_for(rows * cols)), dim3(256), 0, st, e, rows, cols, 0);
            return;
        }
        a = aligned(a);
        b = aligned(b);
        e.wide = 1;
        auto wide = [](const void* p, int64_t stride) { return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0); };
        e.wide = wide(e.out, e.out_stride) && wide(e.pre, e.pre_stride) && wide(e.residual, e.residual_stride);
        const bool swap = !A_MN && rows <= 64;  // few rows: the wide operand fills the tiles' 128 rows
        const int bn = swap ? (rows <= 16 ? 16 : rows <= 32 ? 32 : 64) : cols <= 64 ? 64 : cols <= 128 ? 128 : 256;
        Product p = {};
        p.I = (int32_t)(swap ? cols : rows);
        p.J = (int32_t)(swap ? rows : cols);
        p.blocks = (int32_t)((k + kBK - 1) / kBK);
        p.tiles_i = (p.I + kBM - 1) / kBM;
        p.tiles_j = (p.J + bn - 1) / bn;
        if ((int64_t)p.tiles_i * p.tiles_j >= (int64_t)1 << 30) {
            rc = MLKV_ERR_UNSUPPORTED;
            return;
        }
        // too few tiles for the GPU: k in shares of at least 4 blocks
        const int64_t tiles = (int64_t)p.tiles_i * p.tiles_j;
        int64_t shares = std::max<int64_t>(1, std::min<int64_t>(sms / tiles, p.blocks / 4));
        p.blocks_per_share = (int32_t)((p.blocks + shares - 1) / shares);
        p.shares = (p.blocks + p.blocks_per_share - 1) / p.blocks_per_share;
        p.e = e;
        if (p.shares > 1) {
            p.e.part_stride = cols;
            p.e.part_size = rows * cols;
            p.e.part = static_cast<float*>(arena.take(p.shares * p.e.part_size * 4));
        }
        if (!run) return;
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
            else launch<256, A_MN, B_MN, false>(a, b, p);
        }
        if (p.shares > 1) {
            Epilogue f = p.e;
            launch_kernel(true, k_product_finish, dim3(blocks_for(rows * cols)), dim3(256), 0, st, f, rows, cols, (int)p.shares);
        }
    }

    void forward(const mlkv_linear_args& g) {
        Epilogue e = {};
        e.bias = g.d_bias; e.residual = g.d_residual; e.residual_stride = g.residual_stride;
        e.pre = g.d_pre; e.pre_stride = g.pre_stride; e.out = g.d_y; e.out_stride = g.y_stride; e.act = g.activation;
        product<false, false>({(const uint16_t*)g.d_x, g.x_stride, g.m, g.k}, {(const uint16_t*)g.d_weight, g.weight_stride, g.n, g.k},
                              g.m, g.n, g.k, e);
    }

    void backward(const mlkv_linear_args& g) {
        Matrix p = {(const uint16_t*)g.d_dy, g.dy_stride, g.m, g.n};
        const bool act = g.activation != MLKV_ACT_NONE, products = (g.d_dx || g.d_dweight) && g.m && g.n;
        const bool copy = products && (act || !p.aligned());
        if (g.m && g.n && (copy || g.d_dbias)) {
            Slope s = {};
            s.dy = p.p; s.dy_stride = g.dy_stride; s.pre = (const uint16_t*)g.d_pre; s.pre_stride = g.pre_stride;
            s.rows = g.m; s.cols = g.n; s.type = type; s.act = g.activation; s.dbias = g.d_dbias;
            if (copy) {
                s.p_stride = round_up(g.n, 8);
                s.p = static_cast<uint16_t*>(arena.take(g.m * s.p_stride * 2));
                p = {s.p, s.p_stride, g.m, g.n};
            }
            const Matrix dy = {s.dy, s.dy_stride, 0, 0}, pre = {s.pre, s.pre_stride, 0, 0};
            const int V = g.n % 8 == 0 && dy.aligned() && (!act || pre.aligned()) ? 8 : 1;
            const int64_t across = (g.n + 32 * V - 1) / (32 * V);
            const int64_t shares = std::max<int64_t>(1, std::min<int64_t>((g.m + 31) / 32, 8ll * sms / across));
            s.share = (g.m + shares - 1) / shares;
            const unsigned down = (unsigned)((g.m + s.share - 1) / s.share);
            if (g.d_dbias && down > 1) s.part = static_cast<float*>(arena.take((int64_t)down * g.n * 4));
            if (run) {
                const dim3 grid((unsigned)across, down);
                if (V == 8) launch_kernel(true, k_slope<8>, grid, dim3(256), 0, st, s);
                else launch_kernel(true, k_slope<1>, grid, dim3(256), 0, st, s);
                if (s.part) launch_kernel(true, k_column_sums, dim3((unsigned)((g.n + 255) / 256)), dim3(256), 0, st,
                                          (const float*)s.part, (int)down, g.n, g.d_dbias, type);
            }
        } else if (run && g.d_dbias && g.n) {
            if (cudaMemsetAsync(g.d_dbias, 0, g.n * 2, st) != cudaSuccess) rc = MLKV_ERR_CUDA;
        }
        Epilogue e = {};
        if (g.d_dx) {
            e.out = g.d_dx; e.out_stride = g.dx_stride;
            product<false, true>(p, {(const uint16_t*)g.d_weight, g.weight_stride, g.n, g.k}, g.m, g.k, g.n, e);
        }
        if (g.d_dweight) {
            e.out = g.d_dweight; e.out_stride = g.dweight_stride;
            product<true, true>(p, {(const uint16_t*)g.d_x, g.x_stride, g.m, g.k}, g.n, g.k, g.m, e);
        }
    }
};

bool rows_ok(const void* p, int64_t stride, int64_t rows, int64_t cols, bool may_be_null) {
    if (!p) return may_be_null || rows == 0 || cols == 0;
    return stride >= cols && stride < (int64_t)1 << 38;  // (TMA's strides have 40 bits)
}
bool linear_ok(const mlkv_linear_args* g) {
    if (!g || g->m < 0 || g->n < 0 || g->k < 0) return false;
    if (std::max(g->m, std::max(g->n, g->k)) >= (int64_t)1 << 31) return false;
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
    uint32_t status = 0;
    const uint32_t none = 0;
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess ||
        cudaMemcpyFromSymbol(&status, g_status, sizeof(status)) != cudaSuccess)
        return MLKV_ERR_CUDA;
    if (status && cudaMemcpyToSymbol(g_status, &none, sizeof(none)) != cudaSuccess) return MLKV_ERR_CUDA;
    return (int)status;
}
