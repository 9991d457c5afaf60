// The layer norm's gradients (mlkv_layer_norm_backward).
//
//   dx = r (g - mean(g) - xh mean(g xh)),   g = dy w,  xh = (x - mu) r
//   dw = sum over rows of dy xh,            db = sum over rows of dy
//
// Bound by HBM: x and dy are read once, dx written once.  dw and db are added up
// in registers, in 32 bits, over the rows that a team takes, then over a block's
// teams, then (k_norm_cols) over the blocks, each in a fixed order.
#include "dense_norm.cuh"

using namespace mlkv;

namespace {

constexpr int kBackwardValues = 16;  // most values of x and dy each that a lane holds, beside their columns' sums

// The rows' gradients, and the sums over this block's rows of dy xh and dy.
template <class TX, class TY, int V, int NV>
__global__ void __launch_bounds__(kNormLanes) k_norm_backward(NormArgs a) {
    pdl_enter();
    extern __shared__ float cols[];  // [2][dim], where a block has several teams
    __shared__ float2 buf[64];
    const Team tm(a.lanes);
    const int nvec = a.dim / V;
    float dw[NV][V], db[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) dw[i][e] = db[i][e] = 0.f;
    const int64_t step = (int64_t)gridDim.x * tm.count;
    Pack<TX, V> x[NV];
    Pack<TY, V> dy[NV];
    float mu = 0.f, rs = 0.f;
    auto load = [&](int64_t r) {
        const bool live = r < a.rows;
        const TX* xr = static_cast<const TX*>(a.x) + r * a.x_stride;
        const TY* dr = static_cast<const TY*>(a.dy) + r * a.dy_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
            x[i] = live && j < nvec ? load_pack<TX, V>(xr + j * V) : zero_pack<TX, V>();
            dy[i] = live && j < nvec ? load_pack<TY, V>(dr + j * V) : zero_pack<TY, V>();
        }
        mu = live ? a.stats[2 * r] : 0.f;
        rs = live ? a.stats[2 * r + 1] : 0.f;
    };
    int64_t r = (int64_t)blockIdx.x * tm.count + tm.index;
    load(r);
    int turn = 0;
    // every team of the block takes as many turns (the sums' barriers)
    for (int64_t first = (int64_t)blockIdx.x * tm.count; first < a.rows; first += step, r += step, turn ^= 1) {
        float c1 = 0.f, c2 = 0.f;
        float xh[NV][V], g[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
            float w[V];
            if (a.w && j < nvec) load_weights<V>(a.w, a.w_type, j * V, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = to_float(dy[i].v[e]);
                xh[i][e] = (to_float(x[i].v[e]) - mu) * rs;
                g[i][e] = a.w && j < nvec ? d * w[e] : d;
                c1 += g[i][e];
                c2 += g[i][e] * xh[i][e];
                dw[i][e] += d * xh[i][e];
                db[i][e] += d;
            }
        }
        const float rs_now = rs;
        load(r + step);
        if (!a.out) continue;
        tm.sum(c1, c2, buf, turn);
        c1 /= (float)a.dim;
        c2 /= (float)a.dim;
        if (r >= a.rows) continue;
        TX* o = static_cast<TX*>(a.out) + r * a.out_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
            if (j >= nvec) continue;
            Pack<TX, V> q;
#pragma unroll
            for (int e = 0; e < V; ++e) q.v[e] = from_float<TX>(rs_now * (g[i][e] - c1 - xh[i][e] * c2));
            *reinterpret_cast<Pack<TX, V>*>(o + j * V) = q;
        }
    }
    if (!a.part && !a.dweight && !a.dbias) return;
    // the lanes of a warp that hold the same columns
    for (int o = 16; o >= tm.L; o >>= 1)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dw[i][e] += __shfl_xor_sync(0xffffffffu, dw[i][e], o);
                db[i][e] += __shfl_xor_sync(0xffffffffu, db[i][e], o);
            }
    // ... then the block's teams (a warp's, where it holds several), one after another
    const int teams = tm.L < 32 ? blockDim.x / 32 : tm.count, mine = tm.L < 32 ? threadIdx.x / 32 : tm.index;
    const bool holds = tm.L >= 32 || (threadIdx.x & 31) < tm.L;
    for (int t = 0; t < teams - 1; ++t) {
        if (mine == t && holds)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = tm.lane + i * tm.L;
                if (j >= nvec) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float before_w = t ? cols[j * V + e] : 0.f, before_b = t ? cols[a.dim + j * V + e] : 0.f;
                    cols[j * V + e] = before_w + dw[i][e];
                    cols[a.dim + j * V + e] = before_b + db[i][e];
                }
            }
        __syncthreads();
    }
    if (mine != teams - 1 || !holds) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = tm.lane + i * tm.L;
        if (j >= nvec) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = j * V + e;
            const float sw = dw[i][e] + (teams > 1 ? cols[c] : 0.f), sb = db[i][e] + (teams > 1 ? cols[a.dim + c] : 0.f);
            if (a.part) {
                a.part[(int64_t)blockIdx.x * 2 * a.dim + c] = sw;
                a.part[(int64_t)blockIdx.x * 2 * a.dim + a.dim + c] = sb;
            } else {
                if (a.dweight) store_as(a.dweight, a.w_type, c, sw);
                if (a.dbias) store_as(a.dbias, a.w_type, c, sb);
            }
        }
    }
}

// Rows too long for registers: a block a row ...
template <class TX, class TY>
__global__ void __launch_bounds__(kNormLongLanes) k_norm_backward_long(NormArgs a) {
    pdl_enter();
    __shared__ float2 buf[64];
    const Team tm(kNormLongLanes);
    const TX* x = static_cast<const TX*>(a.x) + blockIdx.x * a.x_stride;
    const TY* dy = static_cast<const TY*>(a.dy) + blockIdx.x * a.dy_stride;
    const float mu = a.stats[2 * blockIdx.x], rs = a.stats[2 * blockIdx.x + 1];
    float c1 = 0.f, c2 = 0.f;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        const float g = to_float(dy[j]) * (a.w ? load_as_float(a.w, a.w_type, j) : 1.f);
        c1 += g;
        c2 += g * ((to_float(x[j]) - mu) * rs);
    }
    tm.sum(c1, c2, buf, 0);
    c1 /= (float)a.dim;
    c2 /= (float)a.dim;
    TX* o = static_cast<TX*>(a.out) + blockIdx.x * a.out_stride;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        const float g = to_float(dy[j]) * (a.w ? load_as_float(a.w, a.w_type, j) : 1.f);
        o[j] = from_float<TX>(rs * (g - c1 - (to_float(x[j]) - mu) * rs * c2));
    }
}

// ... and a thread a column of a share of the rows.
template <class TX, class TY>
__global__ void __launch_bounds__(128) k_norm_cols_long(NormArgs a, int64_t share) {
    pdl_enter();
    const int j = blockIdx.x * 128 + threadIdx.x;
    if (j >= a.dim) return;
    const int64_t r0 = blockIdx.y * share, r1 = min(a.rows, r0 + share);
    float dw = 0.f, db = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float d = to_float(static_cast<const TY*>(a.dy)[r * a.dy_stride + j]);
        dw += d * ((to_float(static_cast<const TX*>(a.x)[r * a.x_stride + j]) - a.stats[2 * r]) * a.stats[2 * r + 1]);
        db += d;
    }
    a.part[(int64_t)blockIdx.y * 2 * a.dim + j] = dw;
    a.part[(int64_t)blockIdx.y * 2 * a.dim + a.dim + j] = db;
}

// dweight and dbias: the blocks' sums of 32 columns, added up by 32 warps of
// which each takes every 32nd block, then over the warps.
__global__ void __launch_bounds__(1024) k_norm_cols(const float* __restrict__ part, int blocks, int dim, void* dweight,
                                                    void* dbias, int32_t w_type) {
    pdl_enter();
    __shared__ float s[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    float t = 0.f;
    if (c < 2 * dim)
        for (int b = w; b < blocks; b += 32) t += part[(int64_t)b * 2 * dim + c];
    s[w][threadIdx.x & 31] = t;
    __syncthreads();
    t = group_sum(s[threadIdx.x & 31][w], 32);  // warp w: column w of the block's
    const int o = blockIdx.x * 32 + w;
    if ((threadIdx.x & 31) == 0 && o < 2 * dim) {
        if (o < dim && dweight) store_as(dweight, w_type, o, t);
        if (o >= dim && dbias) store_as(dbias, w_type, o - dim, t);
    }
}

// Blocks whose sums of columns are kept apart: as many as run at a time.
int64_t backward_blocks(int64_t rows, int teams, int sms, int threads) {
    const int64_t most = (int64_t)sms * std::max(1, 1024 / threads);
    return std::max<int64_t>(1, std::min(most, (rows + teams - 1) / teams));
}
constexpr int64_t kMostBlocks = 256 * 8;  // of any device

}  // namespace

extern "C" int64_t mlkv_layer_norm_backward_workspace(int64_t rows, int64_t dim) {
    if (rows < 0 || rows >= (int64_t)1 << 31 || dim < 1 || dim >= kNormMaxDim) return -1;
    return std::min(kMostBlocks, std::max<int64_t>(rows, 1)) * 2 * dim * (int64_t)sizeof(float);
}

extern "C" int mlkv_layer_norm_backward(const void* d_dy, int64_t dy_stride, int32_t dy_type, const void* d_x,
                                        int64_t x_stride, int32_t x_type, int64_t rows, int64_t dim,
                                        const void* d_weight, int32_t w_type, const float* d_stats, void* d_dx,
                                        int64_t dx_stride, void* d_dweight, void* d_dbias, void* d_workspace,
                                        int64_t workspace_bytes, void* stream) {
    MLKV_DENSE_RANGE("mlkv_layer_norm_backward");
    if (!norm_ok(d_x, x_stride, x_type, dy_type, w_type, rows, dim)) return MLKV_ERR_INVALID;
    if (rows > 0 && (!d_dy || dy_stride < dim || !d_stats || (d_dx && dx_stride < dim))) return MLKV_ERR_INVALID;
    cudaStream_t st = (cudaStream_t)stream;
    if (rows == 0) {
        const size_t bytes = (size_t)dim * dense_type_size(w_type);
        if (d_dweight && cudaMemsetAsync(d_dweight, 0, bytes, st) != cudaSuccess) return MLKV_ERR_CUDA;
        if (d_dbias && cudaMemsetAsync(d_dbias, 0, bytes, st) != cudaSuccess) return MLKV_ERR_CUDA;
        return MLKV_OK;
    }
    const bool want_cols = d_dweight || d_dbias;
    if (!d_dx && !want_cols) return MLKV_OK;
    const int sms = dense_sms();
    if (!sms) return MLKV_ERR_CUDA;
    NormArgs a = {};
    a.x = d_x; a.dy = d_dy; a.out = d_dx; a.w = d_weight; a.stats = const_cast<float*>(d_stats);
    a.x_stride = x_stride; a.dy_stride = dy_stride; a.out_stride = dx_stride; a.rows = rows;
    a.dim = (int32_t)dim; a.w_type = w_type; a.dweight = d_dweight; a.dbias = d_dbias;
    const int xs = dense_type_size(x_type), ys = dense_type_size(dy_type), ws = dense_type_size(w_type);
    const int V = norm_vector_width(dim, {{d_x, xs}, {d_dy, ys}, {d_dx, xs}, {d_weight, ws}},
                               {x_stride, dy_stride, d_dx ? dx_stride : 0}, 16 / xs);
    const NormShape sh = norm_shape(dim, V, kBackwardValues);
    const int threads = sh.lanes ? norm_team_threads(sh.lanes) : kNormLongLanes, teams = sh.lanes ? threads / sh.lanes : 1;
    int64_t blocks = std::min(kMostBlocks, backward_blocks(rows, teams, sms, threads));
    if (!sh.lanes) blocks = std::max<int64_t>(1, std::min<int64_t>(rows, (2 * sms * 128 + dim - 1) / dim));
    const bool parts = want_cols && (blocks > 1 || !sh.lanes);
    if (parts && (!d_workspace || workspace_bytes < blocks * 2 * dim * (int64_t)sizeof(float))) return MLKV_ERR_INVALID;
    a.part = parts ? static_cast<float*>(d_workspace) : nullptr;
    by_types(x_type, dy_type, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        if (!sh.lanes) {
            if (want_cols) {  // first: the rows' gradients may overwrite dy
                const int64_t share = (rows + blocks - 1) / blocks;
                launch_kernel(true, k_norm_cols_long<TX, TY>, dim3((unsigned)((dim + 127) / 128), (unsigned)blocks),
                              dim3(128), 0, st, a, share);
            }
            if (d_dx)
                launch_kernel(true, k_norm_backward_long<TX, TY>, dim3((unsigned)rows), dim3(kNormLongLanes), 0, st, a);
            return;
        }
        a.lanes = sh.lanes;
        by_width<TX, kBackwardValues>(V, sh.NV, [&](auto v, auto nv) {
            auto kernel = k_norm_backward<TX, TY, decltype(v)::value, decltype(nv)::value>;
            const size_t smem = sh.lanes < threads ? 2 * (size_t)dim * sizeof(float) : 0;
            launch_kernel(true, kernel, dim3((unsigned)blocks), dim3(threads), smem, st, a);
        });
    });
    if (parts)
        launch_kernel(true, k_norm_cols, dim3((unsigned)((2 * dim + 31) / 32)), dim3(1024), 0, st,
                      (const float*)d_workspace, (int)blocks, (int)dim, d_dweight, d_dbias, w_type);
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}
