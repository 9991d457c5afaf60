// The layer norm's forward pass (mlkv_layer_norm).
//
//   y = (x - mu) r w + b,   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps)
//
// Bound by HBM: a few operations per value.  The variance is that of the centred
// values, a second pass over registers: as exact for rows far from 0 as for any.
#include "dense_norm.cuh"

using namespace mlkv;

namespace {

constexpr int kForwardValues = 32;  // most values a lane holds

template <class TX, class TY, int V, int NV>
__global__ void __launch_bounds__(kNormLanes) k_norm(NormArgs a) {
    pdl_enter();
    __shared__ float2 buf[64];
    const Team tm(a.lanes);
    const int64_t r = (int64_t)blockIdx.x * tm.count + tm.index;
    const bool live = r < a.rows;
    const TX* x = static_cast<const TX*>(a.x) + r * a.x_stride;
    const int nvec = a.dim / V;
    Pack<TX, V> q[NV];
    float s = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = tm.lane + i * tm.L;
        q[i] = live && j < nvec ? load_pack<TX, V>(x + j * V) : zero_pack<TX, V>();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) s += to_float(q[i].v[e]);
    tm.sum(s, none, buf, 0);
    const float mu = s / (float)a.dim;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (tm.lane + i * tm.L >= nvec) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = to_float(q[i].v[e]) - mu;
            v += d * d;
        }
    }
    tm.sum(v, none, buf, 1);
    const float rs = 1.f / sqrtf(v / (float)a.dim + a.eps);
    if (!live) return;
    if (a.stats && tm.lane == 0) {
        a.stats[2 * r] = mu;
        a.stats[2 * r + 1] = rs;
    }
    TY* y = static_cast<TY*>(a.out) + r * a.out_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = tm.lane + i * tm.L;
        if (j >= nvec) continue;
        float w[V], b[V];
        if (a.w) load_weights<V>(a.w, a.w_type, j * V, w);
        if (a.b) load_weights<V>(a.b, a.w_type, j * V, b);
        Pack<TY, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float t = (to_float(q[i].v[e]) - mu) * rs;
            if (a.w) t *= w[e];
            if (a.b) t += b[e];
            o.v[e] = from_float<TY>(t);
        }
        *reinterpret_cast<Pack<TY, V>*>(y + j * V) = o;
    }
}

// Rows too long for registers: a block a row, read three times (from L2 but for the first).
template <class TX, class TY>
__global__ void __launch_bounds__(kNormLongLanes) k_norm_long(NormArgs a) {
    pdl_enter();
    __shared__ float2 buf[64];
    const Team tm(kNormLongLanes);
    const TX* x = static_cast<const TX*>(a.x) + blockIdx.x * a.x_stride;
    float s = 0.f, none = 0.f, v = 0.f;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) s += to_float(x[j]);
    tm.sum(s, none, buf, 0);
    const float mu = s / (float)a.dim;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        const float d = to_float(x[j]) - mu;
        v += d * d;
    }
    tm.sum(v, none, buf, 1);
    const float rs = 1.f / sqrtf(v / (float)a.dim + a.eps);
    if (a.stats && tm.lane == 0) {
        a.stats[2 * blockIdx.x] = mu;
        a.stats[2 * blockIdx.x + 1] = rs;
    }
    TY* y = static_cast<TY*>(a.out) + blockIdx.x * a.out_stride;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        float t = (to_float(x[j]) - mu) * rs;
        if (a.w) t *= load_as_float(a.w, a.w_type, j);
        if (a.b) t += load_as_float(a.b, a.w_type, j);
        y[j] = from_float<TY>(t);
    }
}

}  // namespace

extern "C" int mlkv_layer_norm(const void* d_x, int64_t x_stride, int32_t x_type, int64_t rows, int64_t dim,
                               const void* d_weight, const void* d_bias, int32_t w_type, float eps, void* d_y,
                               int64_t y_stride, int32_t y_type, float* d_stats, void* stream) {
    MLKV_DENSE_RANGE("mlkv_layer_norm");
    if (!norm_ok(d_x, x_stride, x_type, y_type, w_type, rows, dim) || !(eps >= 0.f)) return MLKV_ERR_INVALID;
    if (rows == 0) return MLKV_OK;
    if (!d_y || y_stride < dim) return MLKV_ERR_INVALID;
    NormArgs a = {};
    a.x = d_x; a.out = d_y; a.w = d_weight; a.b = d_bias; a.stats = d_stats;
    a.x_stride = x_stride; a.out_stride = y_stride; a.rows = rows; a.dim = (int32_t)dim; a.w_type = w_type; a.eps = eps;
    const int xs = dense_type_size(x_type), ys = dense_type_size(y_type), ws = dense_type_size(w_type);
    const int V = norm_vector_width(dim, {{d_x, xs}, {d_y, ys}, {d_weight, ws}, {d_bias, ws}}, {x_stride, y_stride}, 16 / xs);
    const NormShape sh = norm_shape(dim, V, kForwardValues);
    cudaStream_t st = (cudaStream_t)stream;
    by_types(x_type, y_type, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        if (!sh.lanes) {
            launch_kernel(true, k_norm_long<TX, TY>, dim3((unsigned)rows), dim3(kNormLongLanes), 0, st, a);
            return;
        }
        a.lanes = sh.lanes;
        const int threads = norm_team_threads(sh.lanes), teams = threads / sh.lanes;
        by_width<TX, kForwardValues>(V, sh.NV, [&](auto v, auto nv) {
            launch_kernel(true, k_norm<TX, TY, decltype(v)::value, decltype(nv)::value>,
                          dim3((unsigned)((rows + teams - 1) / teams)), dim3(threads), 0, st, a);
        });
    });
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

