// The layer norm's forward pass (mlkv_layer_norm).
//
//   y = (x - mu) r w + b,   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps)
//
// Bound by HBM: a few operations per value.  The variance is that of the centred
// values, a second pass over registers: as exact for rows far from 0 as for any.
#include "dense_norm.cuh"

using namespace mlkv;

namespace {

// Most values a lane holds.  (65,536 rows of 2,048 in bf16: as fast with 64, which spills.)
constexpr int kForwardValues = 32;

// A block's teams take rows in turn; the weights are staged once a block.
template <class TX, class TY, int V, int NV>
__global__ void __launch_bounds__(kNormLanes, 2) k_norm(NormArgs a) {
    pdl_enter();
    extern __shared__ float weights[];  // [2][dim]
    __shared__ float2 buf[64];
    constexpr int H = kPairs<V>;
    const Team tm(a.lanes);
    const int64_t step = (int64_t)gridDim.x * tm.count;
    const int nvec = a.dim / V;
    Values<TX, V> q[NV];
    auto load = [&](int64_t r) {
        const TX* x = static_cast<const TX*>(a.x) + r * a.x_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
            q[i].zero();
            if (r < a.rows && j < nvec) q[i].load(x + j * V);
        }
    };
    int64_t r = (int64_t)blockIdx.x * tm.count + tm.index;
    load(r);
    if (a.w) stage_weights<V>(weights, a.w, a.w_type, a.dim);
    if (a.b) stage_weights<V>(weights + a.dim, a.b, a.w_type, a.dim);
    if (a.w || a.b) __syncthreads();
    // the lanes of a warp take as many turns as its first team does
    for (int64_t first = tm.L < 32 ? r - (threadIdx.x & 31) / tm.L : r; first < a.rows; first += step, r += step) {
        const bool live = r < a.rows;
        float2 s = both(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < H; ++k) s = add2(s, q[i].pair(k));
        const float mu = tm.sum(s.x + s.y, buf, 0) / (float)a.dim;
        const float2 minus = both(-mu);
        float2 v = both(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (tm.lane + i * tm.L >= nvec) continue;
#pragma unroll
            for (int k = 0; k < H; ++k) {
                float2 d = add2(q[i].pair(k), minus);
                if (V == 1) d.y = 0.f;
                v = fma2(d, d, v);
            }
        }
        const float rs = 1.f / sqrtf(tm.sum(v.x + v.y, buf, 1) / (float)a.dim + a.eps);
        if (live) {
            if (a.stats && tm.lane == 0) *reinterpret_cast<float2*>(a.stats + 2 * r) = make_float2(mu, rs);
            TY* y = static_cast<TY*>(a.out) + r * a.out_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = tm.lane + i * tm.L;
                if (j >= nvec) continue;
                float2 w[H], b[H];
                if (a.w) weight_pairs<V>(weights, j, a.dim, w);
                if (a.b) weight_pairs<V>(weights + a.dim, j, a.dim, b);
                Values<TY, V> o;
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    float2 t = mul2(add2(q[i].pair(k), minus), both(rs));
                    if (a.w && a.b) t = fma2(t, w[k], b[k]);
                    else if (a.w) t = mul2(t, w[k]);
                    else if (a.b) t = add2(t, b[k]);
                    o.set(k, t);
                }
                o.store(y + j * V);
            }
        }
        load(r + step);
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
    const int xs = dense_type_size(x_type), ys = dense_type_size(y_type);
    const int V = norm_vector_width(dim, {{d_x, xs}, {d_y, ys}}, {x_stride, y_stride}, 16 / xs);
    const NormShape sh = norm_shape(dim, V, kForwardValues);
    cudaStream_t st = (cudaStream_t)stream;
    const int sms = dense_sms();
    if (!sms) return MLKV_ERR_CUDA;
    bool ok = true;
    by_types(x_type, y_type, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        if (!sh.lanes) {
            launch_kernel(true, k_norm_long<TX, TY>, dim3((unsigned)rows), dim3(kNormLongLanes), 0, st, a);
            return;
        }
        a.lanes = sh.lanes;
        const int threads = norm_team_threads(sh.lanes), teams = threads / sh.lanes;
        const size_t smem = d_weight || d_bias ? 2 * (size_t)dim * sizeof(float) : 0;
        const int64_t resident = std::max<int64_t>(1, std::min<int64_t>(1024 / threads, (200 << 10) / (smem + 1)));
        const unsigned blocks = (unsigned)std::min<int64_t>(sms * resident, (rows + teams - 1) / teams);
        by_width<TX, kForwardValues>(V, sh.NV, [&](auto v, auto nv) {
            auto kernel = k_norm<TX, TY, decltype(v)::value, decltype(nv)::value>;
            ok = dense_smem(kernel, smem);
            if (ok) launch_kernel(true, kernel, dim3(blocks), dim3(threads), smem, st, a);
        });
    });
    return ok && cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

