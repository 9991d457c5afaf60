// The layer norm's forward pass (mlkv_layer_norm).
//
//   y = (x - mu) r w + b,   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps)
//
// Bound by HBM: a few operations per value.  65,536 rows of 2,048 bf16 values take
// 89 us (6.0 TB/s), 200,003 of 100 fp32 values into bf16 27 (4.5: rows of 25
// vectors leave 7 of 32 lanes' places empty), 416 of 128 fp32 values 3.6.  The variance is that of the centred
// values, a second pass over registers: as exact for rows far from 0 as for any.
#include "dense_norm.cuh"

using namespace mlkv;

namespace {

constexpr int kForwardValues = 32;  // most values a lane holds
constexpr int kForwardLanes = 256;   // a block's threads
constexpr int kForwardBlocks = 3;    // blocks an SM: 80 registers a thread

// A block's teams take rows in turn; the weights are staged once a block.  Rows
// come through shared memory, the next one or two of each team on their way (a
// thread reads what it copied itself).  What a lane holds beyond the row's end is
// a copy of its last vector, or 0, left out of the sums.
template <class TX, class TY, int NV, bool ALIGNED>
__global__ void __launch_bounds__(kForwardLanes, kForwardBlocks) k_norm(NormArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) float weights[];  // [2][room]; then the rows on their way
    __shared__ __align__(16) float2 buf[64];
    constexpr int V = 16 / sizeof(TX), H = V / 2;
    const Team tm(a.lanes, buf);
    const int rows = (int)a.rows, step = (int)gridDim.x * tm.count;
    const int nvec = (a.dim + V - 1) / V, room = tm.L * NV * V;
    const Span span(static_cast<const TX*>(a.x), a.rows, a.x_stride, a.dim);
    int at[NV];  // of this lane's vectors, the last one again where there are no more
#pragma unroll
    for (int i = 0; i < NV; ++i) at[i] = min(tm.lane + i * tm.L, nvec - 1) * V;
    using Row = Values<TX, V, ALIGNED>;
    const RowRing<TX, V, NV, ALIGNED> ring(reinterpret_cast<uint8_t*>(weights + 2 * room), tm, room);
    int r = (int)blockIdx.x * tm.count + tm.index, ahead = r;
    const TX* x = static_cast<const TX*>(a.x) + r * a.x_stride;
    TY* y = static_cast<TY*>(a.out) + r * a.out_stride;
    const int64_t x_step = step * a.x_stride, y_step = step * a.out_stride;
    uint32_t by = (uint32_t)reinterpret_cast<uintptr_t>(x) & 15;  // of the row worked on
    // the next row not yet on its way, into slot `slot`
    auto fetch = [&](int slot) {
        if (ahead < rows) ring.fetch(tm, slot, x, at, a.dim, span);
        copy_commit();
        x += x_step;
        ahead += step;
    };
    for (int i = 0; i < kNormAhead; ++i) fetch(i);
    stage_weights<V>(weights, a.w, a.w_type, a.dim, room, 1.f);
    stage_weights<V>(weights + room, a.b, a.w_type, a.dim, room, 0.f);
    __syncthreads();
    const float inverse = 1.f / (float)a.dim;
    int slot = 0;
    // the lanes of a warp take as many turns as its first team does
    for (int first = tm.L < 32 ? r - (int)(threadIdx.x & 31) / tm.L : r; first < rows; first += step, r += step, y += y_step, slot ^= 1) {
        float2 f[NV][H], s = both(0.f), v = both(0.f);
        copy_wait<kNormAhead - 1>();
        if (!ALIGNED) tm.sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Row q;
            ring.take(q, slot, i, at[i], by, a.dim);
#pragma unroll
            for (int k = 0; k < H; ++k) f[i][k] = q.pair(k);
            if (tm.lane + i * tm.L < nvec)
#pragma unroll
                for (int k = 0; k < H; ++k) s = add2(s, f[i][k]);
        }
        const float mu = tm.sum(s.x + s.y, 0) * inverse;
        if (!ALIGNED) __syncwarp();  // (a team of a warp or less: all have read the row)
        fetch(slot);
        by = (by + (uint32_t)(x_step * sizeof(TX))) & 15;
        const float2 minus = both(-mu);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
#pragma unroll
            for (int k = 0; k < H; ++k) f[i][k] = add2(f[i][k], minus);
            if (!ALIGNED && j == nvec - 1)
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    if (j * V + 2 * k >= a.dim) f[i][k].x = 0.f;
                    if (j * V + 2 * k + 1 >= a.dim) f[i][k].y = 0.f;
                }
            if (j < nvec)
#pragma unroll
                for (int k = 0; k < H; ++k) v = fma2(f[i][k], f[i][k], v);
        }
        const float rs = 1.f / sqrtf(tm.sum(v.x + v.y, 1) * inverse + a.eps);
        if (r < rows) {
            if (a.stats && tm.lane == 0) reinterpret_cast<float2*>(a.stats)[r] = make_float2(mu, rs);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = tm.lane + i * tm.L;
                float2 w[H], b[H];
                weight_pairs<V>(weights, j, room, w);
                weight_pairs<V>(weights + room, j, room, b);
                Values<TY, V, ALIGNED> o;
#pragma unroll
                for (int k = 0; k < H; ++k) o.set(k, fma2(mul2(f[i][k], both(rs)), w[k], b[k]));
                if (j < nvec) o.store(y + j * V, a.dim - j * V);
            }
        }
    }
}

// Rows too long for registers (8,192 values): a block a row, read three times (from L2 but for the first).
template <class TX, class TY>
__global__ void __launch_bounds__(kNormLongLanes) k_norm_long(NormArgs a) {
    pdl_enter();
    __shared__ __align__(16) float2 buf[64];
    const Team tm(kNormLongLanes, buf);
    __syncthreads();
    const TX* x = static_cast<const TX*>(a.x) + blockIdx.x * a.x_stride;
    float s = 0.f, none = 0.f, v = 0.f;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) s += to_float(x[j]);
    tm.sum(s, none, 0);
    const float mu = s / (float)a.dim;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        const float d = to_float(x[j]) - mu;
        v += d * d;
    }
    tm.sum(v, none, 1);
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
    const int V = 16 / xs;
    const bool aligned = norm_aligned(d_x, x_stride, xs, dim, V) && norm_aligned(d_y, y_stride, ys, dim, V);
    cudaStream_t st = (cudaStream_t)stream;
    const int sms = dense_sms();
    if (!sms) return MLKV_ERR_CUDA;
    const NormShape sh = norm_shape(rows, dim, V, kForwardValues, kForwardLanes, sms);
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
        const int room = sh.lanes * sh.NV * V;
        const size_t smem = 2 * (size_t)room * sizeof(float) +
                            kNormAhead * (aligned ? (size_t)sh.NV * threads * 16 : (size_t)teams * norm_row(room, xs));
        const int64_t resident = std::max<int64_t>(1, std::min<int64_t>(kForwardBlocks, kDenseSmem / (int64_t)(smem + 2048)));
        const unsigned blocks = (unsigned)std::min<int64_t>(sms * resident, (rows + teams - 1) / teams);
        by_shape<kForwardValues * (int)sizeof(TX) / 16>(sh.NV, aligned, [&](auto nv, auto al) {
            auto kernel = k_norm<TX, TY, decltype(nv)::value, decltype(al)::value>;
            ok = dense_smem(kernel, smem);
            if (ok) launch_kernel(true, kernel, dim3(blocks), dim3(threads), smem, st, a);
        });
    });
    return ok && cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

