// The layer norm's gradients (mlkv_layer_norm_backward).
//
//   dx = r (g - mean(g) - xh mean(g xh)),   g = dy w,  xh = (x - mu) r
//   dw = sum over rows of dy xh,            db = sum over rows of dy
//
// Bound by HBM: x and dy are read once, dx written once.  65,536 rows of 2,048
// bf16 values take 131 us (6.1 TB/s), 200,003 of 100 fp32 values with bf16 dy 39.5 (5.1).  dw and db are added up
// in registers, in 32 bits, over the rows that a team takes, then over a block's
// teams, then (k_norm_cols) over the blocks, each in a fixed order.
#include "dense_norm.cuh"

using namespace mlkv;

namespace {

constexpr int kBackwardValues = 16;  // most values of x and dy each that a lane holds, beside their columns' sums
constexpr int kBackwardLanes = 512;  // threads an SM: 128 registers each

// The rows' gradients, and the sums over this block's rows of dy xh and dy.  Rows
// come through shared memory, the next one or two of each team on their way (a
// thread reads what it copied itself).  What a lane holds beyond the row's end is a copy of its last vector, left out of
// the sums, or, within that vector, 0.
template <class TX, class TY, int NV, bool ALIGNED>
__global__ void __launch_bounds__(kBackwardLanes, 1) k_norm_backward(NormArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) float shared[];  // the weight, [room]; the rows on their way; the teams' sums, [2][dim]
    __shared__ __align__(16) float2 buf[64];
    constexpr int V = 16 / sizeof(TX), H = V / 2;
    const Team tm(a.lanes, buf);
    const int rows = (int)a.rows, step = (int)gridDim.x * tm.count;
    const int nvec = (a.dim + V - 1) / V, room = tm.L * NV * V;
    const Span x_span(static_cast<const TX*>(a.x), a.rows, a.x_stride, a.dim);
    const Span dy_span(static_cast<const TY*>(a.dy), a.rows, a.dy_stride, a.dim);
    float2 dw[NV][H], db[NV][H];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < H; ++k) dw[i][k] = db[i][k] = both(0.f);
    int at[NV];  // of this lane's vectors, the last one again where there are no more
#pragma unroll
    for (int i = 0; i < NV; ++i) at[i] = min(tm.lane + i * tm.L, nvec - 1) * V;
    Values<TX, V, ALIGNED> x[NV];
    Values<TY, V, ALIGNED> dy[NV];
    int r = (int)blockIdx.x * tm.count + tm.index;
    const TX* x_at = static_cast<const TX*>(a.x) + r * a.x_stride;
    const TY* dy_at = static_cast<const TY*>(a.dy) + r * a.dy_stride;
    TX* o = static_cast<TX*>(a.out) + r * a.out_stride;
    const int64_t x_step = step * a.x_stride, dy_step = step * a.dy_stride, o_step = step * a.out_stride;
    uint8_t* rows_at = reinterpret_cast<uint8_t*>(shared + room);
    const RowRing<TX, V, NV, ALIGNED> x_ring(rows_at, tm, room);
    rows_at += x_ring.bytes(tm, room);
    const RowRing<TY, V, NV, ALIGNED> dy_ring(rows_at, tm, room);
    rows_at += dy_ring.bytes(tm, room);
    uint32_t x_by = (uint32_t)reinterpret_cast<uintptr_t>(x_at) & 15, dy_by = (uint32_t)reinterpret_cast<uintptr_t>(dy_at) & 15;  // of the row worked on
    float2 stats_ahead[2] = {both(0.f), both(0.f)};
    int ahead = r;
    // the next row not yet on its way, into slot `slot`
    auto fetch = [&](int slot, float2& its) {
        if (ahead < rows) {
            x_ring.fetch(tm, slot, x_at, at, a.dim, x_span);
            dy_ring.fetch(tm, slot, dy_at, at, a.dim, dy_span);
            its = reinterpret_cast<const float2*>(a.stats)[ahead];
        }
        copy_commit();
        x_at += x_step;
        dy_at += dy_step;
        ahead += step;
    };
    for (int i = 0; i < kNormAhead; ++i) fetch(i, stats_ahead[i]);
    const float inverse = -1.f / (float)a.dim;
    stage_weights<V>(shared, a.w, a.w_type, a.dim, room, 1.f);
    __syncthreads();
    int turn = 0;
    // the lanes of a warp take as many turns as its first team does
    for (int first = tm.L < 32 ? r - (int)(threadIdx.x & 31) / tm.L : r; first < rows; first += step, r += step, o += o_step, turn ^= 1) {
        const float2 stats = stats_ahead[0];
        copy_wait<kNormAhead - 1>();
        if (!ALIGNED) tm.sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x_ring.take(x[i], turn, i, at[i], x_by, a.dim);
            dy_ring.take(dy[i], turn, i, at[i], dy_by, a.dim);
            if (r >= rows) {  // a team past the last row, beside one that is not
                x[i].zero();
                dy[i].zero();
            }
        }
        const float2 minus = both(-stats.x), rs = both(stats.y);
        float2 c1 = both(0.f), c2 = both(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float2 w[H];
            weight_pairs<V>(shared, tm.lane + i * tm.L, room, w);
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const float2 d = dy[i].pair(k), xh = mul2(add2(x[i].pair(k), minus), rs), g = mul2(d, w[k]);
                if (tm.lane + i * tm.L < nvec) {  // (a copy's weight of 0 does not take an infinite value out)
                    c1 = add2(c1, g);
                    c2 = fma2(g, xh, c2);
                }
                dw[i][k] = fma2(d, xh, dw[i][k]);
                db[i][k] = add2(db[i][k], d);
            }
        }
        stats_ahead[0] = stats_ahead[1];
        if (!ALIGNED) tm.sync();  // all have read the row
        fetch(turn, stats_ahead[1]);
        x_by = (x_by + (uint32_t)(x_step * sizeof(TX))) & 15;
        dy_by = (dy_by + (uint32_t)(dy_step * sizeof(TY))) & 15;
        if (a.out) {
            float s1 = c1.x + c1.y, s2 = c2.x + c2.y;
            tm.sum(s1, s2, turn);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                x[i].forget();
                dy[i].forget();
            }
            if (r < rows) {
                const float2 m1 = both(s1 * inverse), m2 = both(s2 * inverse);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int j = tm.lane + i * tm.L;
                    float2 w[H];
                    weight_pairs<V>(shared, j, room, w);
                    Values<TX, V, ALIGNED> p;
#pragma unroll
                    for (int k = 0; k < H; ++k) {
                        const float2 xh = mul2(add2(x[i].pair(k), minus), rs);
                        p.set(k, mul2(fma2(xh, m2, fma2(dy[i].pair(k), w[k], m1)), rs));
                    }
                    if (j < nvec) p.store(o + j * V, a.dim - j * V);
                }
            }
        }
    }
    if (!a.part && !a.dweight && !a.dbias) return;
    // the lanes of a warp that hold the same columns
    for (int o = 16; o >= tm.L; o >>= 1)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < H; ++k) {
                dw[i][k].x += __shfl_xor_sync(0xffffffffu, dw[i][k].x, o);
                db[i][k].x += __shfl_xor_sync(0xffffffffu, db[i][k].x, o);
                dw[i][k].y += __shfl_xor_sync(0xffffffffu, dw[i][k].y, o);
                db[i][k].y += __shfl_xor_sync(0xffffffffu, db[i][k].y, o);
            }
    // ... then the block's teams (a warp's, where it holds several), one after another
    float* cols = reinterpret_cast<float*>(rows_at);
    const int teams = tm.L < 32 ? blockDim.x / 32 : tm.count, mine = tm.L < 32 ? threadIdx.x / 32 : tm.index;
    const bool holds = tm.L >= 32 || (threadIdx.x & 31) < tm.L;
    auto each = [&](auto f) {  // f(column, dw, db)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = tm.lane + i * tm.L;
            if (j >= nvec) continue;
#pragma unroll
            for (int k = 0; k < H; ++k) {
                if (ALIGNED || j * V + 2 * k < a.dim) f(j * V + 2 * k, dw[i][k].x, db[i][k].x);
                if (ALIGNED || j * V + 2 * k + 1 < a.dim) f(j * V + 2 * k + 1, dw[i][k].y, db[i][k].y);
            }
        }
    };
    for (int t = 0; t < teams - 1; ++t) {
        if (mine == t && holds)
            each([&](int c, float w, float b) {
                cols[c] = (t ? cols[c] : 0.f) + w;
                cols[a.dim + c] = (t ? cols[a.dim + c] : 0.f) + b;
            });
        __syncthreads();
    }
    if (mine != teams - 1 || !holds) return;
    each([&](int c, float w, float b) {
        if (teams > 1) {
            w += cols[c];
            b += cols[a.dim + c];
        }
        if (a.part) {
            a.part[(int64_t)blockIdx.x * 2 * a.dim + c] = w;
            a.part[(int64_t)blockIdx.x * 2 * a.dim + a.dim + c] = b;
        } else {
            if (a.dweight) store_as(a.dweight, a.w_type, c, w);
            if (a.dbias) store_as(a.dbias, a.w_type, c, b);
        }
    });
}

// Rows too long for registers: a block a row ...
template <class TX, class TY>
__global__ void __launch_bounds__(kNormLongLanes) k_norm_backward_long(NormArgs a) {
    pdl_enter();
    __shared__ __align__(16) float2 buf[64];
    const Team tm(kNormLongLanes, buf);
    __syncthreads();
    const TX* x = static_cast<const TX*>(a.x) + blockIdx.x * a.x_stride;
    const TY* dy = static_cast<const TY*>(a.dy) + blockIdx.x * a.dy_stride;
    const float mu = a.stats[2 * blockIdx.x], rs = a.stats[2 * blockIdx.x + 1];
    float c1 = 0.f, c2 = 0.f;
    for (int j = tm.lane; j < a.dim; j += kNormLongLanes) {
        const float g = to_float(dy[j]) * (a.w ? load_as_float(a.w, a.w_type, j) : 1.f);
        c1 += g;
        c2 += g * ((to_float(x[j]) - mu) * rs);
    }
    tm.sum(c1, c2, 0);
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
// which each takes every 32nd block, then over the warps (304 blocks' of 2,048 columns: 5 us).
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

// How the rows are dealt out, and the blocks whose sums of columns are kept apart:
// as many as run at a time, or, of rows too long for registers, shares of at most
// kLongShare rows, of which a thread adds one after another, that give every SM at
// least two blocks of k_norm_cols_long.  (Shares by the SMs alone / so, us: 5,000 x
// 16,384 bf16 809 / 492; 12,000 x 39,040 fp32 5,151 / 2,621; the latter, of one chain
// of 12,000 additions, with sums off by 1.2e-4.)
constexpr int64_t kLongShare = 256;
struct BackwardShape {
    NormShape sh;
    int threads, teams;
    int64_t blocks;
};
BackwardShape backward_shape(int64_t rows, int64_t dim, int V, int sms) {
    BackwardShape b;
    b.sh = norm_shape(rows, dim, V, kBackwardValues, kBackwardLanes, sms);
    if (b.sh.lanes) {
        b.threads = norm_team_threads(b.sh.lanes);
        b.teams = b.threads / b.sh.lanes;
        b.blocks = std::min<int64_t>((int64_t)sms * (kBackwardLanes / b.threads), (rows + b.teams - 1) / b.teams);
    } else {
        b.threads = kNormLongLanes;
        b.teams = 1;
        b.blocks = std::max((rows + kLongShare - 1) / kLongShare, std::min<int64_t>(rows, (2ll * sms * 128 + dim - 1) / dim));
        b.blocks = std::min<int64_t>(b.blocks, 65535);  // (a grid's y; rows of 280 GB reach about as many)
    }
    return b;
}

}  // namespace

// (The type of x, and with it the values of a vector, is not known here: of both, what takes more.)
extern "C" int64_t mlkv_layer_norm_backward_workspace(int64_t rows, int64_t dim) {
    if (rows < 0 || rows >= (int64_t)1 << 30 || dim < 1 || dim >= kNormMaxDim) return -1;
    if (rows == 0) return 0;
    const int sms = dense_sms();
    if (!sms) return -1;
    return std::max(backward_shape(rows, dim, 4, sms).blocks, backward_shape(rows, dim, 8, sms).blocks) * 2 * dim * (int64_t)sizeof(float);
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
    const int xs = dense_type_size(x_type), ys = dense_type_size(dy_type);
    const int V = 16 / xs;
    const bool aligned = norm_aligned(d_x, x_stride, xs, dim, V) && norm_aligned(d_dy, dy_stride, ys, dim, V) &&
                         norm_aligned(d_dx, dx_stride, xs, dim, V);
    const BackwardShape shape = backward_shape(rows, dim, V, sms);
    const NormShape& sh = shape.sh;
    const int threads = shape.threads, teams = shape.teams;
    const int64_t blocks = shape.blocks;
    const bool parts = want_cols && (blocks > 1 || !sh.lanes);
    if (!workspace_ok(d_workspace, workspace_bytes, parts ? blocks * 2 * dim * (int64_t)sizeof(float) : 0)) return MLKV_ERR_INVALID;
    a.part = parts ? static_cast<float*>(d_workspace) : nullptr;
    bool ok = true;
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
        by_shape<kBackwardValues * (int)sizeof(TX) / 16>(sh.NV, aligned, [&](auto nv, auto al) {
            auto kernel = k_norm_backward<TX, TY, decltype(nv)::value, decltype(al)::value>;
            const int room = sh.lanes * sh.NV * V;
            const size_t smem = ((size_t)room + (sh.lanes < threads ? 2 : 0) * (size_t)dim) * sizeof(float) +
                                kNormAhead * (aligned ? (size_t)sh.NV * threads * (16 + V * ys) : (size_t)teams * (norm_row(room, xs) + norm_row(room, ys)));
            ok = dense_smem(kernel, smem);
            if (ok) launch_kernel(true, kernel, dim3((unsigned)blocks), dim3(threads), smem, st, a);
        });
    });
    if (parts && ok)
        launch_kernel(true, k_norm_cols, dim3((unsigned)((2 * dim + 31) / 32)), dim3(1024), 0, st,
                      (const float*)d_workspace, (int)blocks, (int)dim, d_dweight, d_dbias, w_type);
    return ok && cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}
