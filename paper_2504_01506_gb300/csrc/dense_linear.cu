// The matrix product with bias, activation and residual, and its gradients
// (mlkv_linear, mlkv_linear_backward), by the kernel of dense_product.cuh.
//
//   forward   y = act(x W^T + b) + r
//   backward  p = dy act'(z),  dx = p W,  dW = p^T x,  db = column sums of p
//
// Sums are fp32 all the way; what is rounded to 16 bits is z (`pre`, which the
// slopes are taken at, while y goes by z itself), y, p and the gradients, once each.
#include "dense_product.cuh"

using namespace mlkv;

namespace {

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
    Epilogue e = p.e;
    if (p.half && i >= p.half) {
        i -= p.half;
        e.out = p.out2;
        e.out_stride = p.out2_stride;
    }
    const int64_t row = (int64_t)i * ((kOf << blocks_per_tile) >> wide) + (q >> wide);
    const int64_t col = ((int64_t)j << (wide + 2)) + (q & ((1 << wide) - 1)) * 4;
    if (row < p.I && col < p.J) put_four<T>(e, sum, row, col, p.J);
}

// Rows whose stride or place TMA does not take (multiples of 16 bytes), laid out anew: up to three matrices at a time.
// Bound by latency at the sizes met (4,099 x 777 and 1,001 x 777: 6 us, 16 MB), by HBM above.
struct Align {
    const uint16_t* in;
    uint16_t* out;
    int64_t stride, out_stride, rows, cols;
};
__global__ void __launch_bounds__(256) k_align(Align a, Align b, Align c) {
    pdl_enter();
    const Align m = blockIdx.y == 0 ? a : blockIdx.y == 1 ? b : c;
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

struct Caller : Products {
    void forward(const mlkv_linear_args& g) {
        Epilogue e = {};
        e.bias = g.d_bias; e.residual = g.d_residual; e.residual_stride = g.residual_stride;
        e.pre = g.d_pre; e.pre_stride = g.pre_stride; e.out = g.d_y; e.out_stride = g.y_stride; e.act = g.activation;
        Matrix x = {(const uint16_t*)g.d_x, g.x_stride, g.m, g.k}, w = {(const uint16_t*)g.d_weight, g.weight_stride, g.n, g.k};
        if (g.m && g.n && g.k) align(x, w);
        finish(product<Plain, false, false>(x, w, g.m, g.n, g.k, e));
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
            dx = product<Plain, false, true>(p, w, g.m, g.k, g.n, e);
        }
        const bool beside = !MLKV_PDL_TRIGGER_FIRST && rc == MLKV_OK && g.d_dx && g.m && g.n && g.k;  // (dx's blocks have waited first)
        if (part) launch_kernel(true, k_column_sums, dim3((unsigned)((g.n + 31) / 32)), dim3(1024), 0, st, part, shares, g.n, g.d_dbias, type, (int)beside);
        if (g.d_dweight) {
            e.out = g.d_dweight; e.out_stride = g.dweight_stride;
            dw = product<Plain, true, true>(p, x, g.n, g.k, g.m, e, beside);
        }
        finish(dx);
        finish(dw);
    }
};

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
    Caller c = {{nullptr, dense_sms(), false, g->type, {nullptr}}};
    if (!c.sms) return -1;
    if (backward) c.backward(*g);
    else c.forward(*g);
    return c.rc == MLKV_OK ? c.arena.used : -2;
}

int run_linear(const mlkv_linear_args* g, bool backward, void* stream) {
    const int64_t need = working_memory(g, backward);
    if (need < 0) return need == -2 ? MLKV_ERR_UNSUPPORTED : MLKV_ERR_CUDA;
    if (!workspace_ok(g->d_workspace, g->workspace_bytes, need)) return MLKV_ERR_INVALID;
    Caller c = {{(cudaStream_t)stream, dense_sms(), true, g->type, {static_cast<char*>(g->d_workspace)}}};
    if (backward) c.backward(*g);
    else c.forward(*g);
    if (c.rc != MLKV_OK) return c.rc;
    return cudaGetLastError() == cudaSuccess ? MLKV_OK : MLKV_ERR_CUDA;
}

}  // namespace

namespace mlkv {
void Products::align(Matrix& a, Matrix& b) {
    Matrix none = {};
    align(a, b, none);
}
void Products::align(Matrix& a, Matrix& b, Matrix& c) {
    Align to[3] = {};
    int n = 0;
    for (Matrix* m : {&a, &b, &c}) {
        if (m->rows == 1) m->stride = round_up(m->cols, 8);  // (the one row's end is its end)
        if (m->aligned() || !m->rows || !m->cols) continue;
        const int64_t stride = round_up(m->cols, 8);
        uint16_t* p = static_cast<uint16_t*>(arena.take(m->rows * stride * 2));
        to[n++] = {m->p, p, m->stride, stride, m->rows, m->cols};
        *m = {p, stride, m->rows, m->cols};
    }
    if (!run || !n) return;
    const int64_t vectors = std::max({to[0].rows * to[0].out_stride, to[1].rows * to[1].out_stride, to[2].rows * to[2].out_stride}) / 8;
    launch_kernel(true, k_align, dim3(blocks_for(vectors), n), dim3(256), 0, st, to[0], to[1], to[2]);
}
void Products::finish_shares(const Product& p, int64_t tiles, int high, int bn) {
    if (!run || !tiles) return;
    const int groups = p.shares >= 8 ? 4 : 1, blocks = high * bn / 1024 * groups, wide = bn == 64 ? 4 : bn == 128 ? 5 : 6;
    int per = 0;
    while (1 << per < blocks) ++per;
    const dim3 grid((unsigned)(tiles * blocks));
    const bool b = type == MLKV_TYPE_BFLOAT;
    const auto kernel = groups == 4 ? (b ? k_product_finish<__nv_bfloat16, 4> : k_product_finish<__half, 4>)
                                    : (b ? k_product_finish<__nv_bfloat16, 1> : k_product_finish<__half, 1>);
    launch_kernel(true, kernel, grid, dim3(256), 0, st, p, per, wide);
}
Rest product_of_rows(Products& c, const Matrix& a, const Matrix& b, int64_t rows, int64_t cols, int64_t k, const Epilogue& e, const Kept& kept) {
    return c.product<Plain, false, true>(a, b, rows, cols, k, e, false, {}, {}, kept);
}
Rest product_of_columns(Products& c, const Matrix& a, const Matrix& b, int64_t rows, int64_t cols, int64_t k, const Epilogue& e, bool beside) {
    return c.product<Plain, true, true>(a, b, rows, cols, k, e, beside);
}
}  // namespace mlkv

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
    constexpr int kDevices = 64, kFiles = 3;
    static std::atomic<uint32_t> told[kDevices];  // of the files' g_timeouts
    int dev = 0;
    uint32_t counts[kFiles] = {};
    const cudaStream_t st = (cudaStream_t)stream;
    // (first the wait, which a stream that is being captured refuses: a copy would be captured)
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices || cudaStreamSynchronize(st) != cudaSuccess ||
        cudaMemcpyFromSymbolAsync(&counts[0], g_timeouts, sizeof(counts[0]), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        timeouts_of_gated(&counts[1], st) != cudaSuccess || timeouts_of_xent(&counts[2], st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return MLKV_ERR_CUDA;
    const uint32_t now = counts[0] + counts[1] + counts[2];
    for (uint32_t before = told[dev].load(); (int32_t)(now - before) > 0;)
        if (told[dev].compare_exchange_weak(before, now)) return MLKV_ERR_TIMEOUT;
    return MLKV_OK;
}
