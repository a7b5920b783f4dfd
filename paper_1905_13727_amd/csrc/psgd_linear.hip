// The linear layer of a plan: y = residual + D(act(x W^T + b)) and its backward pass.  Here what surrounds the products:
// operands laid out for them where they are not yet, dz and the bias gradient, and which launches a call is.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "psgd_epilogue.h"

namespace psgd {

// bf16 dst [rows][dst_ld] = src [rows][cols], rounded if src is fp32; dst_ld a multiple of eight, columns from `cols` on are zero.
// One lane: eight columns.  Memory bounds it: 8192 x 2048 fp32 weights 17 us, 5.9 TB/s.
template <bool SBF>
__global__ __launch_bounds__(kBlock) void k_lay_out(const void* src, int64_t src_ld, bf16_t* dst, int64_t dst_ld, int64_t rows, int64_t cols) {
    const int64_t per_row = dst_ld / 8, at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (at >= rows * per_row) return;
    const int64_t row = at / per_row, j = 8 * (at - row * per_row);
    float x[8];
    ld_oct<SBF>(src, row * src_ld + j, cols - j < 8 ? (int)(cols - j) : 8, x);
    st_oct<true>(dst, row * dst_ld + j, 8, x);
}

// dz = D(dy) act'(pre) without the factor of the elements that stay, which goes into the products' epilogues: where the
// slope is 0 or 1 dz is then exact in any type.  With other slopes it is rounded to bf16 on bf16 plans, as the matrix instructions take bf16: one rounding of half
// a step in front of the products beside the one behind them (against 64 bits 4096 x 8192 x 2048 with gelu is off by 2.35e-3 in norm, by 1.66e-3 with the
// last rounding alone, the square root of two less).  In two bf16 terms dz would keep 16 bits and double both products.  And the sum
// of every column over a block of rows, from the unrounded values.
// One lane: eight columns (one call of the generator) and every eighth row of the block.
// 4096 x 8192 bf16, gelu and dropout 48 us, 4.2 TB/s: some sixty instructions an element, a third of them the generator's, are as long as
// the memory accesses are.
template <bool BF>
__global__ __launch_bounds__(kBlock) void k_dz(const void* dy, int64_t dy_ld, const void* pre, int64_t pre_ld, int act, DropArgs drop,
                                               void* dz, int64_t dz_ld, float* partial, int64_t T, int64_t n) {
    __shared__ float sums[8][264];
    const int lane_c = threadIdx.x & 31, lane_t = threadIdx.x >> 5;
    const int64_t blocks_c = (n + 255) / 256, bt = blockIdx.x / blocks_c, bc = blockIdx.x - bt * blocks_c;
    const int64_t c0 = bc * 256 + 8 * lane_c;
    const int64_t t0 = bt * kSumRows, t1 = t0 + kSumRows < T ? t0 + kSumRows : T;
    const int count = n - c0 < 8 ? (int)(n - c0) : 8;
    Draw d{};
    if (drop.below) d = make_draw(drop.rng, drop.offset);
    float s[8] = {};
    if (count > 0) {
        constexpr int kAhead = 4;   // rows asked for at a time, ahead of the stores that a later load would wait for
        constexpr int z = BF ? 2 : 4;
        for (int64_t t = t0 + lane_t; t < t1; t += 8 * kAhead) {
            RawOct a[kAhead], b[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (t + 8 * q < t1) {
                    a[q] = ld_raw(static_cast<const char*>(dy) + ((t + 8 * q) * dy_ld + c0) * z, count, BF);
                    if (act != PSGD_ACT_IDENTITY) b[q] = ld_raw(static_cast<const char*>(pre) + ((t + 8 * q) * pre_ld + c0) * z, count, BF);
                }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t row = t + 8 * q;
                if (row >= t1) break;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = widened(a[q], j, BF);   // zero behind the last column
                if (act != PSGD_ACT_IDENTITY) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = widened(b[q], j, BF);
                    slope_oct(x, v, act);
                }
                if (drop.below) {
                    const Words r = philox(d, (unsigned)(c0 >> 3), (unsigned)row);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = dropped(r, j, drop.below) ? 0.f : v[j];
                }
                st_oct<BF>(dz, row * dz_ld + c0, dz_ld - c0 < 8 ? (int)(dz_ld - c0) : 8, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += v[j];
            }
        }
    }
    if (!partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[lane_t][8 * lane_c + j] = s[j];
    __syncthreads();
    const int64_t col = bc * 256 + threadIdx.x;
    if (col >= n) return;
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += sums[i][threadIdx.x];
    partial[bt * n + col] = v;
}

namespace {

bool failed(const char* name, std::string* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return false;
    *what = std::string("launch ") + name + ": " + hipGetErrorString(e);
    return true;
}

// Where the parts of the workspace are
struct Parts {
    int64_t w, x, dz, db, partial;   // offsets; w = -1: the weights are read where they are
    int64_t k_ld, n_ld;              // row lengths of laid-out operands
};

Parts parts_of(const LinearCall& c, bool forward) {
    Parts p{};
    const int64_t z = c.bf16 ? 2 : 4;
    p.k_ld = c.bf16 ? up(c.k, 8) : c.k;
    p.n_ld = c.bf16 ? up(c.n, 8) : c.n;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += up(bytes, 256); return was; };
    const bool copies = c.bf16 && (!forward || large_enough(c, false));   // whether x is aligned is not known yet
    p.w = copies && (!c.param_bf16 || c.k % 8) ? take(c.n * p.k_ld * z) : -1;
    p.x = copies ? take(c.T * p.k_ld * z) : 0;
    if (!forward) {
        p.dz = take(c.T * p.n_ld * z);
        p.db = take(up(c.T, kSumRows) / kSumRows * c.n * 4);
    }
    p.partial = at;
    return p;
}

bool lay_out(const void* src, int64_t src_ld, bool src_bf, void* dst, int64_t dst_ld, int64_t rows, int64_t cols, hipStream_t s, std::string* what) {
    const int64_t blocks = (rows * (dst_ld / 8) + kBlock - 1) / kBlock;
    auto k = src_bf ? k_lay_out<true> : k_lay_out<false>;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(kBlock), 0, s, src, src_ld, static_cast<bf16_t*>(dst), dst_ld, rows, cols);
    return !failed("k_lay_out", what);
}

// The weights or the input as operand B or A of the product q.M x q.N x q.K
bool weights(const LinearCall& c, const Parts& p, ProductCall& q, bool other_ready, std::string* what) {
    const Comes w = weights_come(c, other_ready);
    q.b = c.w;
    q.b_ld = c.k;
    q.b_fp32 = c.bf16 && !c.param_bf16 && !w.lay;
    q.b_ready = w.ready || w.lay;
    if (!w.lay) return true;
    void* to = static_cast<char*>(c.workspace) + p.w;
    q.b = to;
    q.b_ld = p.k_ld;
    return lay_out(c.w, c.k, c.param_bf16, to, p.k_ld, c.n, c.k, q.stream, what);
}
bool input(const LinearCall& c, const Parts& p, const ProductCall& q, bool other_ready, const void** x, int64_t* ld, bool* ready, std::string* what) {
    const Comes in = input_comes(c, !q.a_along, other_ready);
    *x = c.x;
    *ld = c.x_ld;
    *ready = in.ready || in.lay;
    if (!in.lay) return true;
    void* to = static_cast<char*>(c.workspace) + p.x;
    *x = to;
    *ld = p.k_ld;
    return lay_out(c.x, c.x_ld, true, to, p.k_ld, c.T, c.k, q.stream, what);
}

}  // namespace

int64_t linear_workspace_bytes(const LinearCall& c) {
    if (c.T == 0) return 0;
    return parts_of(c, false).partial + std::max(product_partial_bytes(c.bf16, c.T, c.n, c.k),
                                          up(product_partial_bytes(c.bf16, c.T, c.k, c.n), 256) + product_partial_bytes(c.bf16, c.n, c.k, c.T));
}

int64_t linear_forward_workspace_bytes(const LinearCall& c) {
    if (c.T == 0) return 0;
    return few_tokens(c) ? 256 : std::max<int64_t>(256, parts_of(c, true).partial + product_partial_bytes(c.bf16, c.T, c.n, c.k));
}

psgd_status launch_linear_forward(const LinearCall& c, std::string* what) {
    EpilogueHost ep;
    ep.bias = c.bias;
    ep.bias_bf = c.param_bf16;
    ep.act = c.act;
    ep.pre = c.pre;
    ep.pre_ld = c.pre_ld;
    ep.residual = c.residual;
    ep.residual_ld = c.residual_ld;
    ep.drop = c.drop;
    if (few_tokens(c)) return launch_few_tokens(c, ep, what);
    const Parts p = parts_of(c, true);
    ProductCall q{};
    q.bf16 = c.bf16;
    q.a_along = q.b_along = true;
    q.c = c.y;
    q.c_ld = c.y_ld;
    q.M = c.T;
    q.N = c.n;
    q.K = c.k;
    q.ep = ep;
    q.partial = reinterpret_cast<float*>(static_cast<char*>(c.workspace) + p.partial);
    q.stream = static_cast<hipStream_t>(c.stream);
    const Comes w = weights_come(c, true), in = input_comes(c, false, true);   // each by itself
    if (!weights(c, p, q, in.ready || in.lay, what) || !input(c, p, q, w.ready || w.lay, &q.a, &q.a_ld, &q.a_ready, what)) return PSGD_EHIP;
    return launch_product(q, what);
}

psgd_status launch_linear_backward(const LinearCall& c, std::string* what) {
    const hipStream_t s = static_cast<hipStream_t>(c.stream);
    const Parts p = parts_of(c, false);
    const float scale = c.drop.below ? c.drop.factor : 1.f;
    if (c.T == 0 && c.accumulate) return PSGD_OK;
    const Comes come = dz_comes(c);
    const bool direct = !come.lay;   // dz is read in dy's place
    char* const ws = static_cast<char*>(c.workspace);
    const int64_t blocks = up(c.T, kSumRows) / kSumRows;
    if ((!direct || c.db) && (c.n + 255) / 256 * blocks > most_groups(kBlock)) return PSGD_EUNSUPPORTED;   // before anything is launched
    const void* dz = c.dy;
    int64_t dz_ld = c.dy_ld;
    const bool dz_ready = come.ready || come.lay;
    if (c.T > 0) {
        if (!direct) {   // rows padded with zeros to multiples of sixteen bytes
            dz = ws + p.dz;
            dz_ld = p.n_ld;
            auto k = c.bf16 ? k_dz<true> : k_dz<false>;
            hipLaunchKernelGGL(k, dim3((unsigned)((c.n + 255) / 256 * blocks)), dim3(kBlock), 0, s, c.dy, c.dy_ld, c.pre, c.pre_ld, c.act, drop_of(c.drop),
                               const_cast<void*>(dz), dz_ld, c.db ? reinterpret_cast<float*>(ws + p.db) : nullptr, c.T, c.n);
            if (failed("k_dz", what)) return PSGD_EHIP;
        }
    }
    const ColumnSums sums{dz == c.dy ? c.dy : nullptr, c.dy_ld, c.T, c.n, reinterpret_cast<float*>(ws + p.db), scale, c.db, (int)c.accumulate};
    ProductCall x{};
    x.bf16 = c.bf16;
    x.ep.scale = scale;
    x.partial = reinterpret_cast<float*>(ws + p.partial);
    x.stream = s;
    x.a = dz;
    x.a_ld = dz_ld;
    x.a_ready = dz_ready;
    x.N = c.k;
    ProductCall w = x;
    const bool want_x = c.dx && c.T > 0;
    if (want_x) {
        x.a_along = true;
        x.c = c.dx;
        x.c_ld = c.dx_ld;
        x.M = c.T;
        x.K = c.n;
        if (!weights(c, p, x, dz_ready, what)) return PSGD_EHIP;
        w.partial += up(product_partial_bytes(c.bf16, c.T, c.k, c.n), 256) / 4;
    }
    if (c.dw) {
        w.c = c.dw;
        w.c_ld = c.k;
        w.M = c.n;
        w.K = c.T;
        if (!input(c, p, w, dz_ready, &w.b, &w.b_ld, &w.b_ready, what)) return PSGD_EHIP;
        if (c.accumulate) {
            w.ep.residual = c.dw;
            w.ep.residual_ld = c.k;
        }
    }
    return launch_backward_products(c.bf16, want_x ? &x : nullptr, c.dw ? &w : nullptr, c.db ? &sums : nullptr, s, what);
}

}  // namespace psgd
