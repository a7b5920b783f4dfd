// The linear layer of a plan: y = residual + D(act(x W^T + b)) and its backward pass.  Here what surrounds the products:
// operands laid out for them where they are not yet, dz and the bias gradient, and which launches a call is.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "psgd_epilogue.h"

namespace psgd {

// bf16 dst [rows][dst_ld] = src [rows][cols], rounded if src is fp32; dst_ld a multiple of eight, columns from `cols` on are zero.
// One lane: eight columns.
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
// slope is 0 or 1 dz is then exact in any type.  And the sum of every column over a block of rows.
// One lane: eight columns (one call of the generator) and every eighth row of the block.
constexpr int kDzRows = 64;

template <bool BF>
__global__ __launch_bounds__(kBlock) void k_dz(const void* dy, int64_t dy_ld, const void* pre, int64_t pre_ld, int act, DropArgs drop,
                                               void* dz, int64_t dz_ld, float* partial, int64_t T, int64_t n) {
    __shared__ float sums[8][264];
    const int lane_c = threadIdx.x & 31, lane_t = threadIdx.x >> 5;
    const int64_t blocks_c = (n + 255) / 256, bt = blockIdx.x / blocks_c, bc = blockIdx.x - bt * blocks_c;
    const int64_t c0 = bc * 256 + 8 * lane_c;
    const int64_t t0 = bt * kDzRows, t1 = t0 + kDzRows < T ? t0 + kDzRows : T;
    const int count = n - c0 < 8 ? (int)(n - c0) : 8;
    Draw d{};
    if (drop.below) d = make_draw(drop.rng, drop.offset);
    float s[8] = {};
    if (count > 0) {
        for (int64_t t = t0 + lane_t; t < t1; t += 8) {
            float v[8];
            ld_oct<BF>(dy, t * dy_ld + c0, count, v);
            if (act != PSGD_ACT_IDENTITY) {
                float z[8];
                ld_oct<BF>(pre, t * pre_ld + c0, count, z);
                slope_oct(z, v, act);
            }
            if (drop.below) {
                const Words r = philox(d, (unsigned)(c0 >> 3), (unsigned)t);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = dropped(r, j, drop.below) ? 0.f : v[j];
            }
            if (dz) {   // up to the end of its rows: zero behind the last column
                if (count < 8)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = j < count ? v[j] : 0.f;
                const int to = dz_ld - c0 < 8 ? (int)(dz_ld - c0) : 8;
                st_oct<BF>(dz, t * dz_ld + c0, to, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += v[j];
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

// db from the blocks' sums: a workgroup 64 columns, its four waves every fourth block, joined in order
template <bool BF>
__global__ __launch_bounds__(kBlock) void k_column_sum(const float* partial, int64_t count, int64_t n, float scale, void* db, int accumulate) {
    __shared__ float sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (col < n)
        for (int64_t i = wave; i < count; i += 4) v += partial[i * n + col];
    sums[wave][lane] = v;
    __syncthreads();
    if (wave || col >= n) return;
    v = ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane])) * scale;
    if (accumulate) v += ld_any(db, col, BF);
    st_any(db, col, v, BF);
}

namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

bool failed(const char* name, std::string* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return false;
    *what = std::string("launch ") + name + ": " + hipGetErrorString(e);
    return true;
}

bool vec_aligned(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }   // bf16

// Where the parts of the workspace are
struct Parts {
    int64_t w, x, dz, db, partial;   // offsets; w = -1: the weights are read where they are
    int64_t k_ld, n_ld;              // row lengths of laid-out operands
};

Parts parts_of(const LinearCall& c) {
    Parts p{};
    const int64_t z = c.bf16 ? 2 : 4;
    p.k_ld = c.bf16 ? up(c.k, 8) : c.k;
    p.n_ld = c.bf16 ? up(c.n, 8) : c.n;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += up(bytes, 256); return was; };
    p.w = c.bf16 && (!c.param_bf16 || c.k % 8) ? take(c.n * p.k_ld * z) : -1;
    p.x = c.bf16 ? take(c.T * p.k_ld * z) : 0;
    p.dz = take(c.T * p.n_ld * z);
    p.db = take(up(c.T, kDzRows) / kDzRows * c.n * 4);
    p.partial = at;
    return p;
}

bool lay_out(const void* src, int64_t src_ld, bool src_bf, void* dst, int64_t dst_ld, int64_t rows, int64_t cols, hipStream_t s, std::string* what) {
    const int64_t blocks = (rows * (dst_ld / 8) + kBlock - 1) / kBlock;
    auto k = src_bf ? k_lay_out<true> : k_lay_out<false>;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(kBlock), 0, s, src, src_ld, static_cast<bf16_t*>(dst), dst_ld, rows, cols);
    return !failed("k_lay_out", what);
}

// The weights or the input as an operand of a product: in place if it can read them there, else laid out
bool weights(const LinearCall& c, const Parts& p, const void** w, int64_t* ld, std::string* what) {
    *w = c.w;
    *ld = c.k;
    if (p.w < 0) return true;
    *w = static_cast<char*>(c.workspace) + p.w;
    *ld = p.k_ld;
    return lay_out(c.w, c.k, c.param_bf16, const_cast<void*>(*w), *ld, c.n, c.k, static_cast<hipStream_t>(c.stream), what);
}
bool input(const LinearCall& c, const Parts& p, const void** x, int64_t* ld, std::string* what) {
    *x = c.x;
    *ld = c.x_ld;
    if (!c.bf16 || (vec_aligned(c.x, c.x_ld) && c.k % 8 == 0)) return true;
    *x = static_cast<char*>(c.workspace) + p.x;
    *ld = p.k_ld;
    return lay_out(c.x, c.x_ld, true, const_cast<void*>(*x), *ld, c.T, c.k, static_cast<hipStream_t>(c.stream), what);
}

}  // namespace

int64_t linear_workspace_bytes(const LinearCall& c) {
    if (c.T == 0) return 0;
    return parts_of(c).partial + std::max({product_partial_bytes(c.bf16, c.T, c.n, c.k), product_partial_bytes(c.bf16, c.T, c.k, c.n),
                                           product_partial_bytes(c.bf16, c.n, c.k, c.T)});
}

psgd_status launch_linear_forward(const LinearCall& c, std::string* what) {
    const Parts p = parts_of(c);
    ProductCall q{};
    q.bf16 = c.bf16;
    q.a_along = q.b_along = true;
    if (!weights(c, p, &q.b, &q.b_ld, what) || !input(c, p, &q.a, &q.a_ld, what)) return PSGD_EHIP;
    q.c = c.y;
    q.c_ld = c.y_ld;
    q.M = c.T;
    q.N = c.n;
    q.K = c.k;
    q.ep.bias = c.bias;
    q.ep.bias_bf = c.param_bf16;
    q.ep.act = c.act;
    q.ep.pre = c.pre;
    q.ep.pre_ld = c.pre_ld;
    q.ep.residual = c.residual;
    q.ep.residual_ld = c.residual_ld;
    q.ep.drop = c.drop;
    q.partial = reinterpret_cast<float*>(static_cast<char*>(c.workspace) + p.partial);
    q.stream = static_cast<hipStream_t>(c.stream);
    return launch_product(q, what);
}

psgd_status launch_linear_backward(const LinearCall& c, std::string* what) {
    const hipStream_t s = static_cast<hipStream_t>(c.stream);
    const Parts p = parts_of(c);
    const float scale = c.drop.below ? c.drop.factor : 1.f;
    if (c.T == 0 && c.accumulate) return PSGD_OK;
    char* const ws = static_cast<char*>(c.workspace);
    const int64_t blocks = up(c.T, kDzRows) / kDzRows;
    const void* dz = c.dy;
    int64_t dz_ld = c.dy_ld;
    if (c.T > 0) {
        const bool direct = c.act == PSGD_ACT_IDENTITY && !c.drop.below && (!c.bf16 || (vec_aligned(c.dy, c.dy_ld) && c.n % 8 == 0));
        if (!direct) {
            dz = ws + p.dz;
            dz_ld = p.n_ld;
        }
        if (!direct || c.db) {
            auto k = c.bf16 ? k_dz<true> : k_dz<false>;
            if ((c.n + 255) / 256 * blocks > 0x7fffffffLL) return PSGD_EUNSUPPORTED;
            hipLaunchKernelGGL(k, dim3((unsigned)((c.n + 255) / 256 * blocks)), dim3(kBlock), 0, s, c.dy, c.dy_ld, c.pre, c.pre_ld, c.act, drop_of(c.drop),
                               direct ? nullptr : const_cast<void*>(dz), dz_ld, c.db ? reinterpret_cast<float*>(ws + p.db) : nullptr, c.T, c.n);
            if (failed("k_dz", what)) return PSGD_EHIP;
        }
    }
    if (c.db) {
        auto k = c.bf16 ? k_column_sum<true> : k_column_sum<false>;
        hipLaunchKernelGGL(k, dim3((unsigned)((c.n + 63) / 64)), dim3(kBlock), 0, s, reinterpret_cast<const float*>(ws + p.db), blocks, c.n, scale,
                           c.db, (int)c.accumulate);
        if (failed("k_column_sum", what)) return PSGD_EHIP;
    }
    ProductCall q{};
    q.bf16 = c.bf16;
    q.ep.scale = scale;
    q.partial = reinterpret_cast<float*>(ws + p.partial);
    q.stream = s;
    q.a = dz;
    q.a_ld = dz_ld;
    q.N = c.k;
    if (c.dx && c.T > 0) {
        q.a_along = true;
        if (!weights(c, p, &q.b, &q.b_ld, what)) return PSGD_EHIP;
        q.c = c.dx;
        q.c_ld = c.dx_ld;
        q.M = c.T;
        q.K = c.n;
        const psgd_status st = launch_product(q, what);
        if (st != PSGD_OK) return st;
    }
    if (c.dw) {
        q.a_along = false;
        q.b = nullptr;
        q.b_ld = 0;
        if (c.T > 0 && !input(c, p, &q.b, &q.b_ld, what)) return PSGD_EHIP;
        q.c = c.dw;
        q.c_ld = c.k;
        q.M = c.n;
        q.K = c.T;
        if (c.accumulate) {
            q.ep.residual = c.dw;
            q.ep.residual_ld = c.k;
        }
        return launch_product(q, what);
    }
    return PSGD_OK;
}

}  // namespace psgd
