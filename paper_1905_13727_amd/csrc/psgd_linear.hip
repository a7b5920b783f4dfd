// The linear layer of a plan: y = residual + D(act(x W^T + b)) and its backward pass.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "psgd_device.h"
#include "psgd_operators.h"
#include "psgd_random.h"

namespace psgd {

__device__ __forceinline__ float ld_any(const void* p, int64_t at, bool bf) {
    return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[at]) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void st_any(void* p, int64_t at, float v, bool bf) {
    if (bf) static_cast<bf16_t*>(p)[at] = f32_to_bf16(v);
    else static_cast<float*>(p)[at] = v;
}

// ---- activations, in fp32 -------------------------------------------------------------------------------------------

// 1 / (1 + exp(-v)) and 1 minus that, both without cancellation or overflow
__device__ __forceinline__ void logistic(float v, float& s, float& rest) {
    const float e = __expf(-fabsf(v)), big = 1.f / (1.f + e), small = e * big;
    s = v >= 0.f ? big : small;
    rest = v >= 0.f ? small : big;
}
constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f;   // 2 sqrt(2 / pi)

__device__ __forceinline__ float act_of(float z, int act) {
    float s, rest;
    switch (act) {
        case PSGD_ACT_RELU: return z < 0.f ? 0.f : z;
        case PSGD_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case PSGD_ACT_GELU_TANH: logistic(kGeluA * (z + kGeluB * z * z * z), s, rest); return z * s;   // (1 + tanh u) / 2
        case PSGD_ACT_SILU: logistic(z, s, rest); return z * s;
        default: return z;
    }
}
__device__ __forceinline__ float act_slope(float z, int act) {
    float s, rest;
    switch (act) {
        case PSGD_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case PSGD_ACT_GELU: return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
        case PSGD_ACT_GELU_TANH:
            logistic(kGeluA * (z + kGeluB * z * z * z), s, rest);
            return s + z * s * rest * kGeluA * (1.f + 3.f * kGeluB * z * z);
        case PSGD_ACT_SILU: logistic(z, s, rest); return s * (1.f + z * rest);
        default: return 1.f;
    }
}

// ---- product --------------------------------------------------------------------------------------------------------

struct Epilogue {
    const void* bias;
    bool bias_bf;
    int act;
    void* pre;
    int64_t pre_ld;
    const void* residual;
    int64_t residual_ld;
    DropArgs drop;
    bool accumulate;
    float scale;
};

// C[i][j] = sum_l A(i, l) B(j, l), element (i, l) of A at i * a_i + l * a_l, and the epilogue
__global__ __launch_bounds__(kBlock) void k_product(const void* A, int64_t a_i, int64_t a_l, bool a_bf, const void* B, int64_t b_j,
                                                    int64_t b_l, bool b_bf, bool round_b, void* C, int64_t c_ld, bool c_bf, int64_t M,
                                                    int64_t N, int64_t K, Epilogue ep) {
    __shared__ float As[16][65], Bs[16][65];
    const int64_t i0 = (int64_t)blockIdx.x * 64, j0 = (int64_t)blockIdx.y * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int64_t l0 = 0; l0 < K; l0 += 16) {
        for (int e = threadIdx.x; e < 1024; e += kBlock) {
            const int r = e >> 4, l = e & 15;
            const bool in = l0 + l < K;
            As[l][r] = in && i0 + r < M ? ld_any(A, (i0 + r) * a_i + (l0 + l) * a_l, a_bf) : 0.f;
            float b = in && j0 + r < N ? ld_any(B, (j0 + r) * b_j + (l0 + l) * b_l, b_bf) : 0.f;
            Bs[l][r] = round_b ? bf16_to_f32(f32_to_bf16(b)) : b;
        }
        __syncthreads();
        for (int l = 0; l < 16; ++l)
            for (int a = 0; a < 4; ++a)
                for (int b = 0; b < 4; ++b) acc[a][b] += As[l][ty + 16 * a] * Bs[l][tx * 4 + b];
        __syncthreads();
    }
    Draw d{};
    if (ep.drop.below) d = make_draw(ep.drop.rng, ep.drop.offset);
    for (int a = 0; a < 4; ++a) {
        const int64_t i = i0 + ty + 16 * a;
        if (i >= M) continue;
        for (int b = 0; b < 4; ++b) {
            const int64_t j = j0 + tx * 4 + b;
            if (j >= N) continue;
            float z = acc[a][b] * ep.scale;
            if (ep.bias) z += ld_any(ep.bias, j, ep.bias_bf);
            if (ep.pre) st_any(ep.pre, i * ep.pre_ld + j, z, c_bf);
            float v = act_of(z, ep.act);
            if (ep.drop.below) v = dropped(philox(d, (unsigned)(j >> 3), (unsigned)i), (int)(j & 7), ep.drop.below) ? 0.f : v * ep.drop.factor;
            if (ep.residual) v += ld_any(ep.residual, i * ep.residual_ld + j, c_bf);
            if (ep.accumulate) v += ld_any(C, i * c_ld + j, c_bf);
            st_any(C, i * c_ld + j, v, c_bf);
        }
    }
}

// dz = D(dy) act'(pre) without the factor of the elements that stay, which goes into the products' epilogues: where the
// slope is 0 or 1 dz is then exact in any type.  And the sum of every column over a block of rows.
// One lane: eight columns (one call of the generator) and every eighth row of the block.
constexpr int kDzRows = 128;

__global__ __launch_bounds__(kBlock) void k_dz(const void* dy, int64_t dy_ld, const void* pre, int64_t pre_ld, int act, bool bf,
                                               DropArgs drop, void* dz, int64_t dz_ld, float* partial, int64_t T, int64_t n) {
    __shared__ float sums[8][257];
    const int64_t c0 = (int64_t)blockIdx.x * 256 + 8 * (threadIdx.x & 31);
    const int64_t t0 = (int64_t)blockIdx.y * kDzRows, t1 = t0 + kDzRows < T ? t0 + kDzRows : T;
    Draw d{};
    if (drop.below) d = make_draw(drop.rng, drop.offset);
    float s[8] = {};
    for (int64_t t = t0 + (threadIdx.x >> 5); t < t1; t += 8) {
        Words r{};
        if (drop.below) r = philox(d, (unsigned)(c0 >> 3), (unsigned)t);
        for (int j = 0; j < 8 && c0 + j < n; ++j) {
            float v = 0.f;
            if (!dropped(r, j, drop.below)) {
                v = ld_any(dy, t * dy_ld + c0 + j, bf);
                if (act != PSGD_ACT_IDENTITY) v *= act_slope(ld_any(pre, t * pre_ld + c0 + j, bf), act);
            }
            if (dz) st_any(dz, t * dz_ld + c0 + j, v, bf);
            s[j] += v;
        }
    }
    if (!partial) return;
    for (int j = 0; j < 8; ++j) sums[threadIdx.x >> 5][8 * (threadIdx.x & 31) + j] = s[j];
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= n) return;
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += sums[i][threadIdx.x];
    partial[(int64_t)blockIdx.y * n + col] = v;
}

__global__ __launch_bounds__(kBlock) void k_column_sum(const float* partial, int64_t count, int64_t n, float scale, void* db, bool bf,
                                                       bool accumulate) {
    const int64_t col = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (col >= n) return;
    float v = 0.f;
    for (int64_t i = 0; i < count; ++i) v += partial[i * n + col];
    v *= scale;
    if (accumulate) v += ld_any(db, col, bf);
    st_any(db, col, v, bf);
}

namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

bool failed(const char* name, std::string* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return false;
    *what = std::string("launch ") + name + ": " + hipGetErrorString(e);
    return true;
}

DropArgs drop_of(const DropHost& h) {
    DropArgs d;
    d.rng = h.rng;
    d.offset = h.offset;
    d.below = h.below;
    d.factor = h.factor;
    return d;
}

}  // namespace

int64_t linear_workspace_bytes(const LinearCall& c) {
    const int64_t z = c.bf16 ? 2 : 4;
    return up(c.T * c.n * z, 256) + up((c.T + kDzRows - 1) / kDzRows * c.n * 4, 256);
}

psgd_status launch_linear_forward(const LinearCall& c, std::string* what) {
    Epilogue ep{};
    ep.bias = c.bias;
    ep.bias_bf = c.param_bf16;
    ep.act = c.act;
    ep.pre = c.pre;
    ep.pre_ld = c.pre_ld;
    ep.residual = c.residual;
    ep.residual_ld = c.residual_ld;
    ep.drop = drop_of(c.drop);
    ep.scale = 1.f;
    const dim3 grid((unsigned)((c.T + 63) / 64), (unsigned)((c.n + 63) / 64));
    hipLaunchKernelGGL(k_product, grid, dim3(kBlock), 0, static_cast<hipStream_t>(c.stream), c.x, c.x_ld, (int64_t)1, c.bf16, c.w, c.k,
                       (int64_t)1, c.param_bf16, c.bf16, c.y, c.y_ld, c.bf16, c.T, c.n, c.k, ep);
    return failed("k_product", what) ? PSGD_EHIP : PSGD_OK;
}

psgd_status launch_linear_backward(const LinearCall& c, std::string* what) {
    const hipStream_t s = static_cast<hipStream_t>(c.stream);
    const int64_t z = c.bf16 ? 2 : 4;
    Epilogue ep{};
    ep.scale = c.drop.below ? c.drop.factor : 1.f;
    if (c.T > 0) {
        char* ws = static_cast<char*>(c.workspace);
        void* dz = ws;
        float* partial = reinterpret_cast<float*>(ws + up(c.T * c.n * z, 256));
        const int64_t blocks = (c.T + kDzRows - 1) / kDzRows;
        hipLaunchKernelGGL(k_dz, dim3((unsigned)((c.n + 255) / 256), (unsigned)blocks), dim3(kBlock), 0, s, c.dy, c.dy_ld, c.pre, c.pre_ld, c.act,
                           c.bf16, drop_of(c.drop), dz, c.n, partial, c.T, c.n);
        if (failed("k_dz", what)) return PSGD_EHIP;
        if (c.dx) {
            hipLaunchKernelGGL(k_product, dim3((unsigned)((c.T + 63) / 64), (unsigned)((c.k + 63) / 64)), dim3(kBlock), 0, s, dz, c.n, (int64_t)1,
                               c.bf16, c.w, (int64_t)1, c.k, c.param_bf16, c.bf16, c.dx, c.dx_ld, c.bf16, c.T, c.k, c.n, ep);
            if (failed("k_product", what)) return PSGD_EHIP;
        }
        if (c.db) {
            hipLaunchKernelGGL(k_column_sum, dim3((unsigned)((c.n + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, partial, blocks, c.n, ep.scale, c.db,
                               c.bf16, c.accumulate);
            if (failed("k_column_sum", what)) return PSGD_EHIP;
        }
        ep.accumulate = c.accumulate;
        if (c.dw) {
            hipLaunchKernelGGL(k_product, dim3((unsigned)((c.n + 63) / 64), (unsigned)((c.k + 63) / 64)), dim3(kBlock), 0, s, dz, (int64_t)1, c.n,
                               c.bf16, c.x, (int64_t)1, c.x_ld, c.bf16, false, c.dw, c.k, c.bf16, c.n, c.k, c.T, ep);
            if (failed("k_product", what)) return PSGD_EHIP;
        }
        return PSGD_OK;
    }
    if (c.accumulate) return PSGD_OK;
    // no tokens: gradients of zero
    if (c.dw) {
        hipLaunchKernelGGL(k_product, dim3((unsigned)((c.n + 63) / 64), (unsigned)((c.k + 63) / 64)), dim3(kBlock), 0, s, nullptr, (int64_t)1, c.n,
                           c.bf16, nullptr, (int64_t)1, c.k, c.bf16, false, c.dw, c.k, c.bf16, c.n, c.k, (int64_t)0, ep);
        if (failed("k_product", what)) return PSGD_EHIP;
    }
    if (c.db) {
        hipLaunchKernelGGL(k_column_sum, dim3((unsigned)((c.n + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, nullptr, (int64_t)0, c.n, 1.f, c.db,
                           c.bf16, false);
        if (failed("k_column_sum", what)) return PSGD_EHIP;
    }
    return PSGD_OK;
}

}  // namespace psgd
