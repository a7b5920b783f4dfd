// The linear layer of few tokens: x W^T where the weights are read once and nothing else counts.
//
// A workgroup owns 16 RF rows of W (columns of y) and all tokens; its eight waves take every eighth stretch of 64 of the
// contraction each, straight from memory into the matrix instructions (no element of W is used twice, so none goes through LDS), in
// whatever type and at whatever alignment the parameters have.  Every load takes 64 consecutive bytes of each of sixteen rows, four
// lanes a row.  Which element of the contraction stands where in an instruction does not matter as long as x, read from the caches,
// has it in the same place: with fp32 weights and bf16 x a lane's eight are two runs of four.  The waves' sums meet in LDS and are
// added in the waves' order.  What the epilogue needs of memory (bias, residual, the generator's words) is asked for first, so that nothing is
// waited for behind the sums: one token, 8192 x 2048 bf16 9.0 us with weights from memory, 3.7 TB/s, 10.0 without that.
#include <hip/hip_runtime.h>

#include "psgd_epilogue.h"

namespace psgd {

constexpr int kFewWaves = 8, kFewDepth = 4;   // stretches a wave has in flight: 4 x 128 bytes of a row (bf16)

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// 64 elements of a row, sixteen to a lane, as the operands of the instructions: bf16 two of eight, fp32 four of four
template <bool BF>
struct Run {
    typedef typename std::conditional<BF, v8bf, v4f>::type Frag;
    static constexpr int kFrags = BF ? 2 : 4;
    Frag f[kFrags];
};

typedef unsigned v2u_any __attribute__((ext_vector_type(2), aligned(2)));

// SBF: type in memory.  FOURS: the lane's elements are 16 q + 4 g + (0 .. 3), q = 0 .. 3, else 32 h + 8 g + (0 .. 7), h = 0, 1.
// p: the first of the 64; g: the lane group.
template <bool BF, bool SBF, bool FOURS>
__device__ __forceinline__ void ld_run(const void* p, int64_t at, int g, Run<BF>& r) {
    if constexpr (SBF && !FOURS) {
        const bf16_t* q = static_cast<const bf16_t*>(p) + at + 8 * g;
#pragma unroll
        for (int h = 0; h < 2; ++h) r.f[h] = __builtin_bit_cast(v8bf, (v4u) * reinterpret_cast<const v4u_any*>(q + 32 * h));
    } else if constexpr (SBF) {
        const bf16_t* q = static_cast<const bf16_t*>(p) + at + 4 * g;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const v2u lo = *reinterpret_cast<const v2u_any*>(q + 32 * h), hi = *reinterpret_cast<const v2u_any*>(q + 32 * h + 16);
            r.f[h] = __builtin_bit_cast(v8bf, v4u{lo.x, lo.y, hi.x, hi.y});
        }
    } else {
        const float* q = static_cast<const float*>(p) + at + 4 * g;
        v4f t[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) t[h] = *reinterpret_cast<const v4f_any*>(q + 16 * h);
        if constexpr (BF) {   // rounded to nearest even
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4f a = t[2 * h], b = t[2 * h + 1];
                r.f[h] = __builtin_bit_cast(v8bf, v4u{pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w)});
            }
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h) r.f[h] = t[h];
        }
    }
}
// the same where the row ends `left` elements after the first of the 64: zeros behind
template <bool BF, bool SBF, bool FOURS>
__device__ __forceinline__ void ld_run_cut(const void* p, int64_t at, int g, int left, Run<BF>& r) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int first = FOURS ? 16 * q + 4 * g : 32 * (q / 2) + 8 * g + 4 * (q % 2);
        v4f t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = first + e < left ? ld_any(p, at + first + e, SBF) : 0.f;
        if constexpr (BF) {
            v4u u = __builtin_bit_cast(v4u, r.f[q / 2]);
            u[2 * (q & 1)] = pack_bf16x2(t.x, t.y);
            u[2 * (q & 1) + 1] = pack_bf16x2(t.z, t.w);
            r.f[q / 2] = __builtin_bit_cast(v8bf, u);
        } else {
            r.f[q] = t;
        }
    }
}

template <bool BF>
__device__ __forceinline__ v4f multiply_run(const Run<BF>& w, const Run<BF>& x, v4f acc) {
    if constexpr (BF) {
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.f[h], x.f[h], acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w.f[h][e], x.f[h][e], acc, 0, 0, 0);
    }
    return acc;
}

// BF: type of x and y; WBF: of the parameters; 16 RF rows of W a workgroup, up to 16 TF tokens
template <bool BF, bool WBF, int RF, int TF>
__global__ __launch_bounds__(kFewWaves* kWave, TF == 1 ? 4 : 2) void k_few_tokens(const void* __restrict__ w, const void* __restrict__ x, int64_t x_ld, void* y, int64_t y_ld,
                                                                    int T, int64_t n, int64_t k, Epilogue ep) {
    constexpr bool kFours = !WBF;
    constexpr int kRow = 16 * RF + 4;   // floats of a token's sums in LDS
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][16 * TF][kRow];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t r0 = (int64_t)blockIdx.x * (16 * RF);
    int64_t w_at[RF], x_at[TF];   // rows and tokens past the end read the last ones; what they give is not stored
#pragma unroll
    for (int f = 0; f < RF; ++f) w_at[f] = (r0 + 16 * f + i < n ? r0 + 16 * f + i : n - 1) * k;
#pragma unroll
    for (int f = 0; f < TF; ++f) x_at[f] = (16 * f + i < T ? 16 * f + i : T - 1) * x_ld;
    v4f acc[RF][TF];
#pragma unroll
    for (int a = 0; a < RF; ++a)
#pragma unroll
        for (int b = 0; b < TF; ++b) acc[a][b] = v4f{0.f, 0.f, 0.f, 0.f};
    // the eight columns of one token that this lane finishes
    static_assert(16 * TF * 2 * RF <= kFewWaves * kWave, "one a lane");
    const int t = threadIdx.x / (2 * RF), c = 8 * (threadIdx.x % (2 * RF));
    const int64_t j = r0 + c;
    const bool finishes = t < T && j < n;
    const int count = n - j < 8 ? (int)(n - j) : 8;
    const RawOct bias = finishes ? bias_ahead(ep, j, n) : RawOct(), residual = finishes ? residual_ahead<BF>(ep, t * ep.residual_ld + j, count) : RawOct();
    const DrawWords words = ep.drop.below ? words_ahead(ep.drop.rng, ep.drop.offset) : DrawWords{0, 0, 0, 0};
    const int whole = (int)(k / 64);
    int s = wave;
    for (; s + (kFewDepth - 1) * kFewWaves < whole; s += kFewDepth * kFewWaves) {
        Run<BF> wr[kFewDepth][RF], xr[kFewDepth][TF];
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            const int64_t l = (int64_t)(s + d * kFewWaves) * 64;
#pragma unroll
            for (int f = 0; f < RF; ++f) ld_run<BF, WBF, kFours>(w, w_at[f] + l, g, wr[d][f]);
#pragma unroll
            for (int f = 0; f < TF; ++f) ld_run<BF, BF, kFours>(x, x_at[f] + l, g, xr[d][f]);
        }
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d)
#pragma unroll
            for (int a = 0; a < RF; ++a)
#pragma unroll
                for (int b = 0; b < TF; ++b) acc[a][b] = multiply_run(wr[d][a], xr[d][b], acc[a][b]);
    }
    for (; s * 64 < k; s += kFewWaves) {
        Run<BF> wr[RF], xr[TF];
        const int64_t l = (int64_t)s * 64;
        if (s < whole) {
#pragma unroll
            for (int f = 0; f < RF; ++f) ld_run<BF, WBF, kFours>(w, w_at[f] + l, g, wr[f]);
#pragma unroll
            for (int f = 0; f < TF; ++f) ld_run<BF, BF, kFours>(x, x_at[f] + l, g, xr[f]);
        } else {
            const int left = (int)(k - l);
#pragma unroll
            for (int f = 0; f < RF; ++f) ld_run_cut<BF, WBF, kFours>(w, w_at[f] + l, g, left, wr[f]);
#pragma unroll
            for (int f = 0; f < TF; ++f) ld_run_cut<BF, BF, kFours>(x, x_at[f] + l, g, left, xr[f]);
        }
#pragma unroll
        for (int a = 0; a < RF; ++a)
#pragma unroll
            for (int b = 0; b < TF; ++b) acc[a][b] = multiply_run(wr[a], xr[b], acc[a][b]);
    }
    // lane i of group g holds rows 4 g .. 4 g + 3 of token i
#pragma unroll
    for (int a = 0; a < RF; ++a)
#pragma unroll
        for (int b = 0; b < TF; ++b) *reinterpret_cast<v4f*>(&sums[wave][16 * b + i][16 * a + 4 * g]) = acc[a][b];
    __syncthreads();
    const Draw d = make_draw(words);
    if (finishes) {
        float v[8] = {}, b[8];
#pragma unroll
        for (int q = 0; q < kFewWaves; ++q) {
            const v4f lo = *reinterpret_cast<const v4f*>(&sums[q][t][c]), hi = *reinterpret_cast<const v4f*>(&sums[q][t][c + 4]);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[4 + e] += hi[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = widened(bias, e, ep.bias_bf);
        finish_oct<BF>(ep, d, y, t * y_ld + j, t * ep.pre_ld + j, t, j, count, v, b, residual);
    }
}

namespace {

template <bool BF, bool WBF>
hipError_t start(const LinearCall& c, const Epilogue& ep) {
    // 32 rows a workgroup where that still is one for every compute unit: x is read from the caches half as often.  8192 x 2048 bf16, 16
    // and 32 tokens: 7.9 and 9.8 us, with 16 rows 9.7 and 13.2; 4096 x 1024, 16 tokens 5.0 and 4.2; fp32 with few tokens loads enough with
    // 16 (8192 x 2048, one token 12.9, with 32 rows 16.1; 32 tokens 23.8 and 18.4)
    const bool two = c.n >= 32 * 256 && (WBF || c.T > 16);
    const int64_t rows = two ? 32 : 16;
    auto k = two ? (c.T <= 16 ? k_few_tokens<BF, WBF, 2, 1> : k_few_tokens<BF, WBF, 2, 2>) : (c.T <= 16 ? k_few_tokens<BF, WBF, 1, 1> : k_few_tokens<BF, WBF, 1, 2>);
    hipLaunchKernelGGL(k, dim3((unsigned)((c.n + rows - 1) / rows)), dim3(kFewWaves * kWave), 0, static_cast<hipStream_t>(c.stream), c.w, c.x, c.x_ld, c.y,
                       c.y_ld, (int)c.T, c.n, c.k, ep);
    return hipGetLastError();
}

}  // namespace

psgd_status launch_few_tokens(const LinearCall& c, const EpilogueHost& host, std::string* what) {
    const Epilogue ep = epilogue_of(host);
    const hipError_t e = !c.bf16 ? start<false, false>(c, ep) : c.param_bf16 ? start<true, true>(c, ep) : start<true, false>(c, ep);
    if (e != hipSuccess) { *what = std::string("launch k_few_tokens: ") + hipGetErrorString(e); return PSGD_EHIP; }
    return PSGD_OK;
}

}  // namespace psgd
