// Dropout and the random mask: the two elementwise operators on the counter-based generator.
#include <hip/hip_runtime.h>

#include <string>

#include "psgd_device.h"
#include "psgd_operators.h"
#include "psgd_random.h"

namespace psgd {

template <bool BF>
__device__ __forceinline__ float ld_elem(const void* p, int64_t at) {
    if constexpr (BF) return bf16_to_f32(static_cast<const bf16_t*>(p)[at]);
    else return static_cast<const float*>(p)[at];
}
template <bool BF>
__device__ __forceinline__ void st_elem(void* p, int64_t at, float v) {
    if constexpr (BF) static_cast<bf16_t*>(p)[at] = f32_to_bf16(v);
    else static_cast<float*>(p)[at] = v;
}

// y = residual + D(x).  One lane: eight consecutive columns of one row (one call of the generator).
template <bool BF>
__global__ __launch_bounds__(kBlock) void k_dropout(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld, void* y,
                                                    int64_t y_ld, int64_t rows, int64_t cols, DropArgs drop) {
    const int64_t groups = (cols + 7) / 8;
    const int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    Draw d{};
    if (drop.below) d = make_draw(drop.rng, drop.offset);
    if (at >= rows * groups) return;
    const int64_t row = at / groups, g = at - row * groups;
    Words r{};
    if (drop.below) r = philox(d, (unsigned)g, (unsigned)row);
    for (int j = 0; j < 8; ++j) {
        const int64_t col = 8 * g + j;
        if (col >= cols) break;
        float v = dropped(r, j, drop.below) ? 0.f : ld_elem<BF>(x, row * x_ld + col) * drop.factor;
        if (residual) v += ld_elem<BF>(residual, row * residual_ld + col);
        st_elem<BF>(y, row * y_ld + col, v);
    }
}

psgd_status launch_dropout(const DropoutCall& c, std::string* what) {
    const int64_t lanes = c.rows * ((c.cols + 7) / 8);
    const int64_t blocks = (lanes + kBlock - 1) / kBlock;
    if (blocks > 0x7fffffffLL) return PSGD_EUNSUPPORTED;
    DropArgs d;
    d.rng = c.drop.rng;
    d.offset = c.drop.offset;
    d.below = c.drop.below;
    d.factor = c.drop.factor;
    auto k = c.bf16 ? k_dropout<true> : k_dropout<false>;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(kBlock), 0, static_cast<hipStream_t>(c.stream), c.x, c.x_ld, c.residual,
                       c.residual_ld, c.y, c.y_ld, c.rows, c.cols, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { *what = std::string("launch k_dropout: ") + hipGetErrorString(e); return PSGD_EHIP; }
    return PSGD_OK;
}

// ---- random mask ---------------------------------------------------------------------------------------------------

// blockIdx.x: a slice of kFlatTileElems elements (as k_ef_add_zero's); one lane: four consecutive entries of one matrix and
// all workers.  Entry `pos` of tensor t takes word pos % 4 of the counter (pos / 4, t) and is kept where it is below
// `threshold`, or, with threshold 0 given, below the share of the entries that the plan's budget is.
template <bool GBF, bool OBF>
__global__ __launch_bounds__(kBlock) void k_random_mask(const MatDesc* __restrict__ mats, const int64_t* __restrict__ first, int n_mats,
                                                        const void* __restrict__ grad, float* __restrict__ err, void* __restrict__ out,
                                                        int workers, int64_t gstride, int64_t estride, int64_t n_mat_elems,
                                                        int64_t n_vec_elems, int budget, uint64_t threshold, const uint64_t* rng,
                                                        uint64_t offset) {
    const int64_t slice = blockIdx.x;
    const float inv_w = 1.0f / (float)workers;
    if (slice >= first[n_mats]) {
        // vector-shaped tensors: aggregated uncompressed (mean over the workers), no error memory
        const int64_t e0 = (slice - first[n_mats]) * kFlatTileElems;
        const int64_t e1 = e0 + kFlatTileElems < n_vec_elems ? e0 + kFlatTileElems : n_vec_elems;
        for (int64_t idx = e0 + threadIdx.x; idx < e1; idx += kBlock) {
            float s = 0.f;
            for (int w = 0; w < workers; ++w) s += ld_elem<GBF>(grad, (int64_t)w * gstride + n_mat_elems + idx);
            st_elem<OBF>(out, n_mat_elems + idx, s * inv_w);
        }
        return;
    }
    int lo = 0, hi = n_mats - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= slice) lo = mid;
        else hi = mid - 1;
    }
    const MatDesc d = mats[lo];
    const int64_t nm = (int64_t)d.n * d.m;
    const int64_t pos = (slice - first[lo]) * kFlatTileElems + 4 * threadIdx.x;
    const uint64_t below = budget ? ((uint64_t)d.kept << 32) / (uint64_t)nm : threshold;
    const Words r = philox(make_draw(rng, offset), (unsigned)(pos >> 2), (unsigned)d.tensor);
    for (int j = 0; j < 4; ++j) {
        if (pos + j >= nm) break;
        const int64_t at = d.off + pos + j;
        const bool keep = r.w[j] < below;
        float s = 0.f;
        for (int w = 0; w < workers; ++w) s += ld_elem<GBF>(grad, (int64_t)w * gstride + at) + err[(int64_t)w * estride + at];
        const float delta = keep ? s * inv_w : 0.f;
        st_elem<OBF>(out, at, delta);
        for (int w = 0; w < workers; ++w) {
            const float m = ld_elem<GBF>(grad, (int64_t)w * gstride + at) + err[(int64_t)w * estride + at];
            err[(int64_t)w * estride + at] = keep ? m - delta : m;
        }
    }
}

psgd_status launch_random_mask(psgd_plan* plan, const void* grad, float* err, double keep, const uint64_t* rng, uint64_t offset,
                               void* out, void* stream) {
    for (const MatDesc& d : plan->mats)
        if ((int64_t)d.n * d.m > (int64_t(1) << 34) || d.kept >= (int64_t(1) << 32)) {
            plan->last_error = "random mask: a matrix of more than 2^34 entries";
            return PSGD_EUNSUPPORTED;
        }
    if (!plan->uploaded) {
        psgd_status st = upload_tables(plan);
        if (st != PSGD_OK) return st;
    }
    const int64_t slices = plan->flat_tiles + plan->flat_vec_tiles;
    if (slices > 0x7fffffffLL) {
        plan->last_error = "random mask: more than 2^31 slices of 1024 elements";
        return PSGD_EUNSUPPORTED;
    }
    if (slices == 0) return PSGD_OK;
    const uint64_t threshold = keep < 0 ? 0 : (uint64_t)(keep * 4294967296.0 + 0.5);
    const bool gbf = plan->grad_dtype == PSGD_BF16, obf = plan->out_dtype == PSGD_BF16;
    auto k = gbf ? (obf ? k_random_mask<true, true> : k_random_mask<true, false>)
                 : (obf ? k_random_mask<false, true> : k_random_mask<false, false>);
    hipLaunchKernelGGL(k, dim3((unsigned)slices), dim3(kBlock), 0, static_cast<hipStream_t>(stream), plan->dev.mats,
                       plan->dev.flat_first, (int)plan->mats.size(), grad, err, out, plan->workers, plan->sizes.grad_stride,
                       plan->sizes.err_stride, plan->sizes.n_mat_elems, plan->sizes.n_vec_elems, keep < 0 ? 1 : 0, threshold, rng, offset);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { plan->last_error = std::string("launch k_random_mask: ") + hipGetErrorString(e); return PSGD_EHIP; }
    return PSGD_OK;
}

}  // namespace psgd
