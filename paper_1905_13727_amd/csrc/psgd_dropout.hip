// Dropout and the random mask: the two elementwise operators on the counter-based generator.
#include <hip/hip_runtime.h>

#include <string>
#include <type_traits>

#include "psgd_epilogue.h"

namespace psgd {

// y = residual + D(x).  One lane: eight consecutive columns of a row, one call of the generator.  A workgroup: `high` rows of a band of
// `wide` groups of eight columns, about kDropItems of them, or one a lane where there are too few for every unit; which row an item lies
// in is a multiplication (recip = ceil(2^32 / wide), 0 for one group; exact below 2^16 items).
// ONCE: large calls read around the caches, so that those are left to what they write: 16384 x 2048 bf16 with a residual 41 us without, 36.6 with
// it; 8192 x 2048 20.3 and 19.6, 4096 x 2048 11.2 and 13.8; rows that begin at any element share lines, 8191 x 8191 57 and 60.
// Memory bounds it, not the generator: 5.5 TB/s and 4.7 for these.
constexpr int kDropItems = 1024, kDropFew = 256 * kDropItems;
constexpr int64_t kDropOnceBytes = int64_t(96) << 20;   // read and written

template <bool BF, bool ONCE>
__global__ __launch_bounds__(kBlock) void k_dropout(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld, void* y,
                                                    int64_t y_ld, int64_t rows, int64_t cols, int wide, int high, unsigned recip,
                                                    int64_t bands, DropArgs drop) {
    const int64_t strip = blockIdx.x / bands, g0 = (blockIdx.x - strip * bands) * wide, row0 = strip * high;
    const int n = (int)(rows - row0 < high ? rows - row0 : high) * wide;
    const DrawWords words = drop.below ? words_ahead(drop.rng, drop.offset) : DrawWords{0, 0, 0, 0};   // in flight with the first loads
    for (int item = threadIdx.x; item < n; item += kBlock) {
        const int r = recip ? (int)__umulhi((unsigned)item, recip) : item;
        const int64_t row = row0 + r, col = 8 * (g0 + item - r * wide);
        const int count = (int)(cols - col < 8 ? cols - col : 8);
        if (count <= 0) continue;
        float v[8], z[8];
        ld_oct<BF, ONCE>(x, row * x_ld + col, count, v);
        if (residual) ld_oct<BF, ONCE>(residual, row * residual_ld + col, count, z);
        if (drop.below) {
            const Words w = philox(make_draw(words), (unsigned)(col >> 3), (unsigned)row);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = dropped(w, e, drop.below) ? 0.f : v[e] * drop.factor;
        }
        if (residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += z[e];
        }
        st_oct<BF>(y, row * y_ld + col, count, v);
    }
}

psgd_status launch_dropout(const DropoutCall& c, std::string* what) {
    const int64_t groups = (c.cols + 7) / 8;
    const int items = c.rows * groups <= kDropFew ? kBlock : kDropItems;   // 700 x 650 fp32 5.0 us with 1024, 3.5 with 256
    const int wide = (int)(groups < items ? groups : items);
    const int high = wide < items ? items / wide : 1;
    const unsigned recip = wide > 1 ? (unsigned)(((uint64_t(1) << 32) + wide - 1) / wide) : 0;
    const int64_t bands = (groups + wide - 1) / wide, blocks = (c.rows + high - 1) / high * bands;
    if (blocks > most_groups(kBlock)) return PSGD_EUNSUPPORTED;   // more than 2^36 elements
    const int64_t z = c.bf16 ? 2 : 4;
    auto aligned = [&](const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * z)) % 16 == 0; };
    const bool once = c.rows * c.cols * z * (c.residual ? 3 : 2) >= kDropOnceBytes && aligned(c.x, c.x_ld) && (!c.residual || aligned(c.residual, c.residual_ld));
    auto k = c.bf16 ? (once ? k_dropout<true, true> : k_dropout<true, false>) : (once ? k_dropout<false, true> : k_dropout<false, false>);
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(kBlock), 0, static_cast<hipStream_t>(c.stream), c.x, c.x_ld, c.residual,
                       c.residual_ld, c.y, c.y_ld, c.rows, c.cols, wide, high, recip, bands, drop_of(c.drop));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { *what = std::string("launch k_dropout: ") + hipGetErrorString(e); return PSGD_EHIP; }
    return PSGD_OK;
}

// ---- random mask ---------------------------------------------------------------------------------------------------

// Four consecutive entries of the gradient, read once, and of Delta', written once
template <bool BF>
__device__ __forceinline__ v4f ld_grad4(const void* p, int64_t at) {
    if constexpr (BF) {
        const v2u t = __builtin_nontemporal_load(reinterpret_cast<const v2u*>(static_cast<const bf16_t*>(p) + at));
        return v4f{__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xffff0000u), __uint_as_float(t.y << 16), __uint_as_float(t.y & 0xffff0000u)};
    } else {
        return __builtin_nontemporal_load(reinterpret_cast<const v4f*>(static_cast<const float*>(p) + at));
    }
}
template <bool BF>
__device__ __forceinline__ void st_out4(void* p, int64_t at, v4f v) {
    if constexpr (BF)
        __builtin_nontemporal_store(v2u{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)}, reinterpret_cast<v2u*>(static_cast<bf16_t*>(p) + at));
    else __builtin_nontemporal_store(v, reinterpret_cast<v4f*>(static_cast<float*>(p) + at));
}

// blockIdx.x: a slice of kFlatTileElems elements (as k_ef_add_zero's); one lane: four consecutive entries of one matrix and
// all workers.  Entry `pos` of tensor t takes word pos % 4 of the counter (pos / 4, t) and is kept where it is below
// `threshold`, or, with `budget`, below the share of the entries that the plan keeps.  Up to CAP workers' M stay in registers from
// the mean to the new error memory, so every element moves once; with more (CAP = 0) M is written, and the lanes that keep
// something read theirs again.  STREAM: the error memory goes around the caches, where the plan says that all workers' is larger than
// they are: fp32, ResNet18-shaped, 16 workers 438 us without, 411 with; transformer of 4 layers, bf16, 590 and 568; 4 workers of the
// first set 88 and 98.
// Memory bounds it: 5.3 and 6.5 TB/s there of 4 W + 8 W + 4 bytes an element; one call of the generator for four entries is hidden.  Beyond 16 workers the
// second walk shows: the first set, 17 workers 513 us, 32 1026, 64 2240, 4.5 to 3.9 TB/s of the same bytes.
template <bool GBF, bool OBF, int CAP, bool STREAM>
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
            for (int w = 0; w < workers; ++w) s += ld_any(grad, (int64_t)w * gstride + n_mat_elems + idx, GBF);
            st_any(out, n_mat_elems + idx, s * inv_w, OBF);
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
    if (pos >= nm) return;
    const int64_t at = d.off + pos;
    const uint64_t below = budget ? ((uint64_t)d.kept << 32) / (uint64_t)nm : threshold;
    auto ld_err = [](const float* e) {
        if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const v4f*>(e));
        else return *reinterpret_cast<const v4f*>(e);
    };
    auto st_err = [](float* e, v4f v) {
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<v4f*>(e));
        else *reinterpret_cast<v4f*>(e) = v;
    };
    if (pos + 4 <= nm) {   // matrices start on multiples of 64 elements: aligned
        v4f sum = v4f{0.f, 0.f, 0.f, 0.f};
        constexpr int kHeld = CAP > 0 ? CAP : 1;
        v4f m[kHeld];
        if constexpr (CAP > 0) {
#pragma unroll
            for (int w = 0; w < CAP; ++w)
                if (w < workers) m[w] = ld_grad4<GBF>(grad, w * gstride + at) + ld_err(err + w * estride + at);
#pragma unroll
            for (int w = 0; w < CAP; ++w)
                if (w < workers) sum += m[w];
        } else {
            for (int w = 0; w < workers; ++w) {
                v4f* e = reinterpret_cast<v4f*>(err + w * estride + at);
                const v4f t = ld_grad4<GBF>(grad, w * gstride + at) + *e;
                *e = t;
                sum += t;
            }
        }
        const Words r = philox(make_draw(rng, offset), (unsigned)(pos >> 2), (unsigned)d.tensor);
        v4f delta;
        bool any = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool keep = r.w[j] < below;
            any |= keep;
            delta[j] = keep ? sum[j] * inv_w : 0.f;
        }
        if constexpr (CAP > 0) {
#pragma unroll
            for (int w = 0; w < CAP; ++w)
                if (w < workers) st_err(err + w * estride + at, m[w] - delta);
        } else if (any) {
            for (int w = 0; w < workers; ++w) {
                v4f* e = reinterpret_cast<v4f*>(err + w * estride + at);
                *e = *e - delta;
            }
        }
        st_out4<OBF>(out, at, delta);
        return;
    }
    const Words r = philox(make_draw(rng, offset), (unsigned)(pos >> 2), (unsigned)d.tensor);
#pragma unroll
    for (int j = 0; j < 4; ++j) {   // a matrix's last one to three entries
        if (pos + j >= nm) break;
        float s = 0.f;
        for (int w = 0; w < workers; ++w) s += ld_any(grad, w * gstride + at + j, GBF) + err[w * estride + at + j];
        const float delta = r.w[j] < below ? s * inv_w : 0.f;
        st_any(out, at + j, delta, OBF);
        for (int w = 0; w < workers; ++w) {
            float* e = err + w * estride + at + j;
            *e = ld_any(grad, w * gstride + at + j, GBF) + *e - delta;
        }
    }
}

psgd_status launch_random_mask(psgd_plan* plan, const void* grad, float* err, double keep, const uint64_t* rng, uint64_t offset,
                               void* out, void* stream) {
    for (const MatDesc& d : plan->mats)
        if (keep < 0 && d.kept >= (int64_t(1) << 32)) {
            plan->last_error = "random mask: a budget of 2^32 entries of a matrix or more";
            return PSGD_EUNSUPPORTED;
        }
    const int64_t slices = plan->flat_tiles + plan->flat_vec_tiles;   // fewer than 2^24, so a matrix has fewer than 2^34 entries too
    if (slices > most_groups(kBlock)) {
        plan->last_error = "random mask: 2^34 elements or more";
        return PSGD_EUNSUPPORTED;
    }
    if (!plan->uploaded) {
        psgd_status st = upload_tables(plan);
        if (st != PSGD_OK) return st;
    }
    if (slices == 0) return PSGD_OK;
    const uint64_t threshold = keep < 0 ? 0 : (uint64_t)(keep * 4294967296.0 + 0.5);
    const bool gbf = plan->grad_dtype == PSGD_BF16, obf = plan->out_dtype == PSGD_BF16;
    auto by_workers = [&](auto g, auto o) {
        constexpr bool G = decltype(g)::value, O = decltype(o)::value;
        auto streamed = [&](auto s) {
            constexpr bool S = decltype(s)::value;
            return plan->workers == 1 ? k_random_mask<G, O, 1, S> : plan->workers <= 4 ? k_random_mask<G, O, 4, S> : k_random_mask<G, O, 16, S>;
        };
        if (plan->workers > 16) return k_random_mask<G, O, 0, false>;   // its second walk reads what the first wrote
        return plan->stream_hints ? streamed(std::true_type()) : streamed(std::false_type());
    };
    auto k = gbf ? (obf ? by_workers(std::true_type(), std::true_type()) : by_workers(std::true_type(), std::false_type()))
                 : (obf ? by_workers(std::false_type(), std::true_type()) : by_workers(std::false_type(), std::false_type()));
    hipLaunchKernelGGL(k, dim3((unsigned)slices), dim3(kBlock), 0, static_cast<hipStream_t>(stream), plan->dev.mats,
                       plan->dev.flat_first, (int)plan->mats.size(), grad, err, out, plan->workers, plan->sizes.grad_stride,
                       plan->sizes.err_stride, plan->sizes.n_mat_elems, plan->sizes.n_vec_elems, keep < 0 ? 1 : 0, threshold, rng, offset);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { plan->last_error = std::string("launch k_random_mask: ") + hipGetErrorString(e); return PSGD_EHIP; }
    return PSGD_OK;
}

}  // namespace psgd
