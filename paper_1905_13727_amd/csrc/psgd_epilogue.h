// Activations and the steps behind a product, on the device, in fp32.
#ifndef PSGD_EPILOGUE_H
#define PSGD_EPILOGUE_H

#include <type_traits>

#include "psgd_device.h"
#include "psgd_product.h"
#include "psgd_random.h"

namespace psgd {

__device__ __forceinline__ float ld_any(const void* p, int64_t at, bool bf) {
    return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[at]) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void st_any(void* p, int64_t at, float v, bool bf) {
    if (bf) static_cast<bf16_t*>(p)[at] = f32_to_bf16(v);
    else static_cast<float*>(p)[at] = v;
}

// The hardware's exponential and reciprocal (one unit in the last place each) in place of the library's division and erff:
// behind a 4096 x 8192 x 2048 bf16 product gelu took 36 us on top of 123 with erff and takes 12 so, silu 24 with a division and 1.
constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + exp(-v)) and 1 minus that, both without cancellation or overflow
__device__ __forceinline__ void logistic(float v, float& s, float& rest) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    s = v >= 0.f ? big : small;
    rest = v >= 0.f ? small : big;
}
constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f;   // 2 sqrt(2 / pi)

// The normal distribution's tail beyond |z| and exp(-z^2 / 2): erfc by Abramowitz and Stegun 7.1.26 (error below 1.5e-7, and what the polynomial's
// terms round: gelu's slope is off by less than 3.1e-7 (1 + |z|), measured)
__device__ __forceinline__ void normal_tail(float z, float& tail, float& e) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    e = __builtin_amdgcn_exp2f(-kLog2e * x * x);
    const float p = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
    tail = 0.5f * p * t * e;
}
// z times the normal distribution function: its logit is odd, z times a polynomial in z^2 that was fitted here by least squares weighted by
// what it does to the product (up to |z| = 5.25, a line beyond).  Accurate in absolute terms: off by less than 1.2e-7 (1 + |z|) (1.19e-7 measured
// here, over 3e8 values within 20).  Of itself below zero it is off by 2e-5 down to z = -3, 3e-4 to -4, 4 % to -5, where it is 1.4e-6, and further out
// by more than it is: five times at -6 (5.9e-9), 200 times at -7; five instructions fewer than from the tail.
__device__ __forceinline__ float normal_times(float z) {
    const float s = fminf(z * z, 27.5625f);
    const float q = fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(5.1916578e-9f, s, -3.843032e-7f), s, 1.14414815e-5f), s, -1.59316e-4f), s, -9.582103e-5f), s, 0.10483888f), s, 2.302207f);
    return fmaxf(z, -40.f) * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-z * q));
}
// At infinities the activations and slopes take their limits: a factor that grows stops where the other has vanished, and NaN stays NaN
constexpr float kFar = 40.f;   // the normal tail is zero from here on, and so is the logistic function's of gelu_tanh's argument
__device__ __forceinline__ float within(float z, float far) { return z > far ? far : z < -far ? -far : z; }

__device__ __forceinline__ float act_of(float z, int act) {
    switch (act) {
        case PSGD_ACT_RELU: return z < 0.f ? 0.f : z;
        case PSGD_ACT_GELU: return normal_times(z);
        case PSGD_ACT_GELU_TANH: return fmaxf(z, -kFar) * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * kGeluA * z * fmaf(kGeluB * z, z, 1.f)));
        case PSGD_ACT_SILU: return fmaxf(z, -200.f) * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        default: return z;
    }
}
__device__ __forceinline__ float act_slope(float z, int act) {
    float s, rest;
    switch (act) {
        case PSGD_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case PSGD_ACT_GELU: {
            float tail, e;
            normal_tail(z, tail, e);
            return (z >= 0.f ? 1.f - tail : tail) + within(z, kFar) * e * 0.39894228040143268f;
        }
        case PSGD_ACT_GELU_TANH:
            z = within(z, kFar);
            logistic(kGeluA * (z + kGeluB * z * z * z), s, rest);
            return s + z * s * rest * kGeluA * (1.f + 3.f * kGeluB * z * z);
        case PSGD_ACT_SILU: z = within(z, 200.f); logistic(z, s, rest); return s * (1.f + z * rest);
        default: return 1.f;
    }
}

// Eight at a time, the choice made once
__device__ __forceinline__ void act_oct(float (&v)[8], int act) {
    auto all = [&](auto kind) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = act_of(v[e], decltype(kind)::value);
    };
    switch (act) {
        case PSGD_ACT_RELU: all(std::integral_constant<int, PSGD_ACT_RELU>()); break;
        case PSGD_ACT_GELU: all(std::integral_constant<int, PSGD_ACT_GELU>()); break;
        case PSGD_ACT_GELU_TANH: all(std::integral_constant<int, PSGD_ACT_GELU_TANH>()); break;
        case PSGD_ACT_SILU: all(std::integral_constant<int, PSGD_ACT_SILU>()); break;
        default: break;
    }
}
__device__ __forceinline__ void slope_oct(const float (&z)[8], float (&v)[8], int act) {   // v times the slope at z
    auto all = [&](auto kind) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= act_slope(z[e], decltype(kind)::value);
    };
    switch (act) {
        case PSGD_ACT_RELU: all(std::integral_constant<int, PSGD_ACT_RELU>()); break;
        case PSGD_ACT_GELU: all(std::integral_constant<int, PSGD_ACT_GELU>()); break;
        case PSGD_ACT_GELU_TANH: all(std::integral_constant<int, PSGD_ACT_GELU_TANH>()); break;
        case PSGD_ACT_SILU: all(std::integral_constant<int, PSGD_ACT_SILU>()); break;
        default: break;
    }
}

struct Epilogue {
    int64_t row0, col0;   // numbers of the first row and column, for the generator (col0 a multiple of eight)
    float scale;
    const void* bias;
    int bias_bf, act;
    void* pre;
    int64_t pre_ld;
    const void* residual;
    int64_t residual_ld;
    DropArgs drop;
};

inline DropArgs drop_of(const DropHost& h) {
    DropArgs d;
    d.rng = h.rng;
    d.offset = h.offset;
    d.below = h.below;
    d.factor = h.factor;
    return d;
}
inline Epilogue epilogue_of(const EpilogueHost& h) {
    return Epilogue{h.row0, h.col0, h.scale, h.bias, h.bias_bf, h.act, h.pre, h.pre_ld, h.residual, h.residual_ld, drop_of(h.drop)};
}

// Sixteen bytes that begin anywhere an element may: this generation's global accesses need no more than that, so rows of odd
// lengths and views that start anywhere take the same wide accesses.
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

template <bool ONCE>
__device__ __forceinline__ v4u ld_four(const v4u_any* p) {   // ONCE: around the caches
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE>
__device__ __forceinline__ v4f ld_four(const v4f_any* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

// Eight consecutive elements of a row, `count` of which exist
template <bool BF, bool ONCE = false>
__device__ __forceinline__ void ld_oct(const void* p, int64_t at, int count, float (&x)[8]) {
    if (count >= 8) {
        if constexpr (BF) {
            const v4u t = ld_four<ONCE>(reinterpret_cast<const v4u_any*>(static_cast<const bf16_t*>(p) + at));
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(t[e] << 16); x[2 * e + 1] = __uint_as_float(t[e] & 0xffff0000u); }
        } else {
            const v4f lo = ld_four<ONCE>(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at));
            const v4f hi = ld_four<ONCE>(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at + 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = lo[e]; x[4 + e] = hi[e]; }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < count ? ld_any(p, at + e, BF) : 0.f;
    }
}
template <bool BF>
__device__ __forceinline__ void st_oct(void* p, int64_t at, int count, const float (&x)[8]) {
    if (count >= 8) {
        if constexpr (BF) {
            *reinterpret_cast<v4u_any*>(static_cast<bf16_t*>(p) + at) =
                v4u{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        } else {
            *reinterpret_cast<v4f_any*>(static_cast<float*>(p) + at) = v4f{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<v4f_any*>(static_cast<float*>(p) + at + 4) = v4f{x[4], x[5], x[6], x[7]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < count) st_any(p, at + e, x[e], BF);
    }
}

// Eight consecutive elements as they lie in memory, `count` of which exist, the others zero: asked for early, widened where they are used
struct RawOct {
    v4u lo = v4u{0, 0, 0, 0}, hi = v4u{0, 0, 0, 0};   // bf16: lo
};
__device__ __forceinline__ RawOct ld_raw(const void* at, int64_t count, bool bf) {
    RawOct x;
    if (bf) {
        const bf16_t* p = static_cast<const bf16_t*>(at);
        if (count >= 8) x.lo = *reinterpret_cast<const v4u_any*>(p);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) x.lo[e >> 1] |= (unsigned)p[e] << (16 * (e & 1));
    } else {
        const float* p = static_cast<const float*>(at);
        if (count >= 8) {
            x.lo = __builtin_bit_cast(v4u, (v4f) * reinterpret_cast<const v4f_any*>(p));
            x.hi = __builtin_bit_cast(v4u, (v4f) * reinterpret_cast<const v4f_any*>(p + 4));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) (e < 4 ? x.lo : x.hi)[e & 3] = __float_as_uint(p[e]);
        }
    }
    return x;
}
__device__ __forceinline__ float widened(const RawOct& x, int e, bool bf) {
    const unsigned half = e & 1 ? x.lo[e >> 1] & 0xffff0000u : x.lo[e >> 1] << 16, word = e < 4 ? x.lo[e & 3] : x.hi[e & 3];
    return __uint_as_float(bf ? half : word);
}

// The bias of eight columns from j (a multiple of eight) on
__device__ __forceinline__ RawOct bias_ahead(const Epilogue& ep, int64_t j, int64_t N) {
    if (!ep.bias || j >= N) return RawOct();
    return ld_raw(static_cast<const char*>(ep.bias) + j * (ep.bias_bf ? 2 : 4), N - j, ep.bias_bf);
}
template <bool BF>
__device__ __forceinline__ RawOct residual_ahead(const Epilogue& ep, int64_t residual_at, int count) {
    return ep.residual && count > 0 ? ld_raw(static_cast<const char*>(ep.residual) + residual_at * (BF ? 2 : 4), count, BF) : RawOct();
}

// Columns j .. j + 7 (j a multiple of eight, `count` of them exist) of row i from their sums: one call of the generator.
// c_at, pre_at: where they are in each array; residual: what residual_ahead brought.
template <bool BF>
__device__ __forceinline__ void finish_oct(const Epilogue& ep, const Draw& d, void* c, int64_t c_at, int64_t pre_at,
                                           int64_t i, int64_t j, int count, const float (&sum)[8], const float (&bias)[8], const RawOct& residual) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sum[e] * ep.scale + bias[e];
    if (ep.pre) st_oct<BF>(ep.pre, pre_at, count, v);
    act_oct(v, ep.act);
    if (ep.drop.below) {
        const Words r = philox(d, (unsigned)((ep.col0 + j) >> 3), (unsigned)(ep.row0 + i));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = dropped(r, e, ep.drop.below) ? 0.f : v[e] * ep.drop.factor;
    }
    if (ep.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += widened(residual, e, BF);
    }
    st_oct<BF>(c, c_at, count, v);
}

// The same where all eight exist and neither dropout nor a residual follows; c and pre point at them
template <bool BF, int ACT>
__device__ __forceinline__ void finish_oct(float scale, const float (&bias)[8], char* c, char* pre, const float (&sum)[8]) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sum[e] * scale + bias[e];
    if (pre) st_oct<BF>(pre, 0, 8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_of(v[e], ACT);
    st_oct<BF>(c, 0, 8, v);
}

}  // namespace psgd

#endif
