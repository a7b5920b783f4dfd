// Products of the linear layer on the matrix cores: C[i][j] = sum_l A(i, l) B(j, l) with an epilogue.
#ifndef PSGD_PRODUCT_H
#define PSGD_PRODUCT_H

#include <stdint.h>

#include <string>

#include "psgd_linear_rules.h"

namespace psgd {

// What follows the sums, in this order: times scale, plus bias, stored as `pre`, activation, dropout, plus residual (or plus what C
// holds: residual = C), stored.
struct EpilogueHost {
    int64_t row0 = 0, col0 = 0;   // numbers of the first row and column, for dropout
    float scale = 1.f;
    const void* bias = nullptr;
    bool bias_bf = false;
    int act = PSGD_ACT_IDENTITY;
    void* pre = nullptr;
    int64_t pre_ld = 0;
    const void* residual = nullptr;
    int64_t residual_ld = 0;
    DropHost drop{};
};

// Either operand lies along the contraction (`along`: element (i, l) at i * ld + l) or across it (l * ld + i).  bf16: `ready` says
// that the base is aligned to 16 bytes, ld a multiple of eight, and so the contiguous extent, or that what follows it up to the next
// multiple is readable and zero; with both ready the operands go straight to LDS.  b_fp32: B is fp32, and rounded.
struct ProductCall {
    bool bf16;
    const void* a;
    int64_t a_ld;
    bool a_along, a_ready;
    const void* b;
    int64_t b_ld;
    bool b_along, b_ready, b_fp32;
    void* c;
    int64_t c_ld;
    int64_t M, N, K;
    EpilogueHost ep;
    float* partial;          // scratch of product_partial_bytes
    hipStream_t stream;
};

// Scratch for the product and for any with fewer rows M or a shorter contraction
int64_t product_partial_bytes(bool bf16, int64_t M, int64_t N, int64_t K);
psgd_status launch_product(const ProductCall& c, std::string* what);

// The bias gradient: sums of the columns over blocks of kSumRows rows, [ceil(T / kSumRows)][n], added up and written (or added) to db.
// With `dy` the blocks' sums are of that array and still to be computed, otherwise `sums` holds them.
struct ColumnSums {
    const void* dy;
    int64_t dy_ld, T, n;
    float* sums;
    float scale;
    void* db;
    int accumulate;
};
// The input gradient (A along, B across) and the weight gradient (both across) of a layer, each may be null, and its bias gradient.
// x and w have scratch of their own.
psgd_status launch_backward_products(bool bf16, const ProductCall* x, const ProductCall* w, const ColumnSums* sums, hipStream_t stream,
                                     std::string* what);

// The forward product where few_tokens says so
psgd_status launch_few_tokens(const LinearCall& c, const EpilogueHost& ep, std::string* what);

}  // namespace psgd

#endif
