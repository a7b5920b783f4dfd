// Host-side arguments of the operators around the compressor step, between the C entry points (psgd_operators.cpp) and
// the launches (psgd_linear.hip, psgd_dropout.hip).
#ifndef PSGD_OPERATORS_H
#define PSGD_OPERATORS_H

#include <stdint.h>

#include "psgd_internal.h"

namespace psgd {

constexpr int64_t kLinMaxDim = int64_t(1) << 20;      // rows, columns and strides: a tile of 256 rows of fp32 stays below 2^31 bytes
constexpr int64_t kLinMaxTokens = int64_t(1) << 30;
constexpr int64_t kLinMaxElems = int64_t(1) << 37;    // of x, y and the weights: then the products' tiles fit a launch (choose)

// The most workgroups of a launch: its lanes are counted in 32 bits
constexpr int64_t most_groups(int lanes) { return 0xffffffffLL / lanes; }

struct DropHost {
    const uint64_t* rng;
    uint64_t offset;
    uint32_t below;
    float factor;
};

// One linear layer of the plan, checked.  T tokens, n out features, k in features.
struct LinearCall {
    int64_t T, n, k;
    bool bf16, param_bf16;   // type of activations and gradients; of the parameters
    int act;
    DropHost drop;
    const void* w;           // weight and bias inside the flat parameters
    const void* bias;        // may be null
    const void* x;
    int64_t x_ld;
    // forward
    const void* residual;    // may be null
    int64_t residual_ld;
    void* pre;               // may be null
    int64_t pre_ld;
    void* y;
    int64_t y_ld;
    // backward
    const void* dy;
    int64_t dy_ld;
    void* dx;                // may be null
    int64_t dx_ld;
    void* dw;                // may be null
    void* db;                // may be null
    bool accumulate;
    void* workspace;
    void* stream;
};

struct DropoutCall {
    int64_t rows, cols;
    bool bf16;
    const void* x;
    int64_t x_ld;
    const void* residual;
    int64_t residual_ld;
    void* y;
    int64_t y_ld;
    DropHost drop;
    void* stream;
};

int64_t linear_workspace_bytes(const LinearCall& c);
int64_t linear_forward_workspace_bytes(const LinearCall& c);   // no more than that
// *what: the launch that failed and HIP's text, where the status is PSGD_EHIP
psgd_status launch_linear_forward(const LinearCall& c, std::string* what);
psgd_status launch_linear_backward(const LinearCall& c, std::string* what);
psgd_status launch_dropout(const DropoutCall& c, std::string* what);
psgd_status launch_random_mask(psgd_plan* plan, const void* grad, float* err, double keep, const uint64_t* rng, uint64_t offset,
                               void* out, void* stream);

}  // namespace psgd

#endif
