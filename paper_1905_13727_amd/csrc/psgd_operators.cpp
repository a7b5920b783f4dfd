// C entry points of the operators around the compressor step: checks of the arguments, nothing else.  Host only.
#include <algorithm>
#include <cmath>
#include <new>

#include "psgd_operators.h"

using psgd::DropHost;
using psgd::LinearCall;

namespace {

bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// p is rounded to a multiple of 2^-16
psgd_status drop_args(double p, const uint64_t* rng, uint64_t offset, DropHost* d) {
    if (!(p >= 0.0 && p <= 1.0)) return PSGD_EINVAL;   // NaN too
    d->below = (uint32_t)std::floor(p * 65536.0 + 0.5);
    d->factor = d->below < 65536u ? (float)(65536.0 / (65536.0 - d->below)) : 0.f;
    d->rng = rng;
    d->offset = offset;
    if (d->below && (!rng || !aligned(rng, 8))) return PSGD_EINVAL;
    return PSGD_OK;
}

// 0: packed rows; otherwise at least `cols`
bool stride_of(int64_t given, int64_t cols, int64_t* ld) {
    *ld = given ? given : cols;
    return given == 0 || given >= cols;
}

// What forward, backward and workspace share: the tensors of the plan, the sizes, dropout
psgd_status linear_args(const psgd_plan* plan, const psgd_linear* op, LinearCall* c) {
    if (!plan || !op) return PSGD_EINVAL;
    const int64_t count = (int64_t)plan->shapes.size();
    if (op->weight < 0 || op->weight >= count || plan->shapes[op->weight].cols < 2) return PSGD_EINVAL;
    c->n = plan->shapes[op->weight].rows;
    c->k = plan->shapes[op->weight].cols;
    if (op->bias >= count || (op->bias >= 0 && (plan->shapes[op->bias].cols != 1 || plan->shapes[op->bias].rows != c->n))) return PSGD_EINVAL;
    if (op->activation < PSGD_ACT_IDENTITY || op->activation > PSGD_ACT_SILU) return PSGD_EINVAL;
    if (op->param_dtype != PSGD_F32 && op->param_dtype != PSGD_BF16) return PSGD_EINVAL;
    if (op->tokens < 0) return PSGD_EINVAL;
    c->bf16 = plan->grad_dtype == PSGD_BF16;
    c->param_bf16 = op->param_dtype == PSGD_BF16;
    if (c->param_bf16 && !c->bf16) return PSGD_EUNSUPPORTED;
    c->T = op->tokens;
    c->act = op->activation;
    if (!stride_of(op->x_stride, c->k, &c->x_ld) || !stride_of(op->dx_stride, c->k, &c->dx_ld) ||
        !stride_of(op->residual_stride, c->n, &c->residual_ld) || !stride_of(op->pre_stride, c->n, &c->pre_ld) ||
        !stride_of(op->y_stride, c->n, &c->y_ld) || !stride_of(op->dy_stride, c->n, &c->dy_ld))
        return PSGD_EINVAL;
    for (int64_t v : {c->n, c->k, c->x_ld, c->dx_ld, c->residual_ld, c->pre_ld, c->y_ld, c->dy_ld})
        if (v > psgd::kLinMaxDim) return PSGD_EUNSUPPORTED;
    if (c->T > psgd::kLinMaxTokens) return PSGD_EUNSUPPORTED;
    const int64_t widest = std::max(c->n, c->k);
    if (c->T > psgd::kLinMaxElems / widest || c->n > psgd::kLinMaxElems / c->k) return PSGD_EUNSUPPORTED;
    return PSGD_OK;
}

const char* at(const void* base, int64_t elems, bool bf16) { return static_cast<const char*>(base) + elems * (bf16 ? 2 : 4); }

psgd_status told(psgd_plan* plan, psgd_status st, const std::string& what) {
    if (st != PSGD_OK && plan && !what.empty()) plan->last_error = what;
    return st;
}

}  // namespace

extern "C" {

psgd_status psgd_linear_workspace(const psgd_plan* plan, const psgd_linear* op, int64_t* bytes) {
    if (!bytes) return PSGD_EINVAL;
    LinearCall c{};
    psgd_status st = linear_args(plan, op, &c);
    if (st != PSGD_OK) return st;
    *bytes = psgd::linear_workspace_bytes(c);
    return PSGD_OK;
}

psgd_status psgd_linear_forward_workspace(const psgd_plan* plan, const psgd_linear* op, int64_t* bytes) {
    if (!bytes) return PSGD_EINVAL;
    LinearCall c{};
    psgd_status st = linear_args(plan, op, &c);
    if (st != PSGD_OK) return st;
    *bytes = psgd::linear_forward_workspace_bytes(c);
    return PSGD_OK;
}

psgd_status psgd_linear_forward(psgd_plan* plan, const psgd_linear* op, const void* param, const void* x, const void* residual,
                                void* pre, void* y, void* workspace, void* hip_stream) try {
    LinearCall c{};
    psgd_status st = linear_args(plan, op, &c);
    if (st != PSGD_OK) return st;
    st = drop_args(op->drop, op->rng, op->offset, &c.drop);
    if (st != PSGD_OK) return st;
    if (!param) return PSGD_EINVAL;
    if (c.T == 0) return PSGD_OK;
    const size_t z = c.bf16 ? 2 : 4;
    if (!x || !y || !aligned(x, z) || !aligned(y, z) || !aligned(residual, z) || !aligned(pre, z) || !aligned(param, 16))
        return PSGD_EINVAL;
    if (!workspace || !aligned(workspace, 256)) return PSGD_EINVAL;
    c.w = at(param, plan->tensor_flat_off[op->weight], c.param_bf16);
    c.bias = op->bias >= 0 ? at(param, plan->tensor_flat_off[op->bias], c.param_bf16) : nullptr;
    c.x = x;
    c.residual = residual;
    c.pre = pre;
    c.y = y;
    c.workspace = workspace;
    c.stream = hip_stream;
    std::string what;
    return told(plan, psgd::launch_linear_forward(c, &what), what);
} catch (...) {
    return PSGD_ENOMEM;
}

psgd_status psgd_linear_backward(psgd_plan* plan, const psgd_linear* op, const void* param, const void* x, const void* pre,
                                 const void* dy, void* dx, void* grad, int32_t worker, int32_t accumulate, void* workspace,
                                 void* hip_stream) try {
    LinearCall c{};
    psgd_status st = linear_args(plan, op, &c);
    if (st != PSGD_OK) return st;
    st = drop_args(op->drop, op->rng, op->offset, &c.drop);
    if (st != PSGD_OK) return st;
    if ((!dx && !grad) || worker < 0 || worker >= plan->workers) return PSGD_EINVAL;
    const size_t z = c.bf16 ? 2 : 4;
    if (!aligned(dx, z) || !aligned(grad, z)) return PSGD_EINVAL;
    if (c.T > 0) {
        if (!dy || !aligned(dy, z)) return PSGD_EINVAL;
        if (c.act != PSGD_ACT_IDENTITY && (!pre || !aligned(pre, z))) return PSGD_EINVAL;
        if (dx && (!param || !aligned(param, 16))) return PSGD_EINVAL;
        if (grad && (!x || !aligned(x, z))) return PSGD_EINVAL;
        if (!workspace || !aligned(workspace, 256)) return PSGD_EINVAL;
    }
    c.w = param ? at(param, plan->tensor_flat_off[op->weight], c.param_bf16) : nullptr;
    c.x = x;
    c.pre = const_cast<void*>(pre);
    c.dy = dy;
    c.dx = dx;
    if (grad) {
        const int64_t base = (int64_t)worker * plan->sizes.grad_stride;
        c.dw = const_cast<char*>(at(grad, base + plan->tensor_flat_off[op->weight], c.bf16));
        c.db = op->bias >= 0 ? const_cast<char*>(at(grad, base + plan->tensor_flat_off[op->bias], c.bf16)) : nullptr;
    }
    c.accumulate = accumulate != 0;
    c.workspace = workspace;
    c.stream = hip_stream;
    std::string what;
    return told(plan, psgd::launch_linear_backward(c, &what), what);
} catch (...) {
    return PSGD_ENOMEM;
}

static psgd_status dropout(psgd_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
                           int64_t residual_stride, void* y, int64_t y_stride, double p, const uint64_t* rng, uint64_t offset,
                           void* hip_stream) {
    psgd::DropoutCall c{};
    if (dtype != PSGD_F32 && dtype != PSGD_BF16) return PSGD_EINVAL;
    if (rows < 0 || cols < 0) return PSGD_EINVAL;
    psgd_status st = drop_args(p, rng, offset, &c.drop);
    if (st != PSGD_OK) return st;
    if (!stride_of(x_stride, cols, &c.x_ld) || !stride_of(residual_stride, cols, &c.residual_ld) || !stride_of(y_stride, cols, &c.y_ld))
        return PSGD_EINVAL;
    for (int64_t v : {rows, cols, c.x_ld, c.residual_ld, c.y_ld})
        if (v > 0x7fffffffLL) return PSGD_EUNSUPPORTED;
    if (rows > 0 && cols > (int64_t(1) << 37) / rows) return PSGD_EUNSUPPORTED;   // more than any launch takes
    if (rows == 0 || cols == 0) return PSGD_OK;
    c.bf16 = dtype == PSGD_BF16;
    const size_t z = c.bf16 ? 2 : 4;
    if (!x || !y || !aligned(x, z) || !aligned(y, z) || !aligned(residual, z)) return PSGD_EINVAL;
    c.rows = rows;
    c.cols = cols;
    c.x = x;
    c.residual = residual;
    c.y = y;
    c.stream = hip_stream;
    std::string what;
    return psgd::launch_dropout(c, &what);
}

psgd_status psgd_dropout_forward(psgd_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
                                 int64_t residual_stride, void* y, int64_t y_stride, double p, const uint64_t* rng, uint64_t offset,
                                 void* hip_stream) try {
    return dropout(dtype, rows, cols, x, x_stride, residual, residual_stride, y, y_stride, p, rng, offset, hip_stream);
} catch (...) {
    return PSGD_ENOMEM;
}

psgd_status psgd_dropout_backward(psgd_dtype dtype, int64_t rows, int64_t cols, const void* dy, int64_t dy_stride, void* dx,
                                  int64_t dx_stride, double p, const uint64_t* rng, uint64_t offset, void* hip_stream) try {
    return dropout(dtype, rows, cols, dy, dy_stride, nullptr, 0, dx, dx_stride, p, rng, offset, hip_stream);
} catch (...) {
    return PSGD_ENOMEM;
}

psgd_status psgd_random_mask_step(psgd_plan* plan, const void* grad, float* err, double keep, const uint64_t* rng, uint64_t offset,
                                  void* out, void* hip_stream) try {
    if (!plan || !grad || !err || !rng || !out) return PSGD_EINVAL;
    if (std::isnan(keep) || keep > 1.0) return PSGD_EINVAL;
    if (!aligned(rng, 8) || !aligned(grad, plan->grad_dtype == PSGD_BF16 ? 8 : 16) || !aligned(err, 16) ||
        !aligned(out, plan->out_dtype == PSGD_BF16 ? 8 : 16))
        return PSGD_EINVAL;
    return psgd::launch_random_mask(plan, grad, err, keep, rng, offset, out, hip_stream);
} catch (...) {
    return PSGD_ENOMEM;
}

}  // extern "C"
