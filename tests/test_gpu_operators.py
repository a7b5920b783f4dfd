"""The linear layer, dropout and the random mask on the GPU against the fp64 oracle.

Tolerances, per element, derived from the formulas (u = half a step of the output type, v = 2^-24):
  forward   a sum of k products of fp32 sums is off by at most (k + 2) v sum |x||w|; an activation passes that on with a
            slope below 1.2 and its own evaluation adds 16 v (1 + |z|); dropout multiplies by its factor; the residual adds one
            rounding, and storing one of u.
  backward  dz is off by 64 v |dy| (1 + |pre|) factor where the slope is evaluated (each of its terms is below 1 + |z| and takes
            some ten roundings, its exponential's argument three more of up to |z|^2), and by u |dz| where it is rounded to
            bf16 for the products (slopes other than 0 and 1); the products and sums as above over n or T terms.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import operators_oracle as OO
from oracle import powersgd_oracle as O
from paper_1905_13727_amd import binding as B

pytestmark = pytest.mark.gpu

V = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
CODE = {"f32": B.PSGD_F32, "bf16": B.PSGD_BF16}
SEED, OFFSET, SHIFT = 0x123456789ABCDEF, (5 << 32) + 77, 3


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _rng(dev, seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device=dev)


def _f64(t):
    return t.detach().double().cpu().numpy()


class Rows:
    """A [rows, cols] array inside a larger allocation: `lead` elements before it, a stride, sentinels around it."""

    def __init__(self, rows, cols, dtype, dev, pad=0, lead=0, values=None):
        self.rows, self.cols, self.ld, self.lead = rows, cols, cols + pad, lead
        self.flat = torch.full((lead + rows * self.ld + 16,), -7.0, dtype=dtype, device=dev)
        if values is not None:
            self.view().copy_(values)

    def view(self):
        return self.flat[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols]

    def ptr(self):
        return self.flat.data_ptr() + self.lead * self.flat.element_size()

    def around_is_untouched(self):
        a = self.flat.clone()
        a[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = -7.0
        return bool((a == -7.0).all())


class Layer:
    """One layer as tensors 1 and 3 of a plan, among others."""

    def __init__(self, n, k, dtype, params, dev, bias=True, workers=2, seed=0, std=None):
        self.n, self.k, self.dtype, self.params, self.dev = n, k, dtype, params, dev
        self.shapes = [(3, 5), (n, k), (7,), (n,), (4, 4)]
        self.plan = B.Plan(self.shapes, 2, workers, CODE[dtype], CODE[dtype])
        s = self.plan.sizes
        self.gen = torch.Generator().manual_seed(1000 + seed)
        self.param = (torch.randn(s.out_elems, generator=self.gen) * (std or 1 / math.sqrt(k))).to(DT[params]).to(dev)
        self.w_at, self.b_at = self.plan.offsets(1)[0], self.plan.offsets(3)[0]
        self.bias = 3 if bias else -1

    def weight(self):
        w = self.param[self.w_at:self.w_at + self.n * self.k]
        return _f64(w.to(DT[self.dtype])).reshape(self.n, self.k)

    def bias_values(self):
        return _f64(self.param[self.b_at:self.b_at + self.n]) if self.bias >= 0 else None

    def normal(self, rows, cols, std=1.0):
        return (torch.randn(rows, cols, generator=self.gen) * std).to(DT[self.dtype]).to(self.dev)

    def workspace(self, T):
        size = self.plan.linear_workspace(1, T, CODE[self.params])
        return torch.full((max(size, 1),), 0xFF, dtype=torch.uint8, device=self.dev)   # NaN wherever it is read unwritten

    def op(self, **more):
        return dict(bias=self.bias, param_dtype=CODE[self.params], stream=_stream(), **more)


def forward_bound(x, W, z, b, act, factor, residual, dtype, k):
    e = (k + 2) * V * (np.abs(x) @ np.abs(W).T + (0 if b is None else np.abs(b)))
    if act != "identity":
        e = 1.2 * e + 16 * V * (1 + np.abs(z))
    e = e * factor
    y = OO.act(z, act) * factor + (0 if residual is None else residual)
    return e + (U[dtype] + 4 * V) * (np.abs(y) + e) + 2 * V * (0 if residual is None else np.abs(residual)) + 1e-37


def near(got, want, bound):
    got = _f64(got)
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, "%.3g of the bound at %s" % (worst, np.unravel_index(np.argmax(np.abs(got - want) / bound), got.shape))


# sizes around the tiles' edges, rows of every alignment, one token to many, few features and many
SIZES = [(1, 1, 2), (1, 512, 640), (2, 33, 17), (3, 130, 650), (7, 1000, 129), (8, 256, 1024), (16, 96, 4096), (17, 2048, 96),
         (31, 10, 512), (33, 64, 64), (64, 5, 40), (65, 257, 72), (100, 650, 130), (127, 128, 256), (128, 384, 128), (129, 255, 136),
         (200, 264, 1000), (256, 256, 512), (257, 520, 264), (300, 1031, 48), (513, 768, 320), (1000, 136, 8),
         (40, 37, 43), (70, 9, 75), (66, 5, 7), (130, 3, 6), (300, 131, 263), (777, 333, 1001), (34, 1, 2), (90, 7, 1029)]
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", SIZES)
def test_forward(T, n, k, dtype, params):
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    x = Rows(T, k, DT[dtype], dev, values=L.normal(T, k))
    y = Rows(T, n, DT[dtype], dev)
    L.plan.linear_forward(1, T, L.param, x.ptr(), y.ptr(), L.workspace(T), **L.op())
    X, W, b = _f64(x.view()), L.weight(), L.bias_values()
    want, z = OO.linear_forward(X, W, b)
    near(y.view(), want, forward_bound(X, W, z, b, "identity", 1.0, None, dtype, k))
    assert y.around_is_untouched()


@pytest.mark.parametrize("act", B.ACTIVATIONS)
@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", [(1, 200, 64), (5, 77, 50), (40, 264, 96), (150, 129, 256), (260, 640, 264)])
def test_forward_epilogue(T, n, k, dtype, params, act):
    """Activation, dropout, residual and the stored pre-activation, over padded rows that start anywhere."""
    dev = _need_gpu()
    for case, (drop, with_res, with_pre, pad, lead) in enumerate([(0.3, True, True, 3, 1), (0.0, True, False, 8, 8), (0.5, False, True, 0, 0),
                                                                 (0.0, False, False, 1, 0)]):
        L = Layer(n, k, dtype, params, dev, bias=case != 2, seed=case)
        x = Rows(T, k, DT[dtype], dev, pad, lead, L.normal(T, k, 2.0))
        res = Rows(T, n, DT[dtype], dev, pad, lead, L.normal(T, n)) if with_res else None
        pre, y = Rows(T, n, DT[dtype], dev, pad, lead), Rows(T, n, DT[dtype], dev, 2 * pad, lead)
        L.plan.linear_forward(1, T, L.param, x.ptr(), y.ptr(), L.workspace(T), residual=res.ptr() if res else None,
                              pre=pre.ptr() if with_pre else None, activation=act, drop=drop, rng=_rng(dev), offset=SHIFT, x_stride=x.ld,
                              residual_stride=n + pad, pre_stride=pre.ld, y_stride=y.ld, **L.op())
        X, W, b = _f64(x.view()), L.weight(), L.bias_values()
        R = _f64(res.view()) if res else None
        factor = OO.drop_factor(T, n, drop, SEED, OFFSET + SHIFT)
        want, z = OO.linear_forward(X, W, b, act, factor, R)
        near(y.view(), want, forward_bound(X, W, z, b, act, factor, R, dtype, k))
        assert y.around_is_untouched() and (res is None or res.around_is_untouched())
        if with_pre:
            near(pre.view(), z, forward_bound(X, W, z, b, "identity", 1.0, None, dtype, k))
        assert pre.around_is_untouched() and (with_pre or bool((pre.flat == -7.0).all()))
        if drop and not with_res:
            assert bool((y.view()[torch.from_numpy(factor == 0).to(dev)] == 0).all())


def test_forward_adds_to_its_residual_in_place():
    dev = _need_gpu()
    for T, n, k, dtype in [(1, 300, 128, "bf16"), (20, 512, 2048, "bf16"), (300, 264, 128, "bf16"), (70, 70, 70, "f32")]:
        L = Layer(n, k, dtype, dtype, dev)
        x, y = L.normal(T, k), L.normal(T, n)
        R = _f64(y)
        L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), residual=y, **L.op())
        X, W, b = _f64(x), L.weight(), L.bias_values()
        want, z = OO.linear_forward(X, W, b, "identity", None, R)
        near(y, want, forward_bound(X, W, z, b, "identity", 1.0, R, dtype, k))


def backward_bounds(x, W, pre, dy, act, factor, dz, dtype):
    T, n = dy.shape
    e = 2 * V * np.abs(dz)
    if act in ("gelu", "gelu_tanh", "silu"):
        e = e + 64 * V * np.abs(dy) * (1 + np.abs(pre)) * factor
    e_db = e.sum(0) + (T + 2) * V * np.abs(dz).sum(0)
    if act in ("gelu", "gelu_tanh", "silu"):
        e = e + U[dtype] * (np.abs(dz) + e)
    a = np.abs(dz) + e
    e_dx = e @ np.abs(W) + (n + 2) * V * (a @ np.abs(W))
    e_dw = e.T @ np.abs(x) + (T + 2) * V * (a.T @ np.abs(x))
    return [err + (U[dtype] + 4 * V) * (np.abs(g) + err) + 1e-37 for err, g in
            ((e_dx, dz @ W), (e_dw, dz.T @ x), (e_db, dz.sum(0)))]


def run_backward(L, T, act, drop, pad=0, lead=0, worker=1, accumulate=False, want=("dx", "grad")):
    dev, dtype, n, k = L.dev, L.dtype, L.n, L.k
    x = Rows(T, k, DT[dtype], dev, pad, lead, L.normal(T, k))
    pre = Rows(T, n, DT[dtype], dev, pad, lead, L.normal(T, n, 2.0))
    dy = Rows(T, n, DT[dtype], dev, pad, lead, L.normal(T, n))
    dx = Rows(T, k, DT[dtype], dev, pad, lead)
    s = L.plan.sizes
    grad = torch.full((L.plan.workers, s.grad_stride), -7.0, dtype=DT[dtype], device=dev)
    if accumulate:
        grad[worker, L.w_at:L.w_at + n * k] = L.normal(1, n * k)[0]
        if L.bias >= 0:
            grad[worker, L.b_at:L.b_at + n] = L.normal(1, n)[0]
    held = _f64(grad[worker])
    L.plan.linear_backward(1, T, L.param if "dx" in want else None, x.ptr() if "grad" in want else None, dy.ptr(),
                           dx.ptr() if "dx" in want else None, grad if "grad" in want else None, L.workspace(T),
                           pre=None if act == "identity" else pre.ptr(), worker=worker, accumulate=accumulate, activation=act, drop=drop,
                           rng=_rng(dev), offset=SHIFT, x_stride=x.ld, pre_stride=pre.ld, dy_stride=dy.ld, dx_stride=dx.ld, **L.op())
    X, W, P, DY = _f64(x.view()), L.weight(), _f64(pre.view()), _f64(dy.view())
    factor = OO.drop_factor(T, n, drop, SEED, OFFSET + SHIFT)
    DX, DW, DB, DZ = OO.linear_backward(X, W, P, DY, act, factor)
    b_dx, b_dw, b_db = backward_bounds(X, W, P, DY, act, factor, DZ, dtype)
    if "dx" in want:
        near(dx.view(), DX, b_dx)
        assert dx.around_is_untouched()
    else:
        assert bool((dx.flat == -7.0).all())
    g = grad[worker].clone()
    if "grad" in want:
        old_w, old_b = (held[a:a + m] * accumulate for a, m in ((L.w_at, n * k), (L.b_at, n)))
        near(g[L.w_at:L.w_at + n * k].view(n, k), DW + old_w.reshape(n, k), b_dw + (U[dtype] + V) * np.abs(old_w).reshape(n, k))
        g[L.w_at:L.w_at + n * k] = -7.0
        if L.bias >= 0:
            near(g[L.b_at:L.b_at + n], DB + old_b, b_db + (U[dtype] + V) * np.abs(old_b))
            g[L.b_at:L.b_at + n] = -7.0
    # nothing else of the gradients is touched: other tensors, padding, other workers
    assert bool((g == -7.0).all()) and all(bool((grad[w] == -7.0).all()) for w in range(L.plan.workers) if w != worker)


@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", SIZES)
def test_backward(T, n, k, dtype, params):
    run_backward(Layer(n, k, dtype, params, _need_gpu()), T, "identity", 0.0)


@pytest.mark.parametrize("act", B.ACTIVATIONS)
@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", [(1, 200, 64), (5, 77, 50), (40, 264, 96), (150, 129, 256), (260, 640, 264)])
def test_backward_through_the_epilogue(T, n, k, dtype, params, act):
    dev = _need_gpu()
    run_backward(Layer(n, k, dtype, params, dev), T, act, 0.3, pad=3, lead=1)
    run_backward(Layer(n, k, dtype, params, dev, bias=False, seed=1), T, act, 0.0, pad=8, lead=8, worker=0, accumulate=True)
    run_backward(Layer(n, k, dtype, params, dev, seed=2), T, act, 0.5, want=("dx",))
    run_backward(Layer(n, k, dtype, params, dev, seed=3), T, act, 0.5, accumulate=True, want=("grad",))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(dtype):
    dev = _need_gpu()
    L = Layer(70, 33, dtype, dtype, dev)
    grad = torch.full((2, L.plan.sizes.grad_stride), -7.0, dtype=DT[dtype], device=dev)
    L.plan.linear_backward(1, 0, L.param, None, None, None, grad, None, worker=1, accumulate=True, activation="gelu", **L.op())
    assert bool((grad == -7.0).all())
    L.plan.linear_backward(1, 0, L.param, None, None, None, grad, None, worker=1, activation="gelu", **L.op())
    g = grad.clone()
    assert bool((g[1, L.w_at:L.w_at + 70 * 33] == 0).all()) and bool((g[1, L.b_at:L.b_at + 70] == 0).all())
    g[1, L.w_at:L.w_at + 70 * 33] = -7.0
    g[1, L.b_at:L.b_at + 70] = -7.0
    assert bool((g == -7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,k", [(3, 100, 96), (70, 300, 200), (300, 256, 520)])
def test_everything_dropped_and_infinities(T, n, k, dtype):
    """p = 1 leaves the residual and gradients of zero; a row of infinities or NaN stays in its row, and out of dropped places."""
    dev = _need_gpu()
    L = Layer(n, k, dtype, dtype, dev)
    x, res, y = L.normal(T, k), L.normal(T, n), torch.full((T, n), -7.0, dtype=DT[dtype], device=dev)
    x[1, 3] = float("inf")
    x[2, k - 1] = float("nan")
    ws = L.workspace(T)
    L.plan.linear_forward(1, T, L.param, x, y, ws, residual=res, drop=1.0, rng=_rng(dev), **L.op())
    assert torch.equal(y, res)
    L.plan.linear_forward(1, T, L.param, x, y, ws, drop=0.5, rng=_rng(dev), activation="relu", **L.op())
    gone = torch.from_numpy(OO.drop_factor(T, n, 0.5, SEED, OFFSET) == 0).to(dev)
    assert bool((y[gone] == 0).all())
    assert not torch.isfinite(y[2][~gone[2]]).any() and bool(torch.isfinite(y[0]).all()) and bool(torch.isfinite(y[3:]).all())
    z = _f64(x[1]) @ L.weight().T
    assert torch.equal(torch.isposinf(y[1]), torch.from_numpy(z > 0).to(dev) & ~gone[1])
    # backward: NaN and infinities of dropped places reach no gradient
    dy, pre = L.normal(T, n), L.normal(T, n)
    dy[gone] = float("nan")
    pre[gone] = float("inf")
    x = L.normal(T, k)
    dx, grad = torch.zeros(T, k, dtype=DT[dtype], device=dev), torch.zeros(2, L.plan.sizes.grad_stride, dtype=DT[dtype], device=dev)
    L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, drop=0.5, rng=_rng(dev), activation="gelu", **L.op())
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(grad).all()) and float(dx.abs().max()) > 0
    L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, drop=1.0, rng=_rng(dev), activation="gelu", **L.op())
    assert not bool(dx.any()) and not bool(grad.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", B.ACTIVATIONS)
def test_activations_far_out(act, dtype):
    """Values and slopes at infinities, far beyond overflow of their squares, and at NaN: their limits, and NaN.  The identity as weights
    hands each value to its own output."""
    dev = _need_gpu()
    n = 40
    L = Layer(n, n, dtype, dtype, dev, bias=False)
    L.param[L.w_at:L.w_at + n * n] = torch.eye(n, device=dev).to(DT[dtype]).view(-1)
    far = torch.tensor([float("inf"), 3e38, 1e20, 1000.0, 100.0, -100.0, -1000.0, -1e20, -3e38, float("-inf")]).to(DT[dtype]).to(dev)
    for T in (10, 80):   # both products
        x = torch.zeros(T, n, dtype=DT[dtype], device=dev)
        x[:10, 3] = torch.where(torch.isinf(far), torch.zeros_like(far), far)   # an infinity times the other weights' zero is NaN
        y, pre = torch.empty_like(x), torch.empty_like(x)
        L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), pre=pre, activation=act, **L.op())
        assert torch.equal(pre, x)
        v = x[:10, 3].double()
        want = v if act == "identity" else v.clamp(min=0)
        assert bool(((y[:10, 3].double() - want).abs() <= U[dtype] * want.abs() + 1e-6).all()), y[:10, 3]
        pre[:10, 3] = far
        pre[:, 5] = float("nan")
        dy = torch.zeros_like(x)
        dy[:, 3] = 1.0
        dy[:, 5] = 1.0
        dx = torch.empty_like(x)
        L.plan.linear_backward(1, T, L.param, x, dy, dx, None, L.workspace(T), pre=pre, activation=act, **L.op())
        slope = torch.ones(10, dtype=torch.float64, device=dev) if act == "identity" else (far.double() > 0).double()
        if act in ("identity", "relu"):
            assert bool(torch.isfinite(dx).all()) and torch.equal(dx[:10, 3].double(), slope)
        else:   # the NaN of column five reaches every output of its row (it meets the other weights' zeros)
            assert bool(torch.isnan(dx).all())
            dy[:, 5] = 0.0
            pre[:, 5] = 0.0
            L.plan.linear_backward(1, T, L.param, x, dy, dx, None, L.workspace(T), pre=pre, activation=act, **L.op())
            assert bool(((dx[:10, 3].double() - slope).abs() <= 1e-6).all()), dx[:10, 3]


def test_activations_at_infinities():
    """One input feature: z = x, the infinities reach the activations."""
    dev = _need_gpu()
    plan = B.Plan([(8, 2)], 1, 1)
    param = torch.zeros(plan.sizes.out_elems, device=dev)
    param[0:16:2] = 1.0
    for T in (3, 100):
        x = torch.zeros(T, 2, device=dev)
        param[1:16:2] = 1.0   # two equal features: infinities of one sign add up
        x[0], x[1], x[2] = float("inf"), float("-inf"), float("nan")
        ws = torch.empty(max(1, plan.linear_workspace(0, T)), dtype=torch.uint8, device=dev)
        for act in B.ACTIVATIONS:
            y = torch.empty(T, 8, device=dev)
            plan.linear_forward(0, T, param, x, y, ws, activation=act, stream=_stream())
            assert bool(torch.isposinf(y[0]).all()) and bool(torch.isnan(y[2]).all()), act
            assert bool((y[1] == (float("-inf") if act == "identity" else 0.0)).all()), act


@pytest.mark.parametrize("act", B.ACTIVATIONS)
def test_activations_over_their_range(act):
    """Values and slopes between -14 and 14, every product exact: what the evaluation itself is off by."""
    dev = _need_gpu()
    plan = B.Plan([(4, 2)], 1, 1)
    param = torch.zeros(plan.sizes.out_elems, device=dev)
    param[0:8:2] = 1.0
    for T in (29, 40000):
        x = torch.zeros(T, 2, device=dev)
        x[:, 0] = torch.linspace(-14, 14, T, device=dev)
        ws = torch.empty(max(1, plan.linear_workspace(0, T)), dtype=torch.uint8, device=dev)
        y, pre, dx = torch.empty(T, 4, device=dev), torch.empty(T, 4, device=dev), torch.empty(T, 2, device=dev)
        plan.linear_forward(0, T, param, x, y, ws, pre=pre, activation=act, stream=_stream())
        z = _f64(x[:, :1])
        assert torch.equal(pre, x[:, :1].expand(T, 4))
        near(y, np.broadcast_to(OO.act(z, act), (T, 4)), (16 * V * (1 + np.abs(z)) + V * np.abs(z)) * np.ones((1, 4)))
        dy = torch.zeros(T, 4, device=dev)
        dy[:, 2] = 1.0
        plan.linear_backward(0, T, param, x, dy, dx, None, ws, pre=pre, activation=act, stream=_stream())
        near(dx[:, :1], OO.act_slope(z, act), 64 * V * (1 + np.abs(z)) + 2 * V)


def near_on_device(got, want, bound):
    assert bool(torch.isfinite(got).all())
    worst = float(((got.double() - want).abs() / bound).max())
    assert worst <= 1.0, "%.3g of the bound" % worst


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", B.ACTIVATIONS)
def test_many_tiles_forward(act, dtype):
    """Large tiles inside the output and at its edges, a contraction that ends inside a step; against fp64 on the device."""
    dev = _need_gpu()
    T, n, k = 4000, 4104, 200
    L = Layer(n, k, dtype, dtype, dev)
    x, y, pre = L.normal(T, k), torch.empty(T, n, dtype=DT[dtype], device=dev), torch.empty(T, n, dtype=DT[dtype], device=dev)
    L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), pre=pre, activation=act, **L.op())
    X, W, b = x.double(), L.param[L.w_at:L.w_at + n * k].double().view(n, k), L.param[L.b_at:L.b_at + n].double()
    z, e = X @ W.T + b, (k + 2) * V * (X.abs() @ W.abs().T + b.abs())
    near_on_device(pre, z, e + (U[dtype] + 4 * V) * (z.abs() + e) + 1e-37)
    want = {"identity": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
            "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[act](z)
    if act != "identity":
        e = 1.2 * e + 16 * V * (1 + z.abs())
    near_on_device(y, want, e + (U[dtype] + 4 * V) * (want.abs() + e) + 1e-37)


@pytest.mark.parametrize("T,n,k", [(4099, 2048, 2048), (4099, 8192, 1032), (4200, 4104, 2048), (4097, 2056, 4096)])
def test_rows_beyond_the_last_tile(T, n, k):
    """Ragged batches: forward with dropout and residual, backward of a layer whose input gradient is as ragged; against fp64 on the device."""
    dev = _need_gpu()
    L = Layer(n, k, "bf16", "bf16", dev)
    W, b = L.param[L.w_at:L.w_at + n * k].double().view(n, k), L.param[L.b_at:L.b_at + n].double()
    x, res, ws, u = L.normal(T, k), L.normal(T, n), L.workspace(T), U["bf16"] + 4 * V
    y, pre = torch.empty_like(res), torch.empty_like(res)
    L.plan.linear_forward(1, T, L.param, x, y, ws, pre=pre, activation="relu", **L.op())
    X = x.double()
    z, e = X @ W.T + b, (k + 2) * V * (X.abs() @ W.abs().T + b.abs())
    near_on_device(pre, z, e + u * (z.abs() + e) + 1e-37)
    e = 1.2 * e + 16 * V * (1 + z.abs())
    near_on_device(y, z.clamp(min=0), e + u * (z.abs() + e) + 1e-37)
    L.plan.linear_forward(1, T, L.param, x, y, ws, residual=res, drop=0.25, rng=_rng(dev), **L.op())
    few = 300
    for first in (0, T - few):   # the generator's rows are the call's, whichever launch has them
        rows = slice(first, first + few)
        factor = torch.from_numpy(OO.drop_factor(few, n, 0.25, SEED, OFFSET, first_row=first)).to(dev)
        e = (k + 2) * V * (X[rows].abs() @ W.abs().T + b.abs()) * factor
        want = z[rows] * factor + res[rows].double()
        near_on_device(y[rows], want, e + u * (want.abs() + e) + 2 * V * res[rows].double().abs() + 2 * V * (z[rows] * factor).abs() + 1e-37)
    dy, dx = L.normal(T, n), torch.empty(T, k, dtype=torch.bfloat16, device=dev)
    L.plan.linear_backward(1, T, L.param, None, dy, dx, None, ws, **L.op())
    dz = dy.double()
    want, e = dz @ W, (n + 2) * V * (dz.abs() @ W.abs())
    near_on_device(dx, want, e + u * (want.abs() + e) + 1e-37)


@pytest.mark.parametrize("act,params", [("identity", "bf16"), ("relu", "f32")])
@pytest.mark.parametrize("T,n,k", [(4096, 3080, 1544), (3000, 2056, 4104), (1500, 4104, 8200)])
def test_large_gradients(T, n, k, act, params):
    """Both gradients of large layers, together in one launch and apart; against fp64 on the device."""
    dev = _need_gpu()
    L = Layer(n, k, "bf16", params, dev)
    x, dy, pre = L.normal(T, k), L.normal(T, n), L.normal(T, n)
    dx, grad = torch.empty(T, k, dtype=torch.bfloat16, device=dev), torch.full((2, L.plan.sizes.grad_stride), -7.0, dtype=torch.bfloat16, device=dev)
    L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, L.workspace(T), pre=pre if act == "relu" else None, worker=1, activation=act, **L.op())
    W = L.param[L.w_at:L.w_at + n * k].to(torch.bfloat16).double().view(n, k)
    dz = dy.double() * (pre > 0) if act == "relu" else dy.double()   # exact in bf16
    X, u = x.double(), U["bf16"] + 4 * V
    for got, want, e in ((dx, dz @ W, (n + 2) * V * (dz.abs() @ W.abs())),
                         (grad[1, L.w_at:L.w_at + n * k].view(n, k), dz.T @ X, (T + 2) * V * (dz.abs().T @ X.abs())),
                         (grad[1, L.b_at:L.b_at + n], dz.sum(0), (T + 2) * V * dz.abs().sum(0))):
        near_on_device(got, want, e + u * (want.abs() + e) + 1e-37)
    grad[1, L.w_at:L.w_at + n * k] = -7.0
    grad[1, L.b_at:L.b_at + n] = -7.0
    assert bool((grad == -7.0).all())


@pytest.mark.parametrize("T,n,k", [(600, 2304, 520), (2048, 2176, 136)])
def test_large_layers_in_a_graph(T, n, k):
    """Forward and backward through the largest tiles, captured and replayed three times with eager work between."""
    dev = _need_gpu()
    L = Layer(n, k, "bf16", "f32", dev)
    x, dy, ws, rng = L.normal(T, k), L.normal(T, n), L.workspace(T), _rng(dev)
    new = lambda c: torch.zeros(T, c, dtype=torch.bfloat16, device=dev)  # noqa: E731

    def run(y, pre, dx, grad):
        L.plan.linear_forward(1, T, L.param, x, y, ws, pre=pre, activation="silu", drop=0.25, rng=rng, **L.op())
        L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, activation="silu", drop=0.25, rng=rng, worker=1, **L.op())

    a, b = [[new(n), new(n), new(k), torch.zeros(2, L.plan.sizes.grad_stride, dtype=torch.bfloat16, device=dev)] for _ in range(2)]
    run(*a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L_op = L.op
        L.op = lambda **m: dict(L_op(**m), stream=torch.cuda.current_stream().cuda_stream)
        run(*b)
    for step in range(3):
        rng[1] = OFFSET + step
        x.copy_(L.normal(T, k))
        run(*a)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(a, b))
        assert bool(torch.isfinite(a[3]).all()) and float(a[3].abs().max()) > 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,k", [(1, 640, 2048), (12, 512, 4096), (40, 128, 1024), (600, 520, 264)])
def test_repeats_bit_for_bit(T, n, k, dtype):
    dev = _need_gpu()
    L = Layer(n, k, dtype, dtype, dev)
    x, dy, pre = L.normal(T, k), L.normal(T, n), L.normal(T, n)
    seen = []
    for fill in (0xFF, 0x00, 0x3F):
        ws = L.workspace(T).fill_(fill)
        y, dx = torch.empty(T, n, dtype=DT[dtype], device=dev), torch.empty(T, k, dtype=DT[dtype], device=dev)
        grad = torch.zeros(2, L.plan.sizes.grad_stride, dtype=DT[dtype], device=dev)
        L.plan.linear_forward(1, T, L.param, x, y, ws, activation="silu", drop=0.2, rng=_rng(dev), **L.op())
        L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, activation="silu", drop=0.2, rng=_rng(dev), **L.op())
        seen.append((y, dx, grad))
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", [(1, 96, 4096), (40, 128, 4096), (70, 33, 1001), (700, 260, 130), (300, 1031, 520), (2100, 700, 264), (130, 64, 9000)])
def test_workspace_is_enough_and_the_longest_batchs_serves_all(T, n, k, dtype, params):
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    sizes = [L.plan.linear_workspace(1, t, CODE[params]) for t in range(1, T + 1, max(1, T // 50))] + [L.plan.linear_workspace(1, T, CODE[params])]
    assert sizes == sorted(sizes)
    ws = torch.full((sizes[-1] + 8192,), 0xA5, dtype=torch.uint8, device=dev)
    x, dy, pre = L.normal(T, k), L.normal(T, n), L.normal(T, n)
    y, dx, grad = torch.empty_like(dy), torch.empty_like(x), torch.zeros(2, L.plan.sizes.grad_stride, dtype=DT[dtype], device=dev)
    L.plan.linear_forward(1, T, L.param, x, y, ws, activation="silu", **L.op())
    L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, activation="silu", drop=0.1, rng=_rng(dev), **L.op())
    L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, **L.op())
    assert bool((ws[sizes[-1]:] == 0xA5).all())


def test_rows_do_not_depend_on_the_others_mask():
    """Element (row, col) draws the same numbers whatever the batch: the first rows of a long call equal a short call's mask."""
    dev = _need_gpu()
    L = Layer(96, 64, "f32", "f32", dev)
    x = torch.ones(500, 64, device=dev)
    ys = []
    for T in (1, 3, 40, 500):
        y = torch.zeros(T, 96, device=dev)
        L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), drop=0.5, rng=_rng(dev), **L.op())
        ys.append(y == 0)
    assert all(torch.equal(ys[-1][:m.shape[0]], m) for m in ys)


@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("T,n,k", [(1027, 2064, 1032), (2055, 2049, 520), (1100, 2180, 1028), (530, 8200, 520), (4100, 520, 1100)])
def test_large_products_with_something_over(T, n, k, dtype, params):
    """Large enough that rows and columns beyond the last tile become products of their own: with everything behind the product,
    and backward."""
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    x, res = L.normal(T, k), L.normal(T, n)
    y, pre, ws = Rows(T, n, DT[dtype], dev, 3, 1), Rows(T, n, DT[dtype], dev), L.workspace(T)
    L.plan.linear_forward(1, T, L.param, x, y.ptr(), ws, residual=res, pre=pre.ptr(), activation="gelu_tanh", drop=0.3, rng=_rng(dev),
                          offset=SHIFT, y_stride=y.ld, **L.op())
    X, W, b, R = _f64(x), L.weight(), L.bias_values(), _f64(res)
    factor = OO.drop_factor(T, n, 0.3, SEED, OFFSET + SHIFT)
    want, z = OO.linear_forward(X, W, b, "gelu_tanh", factor, R)
    near(y.view(), want, forward_bound(X, W, z, b, "gelu_tanh", factor, R, dtype, k))
    near(pre.view(), z, forward_bound(X, W, z, b, "identity", 1.0, None, dtype, k))
    assert y.around_is_untouched() and pre.around_is_untouched()
    run_backward(L, T, "gelu_tanh", 0.3, accumulate=True)


def test_outputs_beyond_32_bit_offsets():
    """[70000][33280] bf16 outputs (4.7 GB) over eight columns of input: rows at both ends and behind 2^31 elements, backward too."""
    dev = _need_gpu()
    T, n, k = 70000, 33280, 8
    L = Layer(n, k, "bf16", "bf16", dev)
    x = L.normal(T, k)
    y = torch.empty(T, n, dtype=torch.bfloat16, device=dev)
    L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), drop=0.25, rng=_rng(dev), **L.op())
    for rows in (slice(0, 3), slice(32263, 32266), slice(64527, 64530), slice(T - 3, T)):
        X, W, b = _f64(x[rows]), L.weight(), L.bias_values()
        factor = OO.drop_factor(3, n, 0.25, SEED, OFFSET, first_row=range(T)[rows][0])
        want, z = OO.linear_forward(X, W, b, "identity", factor)
        near(y[rows], want, forward_bound(X, W, z, b, "identity", factor, None, "bf16", k))
    # the gradient of the sum of the last row: dy is zero but there
    y.zero_()
    y[-1] = 1.0
    dx, grad = torch.full((T, k), -7.0, dtype=torch.bfloat16, device=dev), torch.zeros(2, L.plan.sizes.grad_stride, dtype=torch.bfloat16, device=dev)
    L.plan.linear_backward(1, T, L.param, x, y, dx, grad, L.workspace(T), **L.op())
    assert not bool(dx[:-1].any())
    near(dx[-1:], L.weight().sum(0, keepdims=True), (n + 2) * V * np.abs(L.weight()).sum(0, keepdims=True) + U["bf16"] * np.abs(L.weight().sum(0)))
    assert torch.equal(grad[0, L.w_at:L.w_at + n * k].view(n, k), x[-1:].expand(n, k))
    assert bool((grad[0, L.b_at:L.b_at + n] == 1).all())


# ---- dropout by itself -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 9), (33, 650), (700, 64), (64, 8191), (2, 70001), (1023, 136)])
def test_dropout(rows, cols, dtype):
    dev = _need_gpu()
    gen = torch.Generator().manual_seed(4)
    for p, pad, lead, with_res in [(0.1, 0, 0, False), (0.5, 8, 8, True), (0.9, 3, 1, True), (0.0, 1, 0, True), (1.0, 0, 0, False)]:
        x = Rows(rows, cols, DT[dtype], dev, pad, lead, torch.randn(rows, cols, generator=gen))
        r = Rows(rows, cols, DT[dtype], dev, 2 * pad, lead, torch.randn(rows, cols, generator=gen)) if with_res else None
        y, dx = Rows(rows, cols, DT[dtype], dev, pad, lead), Rows(rows, cols, DT[dtype], dev, 5, 3)
        B.dropout_forward(CODE[dtype], rows, cols, x.ptr(), y.ptr(), p, _rng(dev) if p else None, residual=r.ptr() if r else None,
                          x_stride=x.ld, residual_stride=r.ld if r else 0, y_stride=y.ld, offset=SHIFT, stream=_stream())
        factor = OO.drop_factor(rows, cols, p, SEED, OFFSET + SHIFT)
        X, R = _f64(x.view()), _f64(r.view()) if r else None
        want = OO.dropout(X, factor, R)
        # factor rounded to fp32, product, sum, output
        bound = 2 * V * np.abs(X) * factor + (U[dtype] + V) * (np.abs(want) + 2 * V * np.abs(X) * factor) + 1e-37
        near(y.view(), want, bound)
        assert y.around_is_untouched()
        B.dropout_backward(CODE[dtype], rows, cols, x.ptr(), dx.ptr(), p, _rng(dev) if p else None, dy_stride=x.ld, dx_stride=dx.ld,
                           offset=SHIFT, stream=_stream())
        near(dx.view(), X * factor, 2 * V * np.abs(X) * factor + (U[dtype] + V) * np.abs(X) * factor + 1e-37)
        assert bool((dx.view()[torch.from_numpy(factor == 0).to(dev)] == 0).all()) and dx.around_is_untouched()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_in_place_and_of_infinities(dtype):
    dev = _need_gpu()
    x = torch.full((50, 43), float("inf"), dtype=DT[dtype], device=dev)
    x[::2] = float("nan")
    gone = torch.from_numpy(OO.drop_factor(50, 43, 0.4, SEED, OFFSET) == 0).to(dev)
    B.dropout_backward(CODE[dtype], 50, 43, x, x, 0.4, _rng(dev), stream=_stream())
    assert bool((x[gone] == 0).all()) and not bool(torch.isfinite(x[~gone]).any())
    res = torch.ones(50, 43, dtype=DT[dtype], device=dev)
    x = torch.full_like(res, 3.0)
    B.dropout_forward(CODE[dtype], 50, 43, x, res, 0.5, _rng(dev), residual=res, stream=_stream())
    assert set(res.float().unique().tolist()) == {1.0, 7.0}


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 12000, 2048), ("f32", 12289, 1032), ("bf16", 12291, 2052)])
def test_large_dropout_row_by_row(dtype, rows, cols):
    """Calls that read around the caches, and one of that size whose rows are not aligned: as the same rows a few at a time."""
    dev = _need_gpu()
    gen = torch.Generator(device=dev).manual_seed(rows)
    x, res = (torch.randn(rows, cols, device=dev, generator=gen).to(DT[dtype]) for _ in range(2))
    y = torch.empty_like(x)
    B.dropout_forward(CODE[dtype], rows, cols, x, y, 0.3, _rng(dev), residual=res, stream=_stream())
    factor = torch.from_numpy(OO.drop_factor(300, cols, 0.3, SEED, OFFSET, first_row=rows - 300)).to(dev)
    want = OO.dropout(_f64(x[-300:]), factor.cpu().numpy(), _f64(res[-300:]))
    bound = 2 * V * np.abs(_f64(x[-300:])) * 2 + (U[dtype] + V) * (np.abs(want) + 4 * V * np.abs(_f64(x[-300:]))) + 1e-37
    near(y[-300:], want, bound)
    for first in (0, 5000, rows - 64):   # a small call of the first rows draws the same for them
        if first == 0:
            z = torch.empty(64, cols, dtype=DT[dtype], device=dev)
            B.dropout_forward(CODE[dtype], 64, cols, x, z, 0.3, _rng(dev), residual=res, stream=_stream())
            assert torch.equal(z, y[:64])
        kept = torch.from_numpy(OO.drop_factor(64, cols, 0.3, SEED, OFFSET, first_row=first) == 0).to(dev)
        assert torch.equal(y[first:first + 64][kept], res[first:first + 64][kept])


def test_dropout_beyond_32_bit_offsets():
    dev = _need_gpu()
    rows, cols = 70000, 33280   # 2.3e9 elements
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=dev)
    B.dropout_forward(B.PSGD_BF16, rows, cols, x, x, 0.5, _rng(dev), stream=_stream())
    for first in (0, 32263, 64527, rows - 2):
        want = OO.drop_factor(2, cols, 0.5, SEED, OFFSET, first_row=first)
        assert np.array_equal(_f64(x[first:first + 2]), want)


# ---- random mask -------------------------------------------------------------------------------------------------------

MASK_SHAPES = [(64, 27), (64,), (130, 1028), (7,), (5, 3), (33, 31), (2, 2), (300, 77)]


@pytest.mark.parametrize("gdt,odt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("workers", [1, 2, 5, 16, 17, 40])
def test_random_mask(workers, gdt, odt):
    dev = _need_gpu()
    rank = 2
    plan = B.Plan(MASK_SHAPES, rank, workers, CODE[gdt], CODE[odt])
    s = plan.sizes
    gen = torch.Generator().manual_seed(workers)
    live = torch.zeros(s.out_elems, dtype=torch.bool)
    at = [plan.offsets(t)[0] for t in range(len(MASK_SHAPES))]
    for t, shape in enumerate(MASK_SHAPES):
        live[at[t]:at[t] + int(np.prod(shape))] = True
    for keep in (-1.0, 0.3, 0.0, 1.0):
        grad = torch.randn(workers, s.grad_stride, generator=gen).to(DT[gdt]).to(dev)
        err = torch.where(live[:s.n_mat_elems], torch.randn(workers, s.err_stride, generator=gen), torch.tensor(-7.0)).to(dev)
        out = torch.full((s.out_elems,), -7.0, dtype=DT[odt], device=dev)
        G, E = _f64(grad), _f64(err)
        plan.random_mask_step(grad, err, keep, _rng(dev), out, offset=SHIFT, stream=_stream())
        pick = lambda a, t: a[at[t]:at[t] + int(np.prod(MASK_SHAPES[t]))].reshape(MASK_SHAPES[t])  # noqa: E731
        keeps = [OO.mask_keep(*shape, t, keep, O.kept_count(*shape, rank), SEED, OFFSET + SHIFT) if len(shape) == 2 else None
                 for t, shape in enumerate(MASK_SHAPES)]
        mats = [t for t, shape in enumerate(MASK_SHAPES) if len(shape) == 2]
        want, errs = OO.random_mask_step([[pick(G[w], t) for t in range(len(MASK_SHAPES))] for w in range(workers)],
                                         [[pick(E[w], t) if t in mats else None for t in range(len(MASK_SHAPES))] for w in range(workers)], keeps)
        got, new = _f64(out), _f64(err)
        for t in range(len(MASK_SHAPES)):
            # M is rounded once, the mean W + 1 times, the difference once
            size = sum(np.abs(pick(G[w], t)) + (np.abs(pick(E[w], t)) if t in mats else 0) for w in range(workers)) / workers
            near(torch.from_numpy(pick(got, t)), want[t], (workers + 4) * V * size + U[odt] * np.abs(want[t]) + 1e-37)
            if t in mats:
                assert (pick(got, t)[~keeps[t]] == 0).all()
                for w in range(workers):
                    m = np.abs(pick(G[w], t)) + np.abs(pick(E[w], t))
                    near(torch.from_numpy(pick(new[w], t)), errs[w][t], 2 * V * m + (workers + 5) * V * (size + m) * keeps[t] + 1e-37)
        assert (got[~live.numpy()] == -7.0).all() and (new[:, ~live[:s.n_mat_elems].numpy()] == -7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("workers", [1, 3, 16, 17])
def test_random_mask_around_the_caches(workers, dtype):
    """The error memory of large sets goes around the caches: the same bits."""
    dev = _need_gpu()
    gen = torch.Generator().manual_seed(workers)
    res = []
    for hints in (0, 1):
        plan = B.Plan(MASK_SHAPES, 2, workers, CODE[dtype], CODE[dtype])
        plan.set_tuning("stream_hints", hints)
        s = plan.sizes
        if not res:
            grad = torch.randn(workers, s.grad_stride, generator=gen).to(DT[dtype]).to(dev)
            start = torch.randn(workers, s.err_stride, generator=gen).to(dev)
        err, out = start.clone(), torch.zeros(s.out_elems, dtype=DT[dtype], device=dev)
        for step in range(3):
            plan.random_mask_step(grad, err, 0.4, _rng(dev), out, offset=step, stream=_stream())
        res.append((err.view(torch.uint8).cpu(), out.view(torch.uint8).cpu()))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_random_mask_keeps_the_sum_of_updates():
    """Error feedback loses nothing: after any number of steps, sum of Delta' + mean error = sum of gradients."""
    dev = _need_gpu()
    plan = B.Plan([(40, 60)], 2, 3)
    err = torch.zeros(3, plan.sizes.err_stride, device=dev)
    rng, out = _rng(dev), torch.zeros(plan.sizes.out_elems, device=dev)
    total, sent = np.zeros(2400), np.zeros(2400)
    for step in range(8):
        grad = torch.randn(3, plan.sizes.grad_stride, device=dev, generator=torch.Generator(device=dev).manual_seed(step))
        plan.random_mask_step(grad, err, -1.0, rng, out, offset=step, stream=_stream())
        total += _f64(grad)[:, :2400].mean(0)
        sent += _f64(out)[:2400]
    left = _f64(err)[:, :2400].mean(0)
    # a step rounds sums of magnitude below 8 * 6 a few times
    assert np.abs(sent + left - total).max() < 8 * 8 * 48 * V
    assert np.count_nonzero(sent) > 1000


# ---- streams, graphs, and a run of them together --------------------------------------------------------------------------

def test_work_goes_to_the_given_stream():
    dev = _need_gpu()
    L = Layer(300, 200, "bf16", "bf16", dev)
    x, y = L.normal(90, 200), torch.zeros(90, 300, dtype=torch.bfloat16, device=dev)
    ws = L.workspace(90)
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    with torch.cuda.stream(side):
        x2 = x * 2   # the call has to wait for this, on this stream
        L.plan.linear_forward(1, 90, L.param, x2, y, ws, **L.op())
        z = y.clone()
    side.synchronize()
    X, W, b = 2 * _f64(x), L.weight(), L.bias_values()
    want, pre = OO.linear_forward(X, W, b)
    near(z, want, forward_bound(X, W, pre, b, "identity", 1.0, None, "bf16", 200))


class Net:
    """A feed-forward block with residual, y = x + D(W2 gelu(W1 x + b1) + b2), over W workers' micro-batches, and its step."""

    def __init__(self, dev, dtype, d=96, ff=200, tokens=37, workers=2, seed=0):
        self.dev, self.dtype, self.d, self.ff, self.T, self.W = dev, dtype, d, ff, tokens, workers
        self.plan = B.Plan([(ff, d), (ff,), (d, ff), (d,)], 2, workers, CODE[dtype], CODE[dtype])
        self.plan.check(_stream())
        s, gen = self.plan.sizes, torch.Generator().manual_seed(seed)
        self.at = [self.plan.offsets(t)[0] for t in range(4)]
        self.param = (torch.randn(s.out_elems, generator=gen) * 0.1).to(dev)
        self.mom = torch.zeros(s.out_elems, device=dev)
        self.grad = torch.zeros(workers, s.grad_stride, dtype=DT[dtype], device=dev)
        self.err = torch.zeros(workers, s.err_stride, device=dev)
        self.q = torch.randn(s.q_elems, generator=gen).to(dev)
        self.p = torch.zeros(s.p_elems, device=dev)
        self.ws = torch.empty(s.workspace_bytes + 64, dtype=torch.uint8, device=dev)
        self.lin_ws = torch.empty(max(self.plan.linear_workspace(t, tokens) for t in (0, 2)) or 1, dtype=torch.uint8, device=dev)
        new = lambda c: torch.zeros(tokens, c, dtype=DT[dtype], device=dev)  # noqa: E731
        self.x = torch.randn(workers, tokens, d, generator=gen).to(DT[dtype]).to(dev)
        self.pre, self.h, self.y, self.dh, self.dx = new(ff), new(ff), new(d), new(ff), new(d)
        self.rng = _rng(dev)

    def step(self, lr=0.05):
        """Loss: half the squared outputs, so dy = y."""
        p, s = self.plan, _stream()
        for w in range(self.W):
            p.linear_forward(0, self.T, self.param, self.x[w], self.h, self.lin_ws, bias=1, pre=self.pre, activation="gelu", stream=s)
            p.linear_forward(2, self.T, self.param, self.h, self.y, self.lin_ws, bias=3, residual=self.x[w], drop=0.25, rng=self.rng, offset=w,
                             stream=s)
            p.linear_backward(2, self.T, self.param, self.h, self.y, self.dh, self.grad, self.lin_ws, bias=3, worker=w, drop=0.25,
                              rng=self.rng, offset=w, stream=s)
            p.linear_backward(0, self.T, self.param, self.x[w], self.dh, None, self.grad, self.lin_ws, bias=1, worker=w, pre=self.pre,
                              activation="gelu", stream=s)
        p.step_update(self.grad, self.err, self.q, self.p, self.mom, self.param, lr, 0.9, self.ws, s)

    def oracle_gradients(self, param, offset):
        d, ff = self.d, self.ff
        W1, b1 = param[self.at[0]:self.at[0] + ff * d].reshape(ff, d), param[self.at[1]:self.at[1] + ff]
        W2, b2 = param[self.at[2]:self.at[2] + ff * d].reshape(d, ff), param[self.at[3]:self.at[3] + d]
        got = []
        for w in range(self.W):
            x, factor = _f64(self.x[w]), OO.drop_factor(self.T, d, 0.25, SEED, offset + w)
            h, pre = OO.linear_forward(x, W1, b1, "gelu")
            y, _ = OO.linear_forward(h, W2, b2, "identity", factor, x)
            dh, dW2, db2, _ = OO.linear_backward(h, W2, None, y, "identity", factor)
            _, dW1, db1, _ = OO.linear_backward(x, W1, pre, dh, "gelu")
            got.append([dW1, db1, dW2, db2])
        return got


def test_a_training_step_of_the_operators_together():
    """Forward, backward and the compressed update of two workers, against the oracle's gradients and the oracle's step."""
    dev = _need_gpu()
    net = Net(dev, "f32")
    before, q0 = _f64(net.param), _f64(net.q)
    net.step()
    net.plan.check(_stream())
    want = net.oracle_gradients(before, OFFSET)
    shapes = [(net.ff, net.d), (net.ff,), (net.d, net.ff), (net.d,)]
    for w in range(2):
        for t, shape in enumerate(shapes):
            g = _f64(net.grad[w, net.at[t]:net.at[t] + int(np.prod(shape))]).reshape(shape)
            # a chain of four products of up to 200 terms each, in norm
            assert np.linalg.norm(g - want[w][t]) <= 4 * 202 * V * np.linalg.norm(want[w][t]) + 1e-30
    offs = [net.plan.offsets(t) for t in range(4)]
    qs = [q0[o[2]:o[2] + s[1] * 2].reshape(s[1], 2) if len(s) == 2 else None for o, s in zip(offs, shapes)]
    ref = O.powersgd_step(want, [[np.zeros(s) if len(s) == 2 else None for s in shapes] for _ in range(2)], qs, 2)
    after = _f64(net.param)
    for t, s in enumerate(shapes):
        at, size = net.at[t], int(np.prod(s))
        delta = np.asarray(ref["out"][t]).reshape(-1)
        step = before[at:at + size] - after[at:at + size]   # lr (Delta' + m) with m = Delta'
        assert np.linalg.norm(step - 0.1 * delta) <= 1e-4 * np.linalg.norm(0.1 * delta) + 3 * V * np.linalg.norm(before[at:at + size])


@pytest.mark.parametrize("lr", [0.05, 0.0005])   # the larger one diverges within the replays: infinities and NaN repeat too
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_training_step_draws_anew(dtype, lr):
    """The step in a graph whose last node moves the generator's offset on, replayed with eager work between, against the same
    steps run eagerly: equal bit for bit, and another mask each time."""
    dev = _need_gpu()
    eager, graph = Net(dev, dtype), Net(dev, dtype)

    def one(net):
        net.step(lr)
        net.rng[1].add_(net.W)

    one(eager)
    one(graph)   # the first call may load code
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    held = [t.clone() for t in (graph.param, graph.mom, graph.err, graph.q, graph.rng)]
    with torch.cuda.graph(g):
        one(graph)
    for t, h in zip((graph.param, graph.mom, graph.err, graph.q, graph.rng), held):
        t.copy_(h)
    seen = []
    for _ in range(4):
        one(eager)
        g.replay()
        torch.cuda.synchronize()
        for name in ("param", "mom", "err", "grad", "y", "rng"):
            a, b = (getattr(net, name).contiguous().view(torch.uint8) for net in (eager, graph))
            assert torch.equal(a, b), name
        seen.append(graph.y.clone())
        torch.randn(1000, device=dev).sum().item()
    assert not torch.equal(seen[0], seen[1])
    assert lr > 0.001 or bool(torch.isfinite(seen[-1]).all())
