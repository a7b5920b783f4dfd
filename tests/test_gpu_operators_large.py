"""Large calls of the linear layer on the GPU, against fp64 on the device: the most tokens, and the launches that only large layers take.

Tolerances as in test_gpu_operators.py (u = half a step of the output type, v = 2^-24)."""
import numpy as np
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import operators_oracle as OO
from test_gpu_operators import DT, OFFSET, SEED, SHIFT, U, V, Layer, _need_gpu, _rng, near_on_device

pytestmark = pytest.mark.gpu


def test_the_most_tokens():
    """2^30 tokens of two features: more tiles of 64 rows than one launch takes.  Rows of both ends and around 2^29, whose sums of two
    products and a bias are off by at most 4 v of their terms."""
    dev = _need_gpu()
    T, n, k = 1 << 30, 2, 2
    L = Layer(n, k, "bf16", "bf16", dev)
    x = torch.empty(T, k, dtype=torch.bfloat16, device=dev)
    rows = [slice(0, 128), slice((1 << 29) - 64, (1 << 29) + 64), slice(T - 128, T)]
    for r in rows:
        x[r] = L.normal(128, k)
    y = torch.full((T, n), -7.0, dtype=torch.bfloat16, device=dev)
    L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T), drop=0.25, rng=_rng(dev), **L.op())
    W, b = L.param[L.w_at:L.w_at + n * k].double().view(n, k), L.param[L.b_at:L.b_at + n].double()
    for r in rows:
        factor = torch.from_numpy(OO.drop_factor(128, n, 0.25, SEED, OFFSET, first_row=r.start)).to(dev)
        X = x[r].double()
        want, e = (X @ W.T + b) * factor, 4 * V * (X.abs() @ W.abs().T + b.abs()) * factor
        near_on_device(y[r], want, e + (U["bf16"] + 4 * V) * (want.abs() + e) + 1e-37)


# Every kernel of the products, with and without a divided contraction: pass (f forward, b backward with both gradients, x or w with the
# input's or the weights' alone), tokens, n, k, types of data and parameters, direct (identity without dropout) or not.  That each of
# them takes the launch it is here for is asserted without a GPU (test_linear_routes.py).
BF, MIX, FP = ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")
CALLS = [(p, T, n, k, *types, direct) for p, T, n, k, types, direct in [
    # forward: straight to LDS, through registers, with fp32 weights, fp32; rows and columns beyond the last tile
    ("f", 3135, 1088, 200, BF, 1), ("f", 4482, 1800, 208, BF, 0), ("f", 130, 136, 200, BF, 0), ("f", 66, 72, 1736, BF, 0), ("f", 6105, 72, 8504, BF, 0),
    ("f", 5761, 583, 205, BF, 0), ("f", 66, 6855, 5171, BF, 0), ("f", 130, 131, 251, BF, 1), ("f", 40, 37, 1007, BF, 0),
    ("f", 3281, 944, 200, MIX, 0), ("f", 6165, 75, 5005, MIX, 1), ("f", 130, 136, 200, MIX, 0), ("f", 40, 72, 904, MIX, 0),
    ("f", 7396, 515, 211, FP, 0), ("f", 8731, 81, 1303, FP, 1), ("f", 130, 131, 200, FP, 0), ("f", 40, 37, 363, FP, 0),
    ("f", 1671, 2392, 3160, MIX, 0), ("f", 2061, 8192, 520, BF, 0), ("f", 3793, 1121, 361, FP, 0), ("f", 3016, 2104, 1576, MIX, 0),
    # the input gradient
    ("x", 332, 200, 8736, BF, 0), ("x", 7188, 208, 1144, BF, 1), ("x", 130, 216, 136, BF, 0), ("x", 40, 920, 72, BF, 1), ("x", 69, 5736, 6200, BF, 0),
    ("x", 6362, 211, 485, BF, 0), ("x", 71, 7471, 5277, BF, 1), ("x", 130, 211, 99, BF, 1), ("x", 40, 1207, 43, BF, 0),
    ("x", 1506, 200, 2064, MIX, 0), ("x", 69, 5608, 6656, MIX, 1), ("x", 130, 216, 136, MIX, 0), ("x", 40, 923, 43, MIX, 1),
    ("x", 8387, 200, 464, FP, 1), ("x", 68, 1208, 8640, FP, 0), ("x", 130, 131, 72, FP, 0), ("x", 40, 376, 72, FP, 1),
    ("x", 2384, 736, 6928, BF, 0), ("x", 1924, 1808, 4256, BF, 0),
    # the weight gradient
    ("w", 208, 8600, 344, BF, 0), ("w", 205, 4648, 1712, BF, 1), ("w", 202, 136, 72, BF, 0), ("w", 903, 72, 136, BF, 1), ("w", 6288, 88, 6312, BF, 0),
    ("w", 203, 2059, 1497, BF, 1), ("w", 3799, 71, 8225, BF, 1), ("w", 239, 99, 131, BF, 0), ("w", 899, 43, 37, BF, 1),
    ("w", 200, 7855, 541, FP, 0), ("w", 1188, 8424, 72, FP, 1), ("w", 203, 131, 72, FP, 0), ("w", 353, 40, 37, FP, 1), ("w", 332, 1112, 3664, FP, 0),
    # both in one launch
    ("b", 2187, 1744, 2432, MIX, 0), ("b", 2187, 1744, 2432, BF, 1), ("b", 997, 1992, 4368, MIX, 0), ("b", 997, 1992, 4368, BF, 1),
    ("b", 965, 208, 4152, FP, 0), ("b", 209, 216, 72, FP, 1), ("b", 459, 209, 8317, MIX, 0), ("b", 232, 232, 72, MIX, 1),
    ("b", 209, 3633, 1177, BF, 0), ("b", 203, 223, 43, BF, 1), ("b", 2187, 1745, 2700, MIX, 1), ("w", 2187, 1745, 1201, BF, 1), ("x", 2187, 4091, 2433, BF, 1), ("b", 6301, 200, 664, BF, 0), ("b", 210, 248, 72, BF, 1),
]] + [("f", T, n, 136, *types, direct) for T, n in ((1, 8200), (16, 8193), (20, 8208), (32, 8195)) for types in (BF, MIX, FP) for direct in (0, 1)]


def _noise(L, gen, rows, cols, std=1.0):
    return (torch.randn(rows, cols, generator=gen, device=L.dev) * std).to(DT[L.dtype])


def _gelu_slope(z):
    return 0.5 * (1 + torch.erf(z / 2 ** 0.5)) + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5


def _check_forward(L, T, direct, gen):
    dev, dtype, n, k = L.dev, L.dtype, L.n, L.k
    x, res = _noise(L, gen, T, k), None if direct else _noise(L, gen, T, n)
    more = {} if direct else dict(activation="gelu", drop=0.25, rng=_rng(dev), offset=SHIFT, residual=res)
    seen = []
    for fill in (0xFF, 0x00):   # NaN wherever the workspace is read unwritten; and the same bits whatever it holds
        y, pre = torch.full((T, n), -7.0, dtype=DT[dtype], device=dev), None if direct else torch.empty(T, n, dtype=DT[dtype], device=dev)
        L.plan.linear_forward(1, T, L.param, x, y, L.workspace(T).fill_(fill), pre=pre, **more, **L.op())
        seen.append([y] if direct else [y, pre])
    assert all(torch.equal(a, b) for a, b in zip(*seen))
    X, W, b = x.double(), L.param[L.w_at:L.w_at + n * k].to(DT[dtype]).double().view(n, k), L.param[L.b_at:L.b_at + n].double()
    z, e, u = X @ W.T + b, (k + 2) * V * (X.abs() @ W.abs().T + b.abs()), U[dtype] + 4 * V
    if direct:
        near_on_device(y, z, e + u * (z.abs() + e) + 1e-37)
        return
    near_on_device(pre, z, e + u * (z.abs() + e) + 1e-37)
    factor = torch.from_numpy(OO.drop_factor(T, n, 0.25, SEED, OFFSET + SHIFT)).to(dev)
    want, e = torch.nn.functional.gelu(z) * factor + res.double(), (1.2 * e + 16 * V * (1 + z.abs())) * factor
    near_on_device(y, want, e + u * (want.abs() + e) + 2 * V * res.double().abs() + 2 * V * (want - res.double()).abs() + 1e-37)


def _check_backward(L, T, direct, which, gen):
    dev, dtype, n, k = L.dev, L.dtype, L.n, L.k
    x, dy, pre = _noise(L, gen, T, k), _noise(L, gen, T, n), None if direct else _noise(L, gen, T, n, 2.0)
    more = {} if direct else dict(activation="gelu", pre=pre, drop=0.25, rng=_rng(dev), offset=SHIFT, accumulate=True)
    held = torch.full((2, L.plan.sizes.grad_stride), -7.0, dtype=DT[dtype], device=dev)
    if not direct:
        held[1, L.w_at:L.w_at + n * k] = _noise(L, gen, 1, n * k)[0]
        held[1, L.b_at:L.b_at + n] = _noise(L, gen, 1, n)[0]
    seen = []
    for fill in (0xFF, 0x00):
        dx, grad = torch.full((T, k), -7.0, dtype=DT[dtype], device=dev), held.clone()
        L.plan.linear_backward(1, T, L.param, x, dy, dx if which != "w" else None, grad if which != "x" else None, L.workspace(T).fill_(fill), worker=1,
                               **more, **L.op())
        seen.append([dx, grad])
    assert all(torch.equal(a, b) for a, b in zip(*seen))
    X, W, DY = x.double(), L.param[L.w_at:L.w_at + n * k].to(DT[dtype]).double().view(n, k), dy.double()
    dz, e, u = DY, torch.zeros(1, 1, dtype=torch.float64, device=dev).expand(T, n), U[dtype] + 4 * V
    if not direct:
        factor = torch.from_numpy(OO.drop_factor(T, n, 0.25, SEED, OFFSET + SHIFT)).to(dev)
        dz = DY * _gelu_slope(pre.double()) * factor
        e = 64 * V * DY.abs() * (1 + pre.double().abs()) * factor + 2 * V * dz.abs()
    e_db = e.sum(0) + (T + 2) * V * dz.abs().sum(0)
    if not direct:   # dz is rounded to the data's type for the products
        e = e + U[dtype] * (dz.abs() + e)
    a = dz.abs() + e
    if which != "w":
        err, want = e @ W.abs() + (n + 2) * V * (a @ W.abs()), dz @ W
        near_on_device(dx, want, err + u * (want.abs() + err) + 1e-37)
    if which != "x":
        for at, size, want, err in ((L.w_at, n * k, dz.T @ X, e.T @ X.abs() + (T + 2) * V * (a.T @ X.abs())), (L.b_at, n, dz.sum(0), e_db)):
            old = 0 if direct else held[1, at:at + size].double().view(want.shape)
            size_of_old = 0 if direct else old.abs()
            near_on_device(grad[1, at:at + size].view(want.shape), want + old, err + u * (want.abs() + err) + (U[dtype] + 4 * V) * size_of_old + 1e-37)
        grad[1, L.w_at:L.w_at + n * k] = held[1, L.w_at:L.w_at + n * k]
        grad[1, L.b_at:L.b_at + n] = held[1, L.b_at:L.b_at + n]
        assert torch.equal(grad, held)


@pytest.mark.parametrize("which,T,n,k,dtype,params,direct", CALLS)
def test_every_launch(which, T, n, k, dtype, params, direct):
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    gen = torch.Generator(device=dev).manual_seed(T)
    if which == "f":
        _check_forward(L, T, direct, gen)
    else:
        _check_backward(L, T, direct, which, gen)


# one layer whose forward pass takes the largest tiles and whose gradients share a launch of them, with either first; one with rows over in
# the same launch
GRAPHS = [(4096, 3080, 1544), (1500, 4104, 8200), (2061, 8192, 648)]


@pytest.mark.parametrize("T,n,k", GRAPHS)
def test_the_largest_tiles_in_a_graph(T, n, k):
    """Captured and replayed three times with eager work between, against the same calls run eagerly."""
    dev = _need_gpu()
    L = Layer(n, k, "bf16", "f32", dev)
    gen = torch.Generator(device=dev).manual_seed(T)
    x, dy, ws, rng = _noise(L, gen, T, k), _noise(L, gen, T, n), L.workspace(T), _rng(dev)
    op = {k2: v for k2, v in L.op().items() if k2 != "stream"}

    def run(y, pre, dx, grad):
        s = torch.cuda.current_stream().cuda_stream
        L.plan.linear_forward(1, T, L.param, x, y, ws, pre=pre, activation="silu", drop=0.25, rng=rng, stream=s, **op)
        L.plan.linear_backward(1, T, L.param, x, dy, dx, grad, ws, pre=pre, activation="silu", drop=0.25, rng=rng, worker=1, stream=s, **op)

    def buffers():
        return [torch.zeros(T, c, dtype=torch.bfloat16, device=dev) for c in (n, n, k)] + [torch.zeros(2, L.plan.sizes.grad_stride, dtype=torch.bfloat16, device=dev)]

    eager, replayed = buffers(), buffers()
    run(*eager)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(*replayed)
    for step in range(3):
        rng[1] = OFFSET + step
        x.copy_(_noise(L, gen, T, k))
        run(*eager)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, replayed))
        assert bool(torch.isfinite(eager[3]).all()) and float(eager[3].abs().max()) > 0


@pytest.mark.parametrize("which,T,n,k,dtype,params,direct", [c for c in CALLS if c[0] == "f" and not c[-1]])
def test_adding_to_the_residual_in_place(which, T, n, k, dtype, params, direct):
    """y is the residual itself, whichever launches a call is: the same bits as into another buffer."""
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    gen = torch.Generator(device=dev).manual_seed(n)
    x, res, ws = _noise(L, gen, T, k), _noise(L, gen, T, n), L.workspace(T)
    y, z = torch.empty_like(res), res.clone()
    for to, add in ((y, res), (z, z)):
        L.plan.linear_forward(1, T, L.param, x, to, ws, residual=add, activation="silu", drop=0.25, rng=_rng(dev), **L.op())
    assert torch.equal(y, z)


@pytest.mark.parametrize("T,n,k,dtype,params", [(20, 8208, 136, "bf16", "f32"), (66, 72, 1736, "bf16", "bf16"), (997, 1992, 4368, "bf16", "bf16"),
                                               (700, 2600, 650, "f32", "f32"), (2187, 1745, 1201, "bf16", "f32")])
def test_calls_at_the_same_time(T, n, k, dtype, params):
    """Two streams with a workspace each, over one plan and one set of parameters, and two graphs that share a workspace, replayed in turn: the
    bits of the same calls one after the other."""
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    gen = torch.Generator(device=dev).manual_seed(k)
    op = {name: v for name, v in L.op().items() if name != "stream"}
    sets = [dict(x=_noise(L, gen, T, k), dy=_noise(L, gen, T, n), ws=L.workspace(T), worker=w) for w in range(2)]

    def run(s, out, ws):
        st = torch.cuda.current_stream().cuda_stream
        L.plan.linear_forward(1, T, L.param, s["x"], out["y"], ws, pre=out["pre"], activation="gelu", drop=0.25, rng=rng, offset=s["worker"], stream=st, **op)
        L.plan.linear_backward(1, T, L.param, s["x"], s["dy"], out["dx"], grad[out["name"]], ws, pre=out["pre"], worker=s["worker"], activation="gelu", drop=0.25,
                               rng=rng, offset=s["worker"], stream=st, **op)
        L.plan.linear_backward(1, T, L.param, s["x"], s["dy"], out["dx2"], None, ws, worker=s["worker"], stream=st, **op)

    rng, dt = _rng(dev), DT[dtype]
    grad = {name: torch.zeros(2, L.plan.sizes.grad_stride, dtype=dt, device=dev) for name in ("one", "streams", "graphs")}
    outs = {name: [dict(name=name, y=torch.zeros(T, n, dtype=dt, device=dev), pre=torch.zeros(T, n, dtype=dt, device=dev), dx=torch.zeros(T, k, dtype=dt, device=dev),
                        dx2=torch.zeros(T, k, dtype=dt, device=dev)) for _ in range(2)] for name in grad}
    for s, out in zip(sets, outs["one"]):
        run(s, out, s["ws"])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    for _ in range(5):
        for st, s, out in zip(streams, sets, outs["streams"]):
            with torch.cuda.stream(st):
                run(s, out, s["ws"])
    torch.cuda.synchronize()
    graphs = []
    for s, out in zip(sets, outs["graphs"]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(s, out, sets[0]["ws"])
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.randn(1000, device=dev).sum().item()
    torch.cuda.synchronize()
    for name in ("streams", "graphs"):
        assert torch.equal(grad["one"], grad[name])
        assert all(torch.equal(a[f], b[f]) for a, b in zip(outs["one"], outs[name]) for f in ("y", "pre", "dx", "dx2"))
