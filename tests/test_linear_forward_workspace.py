"""Scratch of the forward pass by itself: its size (CPU), and that the pass stays within it (GPU)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1905_13727_amd import binding as B

TYPES = [(B.PSGD_F32, B.PSGD_F32), (B.PSGD_BF16, B.PSGD_BF16), (B.PSGD_BF16, B.PSGD_F32)]


@pytest.mark.parametrize("dtype,params", TYPES)
@pytest.mark.parametrize("n,k", [(2048, 8192), (650, 2601), (8200, 64), (7, 3000), (50304, 2048)])
def test_no_more_than_both_passes_need_and_growing(n, k, dtype, params):
    plan = B.Plan([(n, k), (n,)], 2, 1, dtype, dtype)
    tokens = [0, 1, 4, 5, 16, 17, 32, 33, 100, 639, 640, 999, 1000, 4096, 65537, 1 << 20]
    sizes = [plan.linear_forward_workspace(0, t, params) for t in tokens]
    assert sizes == sorted(sizes) and sizes[0] == 0 < sizes[1]
    assert all(s <= plan.linear_workspace(0, t, params) for s, t in zip(sizes, tokens))


def test_logits_need_no_scratch_for_gradients():
    plan = B.Plan([(50304, 2048)], 2, 1, B.PSGD_BF16, B.PSGD_BF16)
    # at most a copy of x and the sums of a divided contraction
    assert plan.linear_forward_workspace(0, 8192, B.PSGD_BF16) <= 8192 * 2048 * 2 + (64 << 20)
    assert plan.linear_workspace(0, 8192, B.PSGD_BF16) > 8192 * 50304 * 2


def test_refuses_as_the_other():
    plan, n, op = B.Plan([(6, 8), (6,)], 2), C.c_int64(), B.psgd_linear(weight=0, bias=-1, tokens=3)
    lib = plan._lib
    assert lib.psgd_linear_forward_workspace(plan._h, C.byref(op), None) == B.PSGD_EINVAL
    assert lib.psgd_linear_forward_workspace(None, C.byref(op), C.byref(n)) == B.PSGD_EINVAL
    assert lib.psgd_linear_forward_workspace(plan._h, None, C.byref(n)) == B.PSGD_EINVAL
    for fields, status in ((dict(weight=1), B.PSGD_EINVAL), (dict(tokens=-1), B.PSGD_EINVAL), (dict(param_dtype=B.PSGD_BF16), B.PSGD_EUNSUPPORTED)):
        op = B.psgd_linear(**{**dict(weight=0, bias=-1, tokens=3), **fields})
        assert lib.psgd_linear_forward_workspace(plan._h, C.byref(op), C.byref(n)) == status


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,n,k", [(1, 96, 4096), (20, 512, 2048), (40, 128, 4096), (300, 1031, 520), (700, 4100, 4095), (1500, 2601, 2600), (4099, 2048, 2048),
                                   (130, 64, 9000), (66, 6855, 5171)])
def test_forward_stays_within_it(T, n, k, dtype, params):
    """Guard bytes behind the scratch, and the result of a call with the scratch of both passes."""
    from test_gpu_operators import CODE, DT, Layer, Rows, _need_gpu
    dev = _need_gpu()
    L = Layer(n, k, dtype, params, dev)
    x = Rows(T, k, DT[dtype], dev, 3, 1, L.normal(T, k))   # rows that begin anywhere: x is laid out too where that pays
    size = L.plan.linear_forward_workspace(1, T, CODE[params])
    ws = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device=dev)
    y, z = torch.empty(T, n, dtype=DT[dtype], device=dev), torch.empty(T, n, dtype=DT[dtype], device=dev)
    L.plan.linear_forward(1, T, L.param, x.ptr(), y, ws, x_stride=x.ld, activation="silu", **L.op())
    L.plan.linear_forward(1, T, L.param, x.ptr(), z, L.workspace(T), x_stride=x.ld, activation="silu", **L.op())
    assert bool((ws[size:] == 0xFF).all()) and torch.equal(y, z) and bool(torch.isfinite(y).all())
