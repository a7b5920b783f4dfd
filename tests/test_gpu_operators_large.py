"""Large calls of the linear layer on the GPU, against fp64 on the device: the most tokens, and the launches that only large layers take.

Tolerances as in test_gpu_operators.py (u = half a step of the output type, v = 2^-24)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import operators_oracle as OO
from test_gpu_operators import DT, OFFSET, SEED, U, V, Layer, _need_gpu, _rng, near_on_device

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
