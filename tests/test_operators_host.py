"""The operators around the step, without a GPU: the oracle's generator against published vectors, its gradients against
differences, and what the entry points refuse (all of it checked before any GPU call)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import operators_oracle as OO
from paper_1905_13727_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("counter,key,want", [
    # the known-answer vectors that the generator's authors give for Philox4x32-10
    ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
])
def test_generator_of_the_oracle(counter, key, want):
    assert OO.philox4x32(counter, key) == want
    got = OO.philox_words([counter[0]], [counter[1]], key[0] | key[1] << 32, counter[2] | counter[3] << 32)
    assert got.reshape(-1).tolist() == want


def test_share_of_dropped_elements():
    # 2^18 draws: the standard deviation of the share is below 0.001
    for p in (0.1, 0.5, 0.9):
        gone = OO.drop_factor(256, 1024, p, seed=5, offset=7) == 0
        assert abs(gone.mean() - p) < 5e-3
        assert np.abs(gone.reshape(256, -1, 8).mean((0, 1)) - p).max() < 1.5e-2   # every place of a group of eight alike
    keep = OO.mask_keep(512, 512, 3, 0.01, 0, 11, 13)
    assert abs(keep.mean() - 0.01) < 1e-3
    assert (OO.mask_keep(64, 64, 3, -1.0, 256, 1, 2).sum() - 256) < 80


@pytest.mark.parametrize("kind", B.ACTIVATIONS)
def test_gradients_of_the_oracle_against_differences(kind):
    rng = np.random.default_rng(3)
    T, n, k = 5, 7, 6
    x, W, b, dy = (rng.standard_normal(s) for s in ((T, k), (n, k), (n,), (T, n)))
    factor = OO.drop_factor(T, n, 0.3, 9, 2)

    def loss(x, W, b):
        return float((OO.linear_forward(x, W, b, kind, factor)[0] * dy).sum())

    z = OO.linear_forward(x, W, b, kind, factor)[1]
    got = OO.linear_backward(x, W, z, dy, kind, factor)[:3]
    h = 1e-6   # central differences: error h^2 f''' / 6 and 1e-16 / h
    for i, (a, g) in enumerate(zip((x, W, b), got)):
        for at in np.ndindex(a.shape):
            lo, hi = [x, W, b], [x, W, b]
            lo[i], hi[i] = a.copy(), a.copy()
            lo[i][at] -= h
            hi[i][at] += h
            assert abs((loss(*hi) - loss(*lo)) / (2 * h) - g[at]) < 1e-7


def test_struct_has_the_headers_layout(tmp_path):
    src = tmp_path / "size.c"
    names = [f for f, _ in B.psgd_linear._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "psgd.h"\nint main(void) { printf("%zu", sizeof(psgd_linear));'
                   + "".join(' printf(" %%zu", offsetof(psgd_linear, %s));' % n for n in names) + " return 0; }\n")
    exe = str(tmp_path / "size")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(v) for v in subprocess.run([exe], stdout=subprocess.PIPE, check=True, text=True).stdout.split()]
    assert got == [C.sizeof(B.psgd_linear)] + [getattr(B.psgd_linear, n).offset for n in names]
    hdr = open(os.path.join(ROOT, "include", "psgd.h")).read()
    for i, name in enumerate(B.ACTIVATIONS):
        assert "PSGD_ACT_%s = %d" % (name.upper(), i) in hdr


# ---- refusals: none of these makes a GPU call ---------------------------------------------------------------------------

P, P2 = 1 << 20, 1 << 24   # addresses that are never read: the calls below are refused first


def _forward(plan, op=None, param=P, x=P, residual=None, pre=None, y=P2, workspace=P, **fields):
    a = dict(weight=0, bias=1, activation=0, param_dtype=B.PSGD_F32, tokens=4)
    a.update(fields)
    s = B.psgd_linear(**a)
    return plan._lib.psgd_linear_forward(plan._h, C.byref(s), param, x, residual, pre, y, workspace, None)


def _backward(plan, param=P, x=P, pre=P, dy=P, dx=P2, grad=P2, worker=0, accumulate=0, workspace=P, **fields):
    a = dict(weight=0, bias=1, activation=2, param_dtype=B.PSGD_F32, tokens=4)
    a.update(fields)
    s = B.psgd_linear(**a)
    return plan._lib.psgd_linear_backward(plan._h, C.byref(s), param, x, pre, dy, dx, grad, worker, accumulate, workspace, None)


SHAPES = [(6, 8), (6,), (5,), (8, 8)]

TENSORS = [
    (dict(weight=-1), B.PSGD_EINVAL), (dict(weight=4), B.PSGD_EINVAL), (dict(weight=1), B.PSGD_EINVAL),
    (dict(bias=4), B.PSGD_EINVAL), (dict(bias=2), B.PSGD_EINVAL), (dict(bias=3), B.PSGD_EINVAL),
    (dict(activation=5), B.PSGD_EINVAL), (dict(activation=-1), B.PSGD_EINVAL),
    (dict(param_dtype=2), B.PSGD_EINVAL), (dict(param_dtype=B.PSGD_BF16), B.PSGD_EUNSUPPORTED),
    (dict(tokens=-1), B.PSGD_EINVAL), (dict(tokens=(1 << 30) + 1), B.PSGD_EUNSUPPORTED),
    (dict(x_stride=7), B.PSGD_EINVAL), (dict(residual_stride=5), B.PSGD_EINVAL), (dict(pre_stride=5), B.PSGD_EINVAL),
    (dict(y_stride=-6), B.PSGD_EINVAL), (dict(dy_stride=5), B.PSGD_EINVAL), (dict(dx_stride=7), B.PSGD_EINVAL),
    (dict(x_stride=(1 << 20) + 1), B.PSGD_EUNSUPPORTED), (dict(dx_stride=1 << 40), B.PSGD_EUNSUPPORTED),
]
DROPS = [
    (dict(drop=-0.1, rng=P), B.PSGD_EINVAL), (dict(drop=1.5, rng=P), B.PSGD_EINVAL), (dict(drop=float("nan"), rng=P), B.PSGD_EINVAL),
    (dict(drop=0.5), B.PSGD_EINVAL), (dict(drop=0.5, rng=P + 4), B.PSGD_EINVAL),
]


@pytest.mark.parametrize("fields,status", TENSORS + DROPS + [
    (dict(param=None), B.PSGD_EINVAL), (dict(x=None), B.PSGD_EINVAL), (dict(y=None), B.PSGD_EINVAL),
    (dict(x=P + 2), B.PSGD_EINVAL), (dict(y=P2 + 1), B.PSGD_EINVAL), (dict(residual=P + 2), B.PSGD_EINVAL),
    (dict(pre=P + 3), B.PSGD_EINVAL), (dict(param=P + 2), B.PSGD_EINVAL), (dict(workspace=None), B.PSGD_EINVAL),
    (dict(workspace=P + 128), B.PSGD_EINVAL),
])
def test_linear_forward_refuses(fields, status):
    plan = B.Plan(SHAPES, 2, 2)
    assert _forward(plan, **fields) == status


@pytest.mark.parametrize("fields,status", TENSORS + DROPS + [
    (dict(dx=None, grad=None), B.PSGD_EINVAL), (dict(worker=-1), B.PSGD_EINVAL), (dict(worker=2), B.PSGD_EINVAL),
    (dict(dy=None), B.PSGD_EINVAL), (dict(pre=None), B.PSGD_EINVAL), (dict(param=None), B.PSGD_EINVAL), (dict(x=None), B.PSGD_EINVAL),
    (dict(dx=P2 + 2), B.PSGD_EINVAL), (dict(grad=P2 + 2), B.PSGD_EINVAL), (dict(dy=P + 2), B.PSGD_EINVAL),
    (dict(workspace=None), B.PSGD_EINVAL), (dict(workspace=P + 16), B.PSGD_EINVAL),
])
def test_linear_backward_refuses(fields, status):
    plan = B.Plan(SHAPES, 2, 2)
    assert _backward(plan, **fields) == status


def test_linear_refuses_null_handles_and_wide_layers():
    plan = B.Plan(SHAPES, 2)
    lib, op, n = plan._lib, B.psgd_linear(weight=0, bias=-1, tokens=3), C.c_int64()
    assert lib.psgd_linear_forward(None, C.byref(op), P, P, None, None, P, P, None) == B.PSGD_EINVAL
    assert lib.psgd_linear_forward(plan._h, None, P, P, None, None, P, P, None) == B.PSGD_EINVAL
    assert lib.psgd_linear_backward(None, C.byref(op), P, P, None, P, P, P, 0, 0, P, None) == B.PSGD_EINVAL
    assert lib.psgd_linear_backward(plan._h, None, P, P, None, P, P, P, 0, 0, P, None) == B.PSGD_EINVAL
    assert lib.psgd_linear_workspace(plan._h, C.byref(op), None) == B.PSGD_EINVAL
    assert lib.psgd_linear_workspace(None, C.byref(op), C.byref(n)) == B.PSGD_EINVAL
    assert lib.psgd_linear_workspace(plan._h, None, C.byref(n)) == B.PSGD_EINVAL
    wide = B.Plan([(2, (1 << 20) + 4), ((1 << 20) + 1, 2)], 2)
    for t in (0, 1):
        with pytest.raises(B.PsgdError) as e:
            wide.linear_workspace(t, 3)
        assert e.value.status == B.PSGD_EUNSUPPORTED
    # no tokens: nothing to compute, no buffer of a token is needed and no GPU call is made
    assert _forward(plan, x=None, y=None, workspace=None, tokens=0) == B.PSGD_OK
    assert _backward(plan, x=None, dy=None, pre=None, workspace=None, tokens=0, accumulate=1) == B.PSGD_OK
    assert plan.linear_workspace(0, 0) == 0


def test_linear_workspace_grows_with_the_tokens_only():
    plan = B.Plan([(512, 256), (512,)], 2, 1, B.PSGD_BF16, B.PSGD_BF16)
    sizes = [plan.linear_workspace(0, t) for t in (1, 100, 4096, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[-1] >= (1 << 20) * 512 * 2
    assert plan.linear_workspace(0, 100) == plan.linear_workspace(0, 100, drop=0.5, offset=3)


@pytest.mark.parametrize("fields,status", [
    (dict(dtype=2), B.PSGD_EINVAL), (dict(rows=-1), B.PSGD_EINVAL), (dict(cols=-1), B.PSGD_EINVAL),
    (dict(p=-1e-9), B.PSGD_EINVAL), (dict(p=1.01), B.PSGD_EINVAL), (dict(p=float("nan")), B.PSGD_EINVAL),
    (dict(rng=None), B.PSGD_EINVAL), (dict(rng=P + 4), B.PSGD_EINVAL), (dict(x=None), B.PSGD_EINVAL), (dict(y=None), B.PSGD_EINVAL),
    (dict(x=P + 2), B.PSGD_EINVAL), (dict(y=P + 2), B.PSGD_EINVAL), (dict(residual=P + 1), B.PSGD_EINVAL),
    (dict(x_stride=7), B.PSGD_EINVAL), (dict(y_stride=-8), B.PSGD_EINVAL), (dict(residual_stride=3), B.PSGD_EINVAL),
    (dict(rows=1 << 31), B.PSGD_EUNSUPPORTED), (dict(cols=1 << 31), B.PSGD_EUNSUPPORTED), (dict(x_stride=1 << 31), B.PSGD_EUNSUPPORTED),
    (dict(rows=1 << 30, cols=1 << 13), B.PSGD_EUNSUPPORTED),
])
def test_dropout_refuses(fields, status):
    a = dict(dtype=B.PSGD_F32, rows=4, cols=8, x=P, x_stride=0, residual=None, residual_stride=0, y=P2, y_stride=0, p=0.5, rng=P)
    a.update(fields)
    lib = B.load_library()
    got = lib.psgd_dropout_forward(a["dtype"], a["rows"], a["cols"], a["x"], a["x_stride"], a["residual"], a["residual_stride"],
                                   a["y"], a["y_stride"], a["p"], a["rng"], 0, None)
    assert got == status
    if "residual" not in fields and "residual_stride" not in fields:
        assert lib.psgd_dropout_backward(a["dtype"], a["rows"], a["cols"], a["x"], a["x_stride"], a["y"], a["y_stride"], a["p"],
                                         a["rng"], 0, None) == status


def test_dropout_of_nothing_needs_no_gpu():
    lib = B.load_library()
    for rows, cols in ((0, 8), (8, 0), (0, 0)):
        assert lib.psgd_dropout_forward(B.PSGD_BF16, rows, cols, None, 0, None, 0, None, 0, 0.5, P, 0, None) == B.PSGD_OK
        assert lib.psgd_dropout_backward(B.PSGD_F32, rows, cols, None, 0, None, 0, 0.5, P, 0, None) == B.PSGD_OK


@pytest.mark.parametrize("fields,status", [
    (dict(grad=None), B.PSGD_EINVAL), (dict(err=None), B.PSGD_EINVAL), (dict(rng=None), B.PSGD_EINVAL), (dict(out=None), B.PSGD_EINVAL),
    (dict(keep=1.0001), B.PSGD_EINVAL), (dict(keep=float("nan")), B.PSGD_EINVAL), (dict(rng=P + 4), B.PSGD_EINVAL),
    (dict(grad=P + 4), B.PSGD_EINVAL), (dict(err=P + 8), B.PSGD_EINVAL), (dict(out=P + 4), B.PSGD_EINVAL),
])
def test_random_mask_refuses(fields, status):
    plan = B.Plan(SHAPES, 2, 2)
    a = dict(grad=P, err=P, keep=0.5, rng=P, out=P2)
    a.update(fields)
    assert plan._lib.psgd_random_mask_step(plan._h, a["grad"], a["err"], a["keep"], a["rng"], 0, a["out"], None) == status
    assert plan._lib.psgd_random_mask_step(None, P, P, 0.5, P, 0, P2, None) == B.PSGD_EINVAL


def test_random_mask_refuses_matrices_beyond_its_counter():
    plan = B.Plan([(1 << 14, (1 << 20) + 4)], 2)
    assert plan._lib.psgd_random_mask_step(plan._h, P, P, 0.5, P, 0, P2, None) == B.PSGD_EUNSUPPORTED
    assert "2^34" in plan.last_error()
