"""What a launch cannot take is refused before anything is launched: its lanes are counted in 32 bits, 2^24 - 1 workgroups of 256.  None of
these calls reaches the GPU; the addresses are never read."""
import ctypes as C

import pytest

from paper_1905_13727_amd import binding as B

P, P2 = 1 << 20, 1 << 24


def _backward(plan, tokens, bias=-1, activation=0, drop=0.0):
    s = B.psgd_linear(weight=0, bias=bias, activation=activation, param_dtype=B.PSGD_F32, tokens=tokens, drop=drop, rng=P)
    return plan._lib.psgd_linear_backward(plan._h, C.byref(s), P, P, P, P, P2, P2, 0, 0, P, None)


def _forward(plan, tokens):
    s = B.psgd_linear(weight=0, bias=-1, activation=0, param_dtype=B.PSGD_F32, tokens=tokens)
    return plan._lib.psgd_linear_forward(plan._h, C.byref(s), P, P, None, None, P2, P, None)


@pytest.mark.parametrize("dtype", [B.PSGD_F32, B.PSGD_BF16])
@pytest.mark.parametrize("fields", [dict(bias=1), dict(activation=2), dict(drop=0.5), dict(bias=1, activation=4, drop=0.5)])
@pytest.mark.parametrize("tokens", [(1 << 30) - 63, 1 << 30])
def test_backward_refuses_more_blocks_of_tokens_than_a_launch_takes(tokens, fields, dtype):
    plan = B.Plan([(4, 2), (4,)], 2, 1, dtype, dtype)
    assert _backward(plan, tokens, **fields) == B.PSGD_EUNSUPPORTED


def test_linear_refuses_more_elements_than_its_tiles_cover():
    for shapes, tokens in (([((1 << 20), 2)], (1 << 17) + 1), ([(2, 1 << 20)], (1 << 17) + 1)):
        plan = B.Plan(shapes, 1)
        assert _forward(plan, tokens) == B.PSGD_EUNSUPPORTED and _backward(plan, tokens) == B.PSGD_EUNSUPPORTED
        with pytest.raises(B.PsgdError) as e:
            plan.linear_workspace(0, tokens)
        assert e.value.status == B.PSGD_EUNSUPPORTED
        assert plan.linear_workspace(0, tokens - 1) >= 0


@pytest.mark.parametrize("rows,cols", [((1 << 31) - 1, 65), (1 << 24, 8193), (1 << 17, 1 << 20), (1 << 25, 4104)])
def test_dropout_refuses_more_elements_than_a_launch_takes(rows, cols):
    lib = B.load_library()
    for dtype in (B.PSGD_F32, B.PSGD_BF16):
        assert rows * cols > 1 << 36
        assert lib.psgd_dropout_forward(dtype, rows, cols, P, 0, None, 0, P2, 0, 0.5, P, 0, None) == B.PSGD_EUNSUPPORTED
        assert lib.psgd_dropout_backward(dtype, rows, cols, P, 0, P2, 0, 0.5, P, 0, None) == B.PSGD_EUNSUPPORTED


def test_random_mask_refuses_more_slices_than_a_launch_takes():
    for shapes in ([(1 << 14, 1 << 20)], [(1 << 13, 1 << 20), (1 << 13, (1 << 20) - 1), (1 << 20,)]):
        plan = B.Plan(shapes, 2)
        for keep in (0.5, -1.0):
            assert plan._lib.psgd_random_mask_step(plan._h, P, P, keep, P, 0, P2, None) == B.PSGD_EUNSUPPORTED
            assert "2^34" in plan.last_error()
