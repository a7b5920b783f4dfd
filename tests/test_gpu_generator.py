"""What of the generator's words decides a draw: the seed and the sum of the device's offset and the call's."""
import pytest

torch = pytest.importorskip("torch")

from paper_1905_13727_amd import binding as B
from test_gpu_operators import _need_gpu, _stream

pytestmark = pytest.mark.gpu


def test_only_the_sum_of_the_offsets_counts():
    dev = _need_gpu()
    plan = B.Plan([(40, 64)], 2)
    grad, err = torch.randn(plan.sizes.grad_stride, device=dev), torch.zeros(plan.sizes.err_stride, device=dev)

    def draw(at, offset, seed=7):
        rng = torch.tensor([seed, at], dtype=torch.int64, device=dev)
        y, out = torch.empty(50, 43, device=dev), torch.zeros(plan.sizes.out_elems, device=dev)
        B.dropout_forward(B.PSGD_F32, 50, 43, torch.ones_like(y), y, 0.5, rng, offset=offset, stream=_stream())
        plan.random_mask_step(grad, err.clone(), 0.5, rng, out, offset=offset, stream=_stream())
        return torch.cat([(y == 0).reshape(-1), out == 0])

    # three calls a step: moving on by three draws anew for all of them, by one repeats two of the step before
    first = [draw(10, i) for i in range(3)]
    assert all(torch.equal(draw(11, i), first[i + 1]) for i in range(2))
    assert not any(torch.equal(draw(13, i), other) for i in range(3) for other in first)
    assert torch.equal(draw(1 << 40, 5), draw((1 << 40) + 5, 0)) and not torch.equal(draw(10, 0, seed=8), first[0])
