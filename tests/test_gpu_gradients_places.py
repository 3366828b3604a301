"""Where tensors lie and the norm of their numbers.

The order of the sums depends on the tensors' sizes, types and addresses modulo 32 alone: tensors that begin alike give equal bits, wherever they lie; others
stay within the bound of test_gpu_gradients.py, 2 u of the norm, u = 2^-24.
"""
import pytest
import torch

import paper_1505_04956_b200 as pkg

from .test_gpu_gradients import BF, F16, F32, U, _norm64, _tensors

pytestmark = pytest.mark.gpu


def _placed(ts, shift, room):
    """The same tensors, beginning `shift` numbers (and 32 `room` bytes) into buffers of their own."""
    out = []
    for t in ts:
        first = shift + room * 32 // t.element_size()
        buffer = torch.full((first + t.numel() + 3,), float("nan"), device="cuda", dtype=t.dtype)
        buffer[first:first + t.numel()] = t
        out.append(buffer[first:first + t.numel()])
    return out


@pytest.mark.parametrize("sizes, types", [([1_000_003, 77, 4096], [F32, BF, F16]), ([300_001] * 3, [BF]), ([5, 1, 700, 31], [F16, F32]), ([999] * 700, [F32, BF])])
def test_the_same_numbers_elsewhere(sizes, types):
    ts = _tensors(9, sizes, types)
    want = _norm64(ts)
    for shift in (0, 1, 2, 3, 7, 8, 15):
        norms = [pkg.asgd_grad_norm(_placed(ts, shift, room)) for room in (0, 1, 5)]
        assert abs(float(norms[0]) - want) <= 2 * U * want
        assert torch.equal(norms[0], norms[1]) and torch.equal(norms[0], norms[2])
        limit = 0.5 * want
        placed, again = _placed(ts, shift, 0), _placed(ts, shift, 3)
        assert torch.equal(pkg.asgd_clip_grads(placed, limit), norms[0]) and torch.equal(pkg.asgd_clip_grads(again, limit), norms[0])
        assert all(torch.equal(a, b) for a, b in zip(placed, again))
