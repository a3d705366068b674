"""The checks that the GPU tests of attention weights use, on the CPU: what they let pass and what they do not."""

import pytest
import torch

from tests import test_gpu_evict as evict
from tests.context_util import near, weights_of
from tests.test_gpu_evict_nan import Checked


def test_near():
    want, off = torch.tensor([1.0, 0.0, 2.0]), torch.tensor([0.1, 0.0, 0.5])
    assert near(torch.tensor([1.05, 0.0, 1.6]), want, off) and near(want[:0], want[:0], off[:0])
    for bad in ([1.2, 0.0, 2.0], [float("nan"), 0.0, 2.0], [1.0, float("inf"), 2.0], [1.0, 0.0, float("-inf")]):
        assert not near(torch.tensor(bad), want, off)
    for bad in (float("nan"), float("inf")):
        assert not near(torch.tensor([bad] * 3), want, off)


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("fp8", 16), ("f32", 4)])
def test_a_wrong_weight_fails(monkeypatch, dtype, page):
    """The 64-bit form itself passes, also beside NaN where no call looks; a NaN or a wrong element does not."""
    monkeypatch.setattr(evict, "make_op", lambda *a: None)
    c = Checked([1, 40, 90, 33], [1, 40, 17, 0], dtype, 2, 4, 64, page)
    prior = torch.rand((4, 90), generator=c.gen)
    for b, n in enumerate(c.ctx.lens):
        prior[b, n - c.new[b]:] = float("nan")
    lse = c.lse.clone()
    lse[3, 1] = -float("inf")
    out = torch.full((4, 95), float("nan"), dtype=torch.float64)  # elements past a context are not the check's
    for b, (w, _) in enumerate(weights_of(c.ctx, c.q, lse, c.new, c.scale, prior, 0.5)):
        if c.new[b]:
            out[b, :c.ctx.lens[b]] = w
    c.check(out, prior, 0.5, lse=lse)
    for b, t in ((0, 0), (1, 39), (2, 5), (2, 80)):
        for bad in (float("nan"), float("inf"), float(out[b, t]) * 1.01 + 1e-3):
            wrong = out.clone()
            wrong[b, t] = bad
            with pytest.raises(AssertionError):
                c.check(wrong, prior, 0.5, lse=lse)
