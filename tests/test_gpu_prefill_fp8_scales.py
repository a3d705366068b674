"""FP8 prefill with V scales near the ends of float32.

A power of two as the scale changes no bit of an output but the exponent, as long as no output is subnormal: the codes
here are 1 and more, so outputs are at least the scale. The results with scale 1 are checked against 64 bits in
test_gpu_prefill_fp8.
"""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_prefill_fp8 import DEV, Case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,lens,new", [("full blocks", [300, 1000], [300, 70]), ("few rows", [100, 700, 33], [3, 16, 1]),
                                           ("split", [9000], [40]), ("few rows, split", [9000, 5000], [9, 16])])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_any_size(form, lens, new, d):
    say("V scales", form, d)
    got = {}
    for power in (0, -118, -100, -60, 60, 110):
        c = Case(lens, new, d=d, page=16, seed=2, k_scale=1.0, v_scale=1.0)
        c.v.copy_(0x38 + c.v % 64)  # 1 .. 240
        c.k_scale, c.v_scale = 2.0 ** -6, 2.0 ** power
        c.k.copy_((torch.randn(c.k.shape, generator=torch.Generator().manual_seed(5)) * 64).to(torch.float8_e4m3fn)
                  .view(torch.uint8))
        op = c.op()
        size = op.prefill_workspace_bytes(len(lens), max(new), max(lens)) if "split" in form else 0
        assert (size > 0) == ("split" in form)
        out, lse = c.run(op=op, workspace=torch.empty(size, dtype=torch.uint8, device=DEV))
        assert bool((out >= 2.0 ** power).all())
        got[power] = out.double() * 2.0 ** -power, lse
        assert torch.equal(got[power][1], got[0][1])
        assert torch.equal(got[power][0], got[0][0]), f"2^{power}"
