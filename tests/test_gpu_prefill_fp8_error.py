"""FP8 prefill: the error that the header promises for a weight, 2^-23 of itself (two f16 values, each to nearest).

A weight of the second f16 value: with 2^e <= p < 2^(e + 1) the first one is a multiple of 2^(e - 10), the rest is at most
2^(e - 11), the second a multiple of 2^(e - 22) or finer, so the sum is off by 2^(e - 23) at most.

Outputs (NORM). Of each weight: its score's sum of 128 products 3e-7, the exponent's argument 5e-7, the split 2^-23 =
1.2e-7, independent from key to key: 6e-7 together (the root of the squares' sum), four times that is the gate.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_prefill_fp8 import DEV, RAGGED_L, RAGGED_M, Case  # noqa: E402

pytestmark = pytest.mark.gpu

NORM = 2.4e-6


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what,kw", [
    ("ragged", dict(lens=RAGGED_L, new=RAGGED_M, page=16, bound=1010)),
    ("uncached", dict(lens=[3000], new=[3000], hq=4, hkv=1)),
    ("few rows", dict(lens=[3000, 700, 64, 5], new=[16, 3, 16, 1], page=16)),
    ("split", dict(lens=[9000, 12000], new=[40, 17], hq=32, hkv=8, page=64)),
    ("few rows, split", dict(lens=[9000], new=[9], hq=32, hkv=8)),
])
def test_error_of_the_outputs(what, kw, d):
    c = Case(**kw, d=d, seed=21)
    out, _ = c.run()
    ref, _, _ = c.want()
    err = float((out.double() - ref).norm() / ref.norm())
    say("fp8 prefill", what, d, f"error {err:.2e} of the norm")
    assert err <= NORM


@pytest.mark.parametrize("few", [False, True])
def test_a_weight_and_its_two_parts(few):
    """Two keys, both values 1: the output is (512 + parts of p) / (512 + p), p from 256 to 512, and the same p in both.

    What the parts lack is at most 2^-23 of p, half of the sum: 2^-24. To that come half a step of the sum of weights, of
    the division and of the product with it, 2^-24 each, and a whole step, 2^-23, in the matrix cores' sum.
    """
    m = 16 if few else 400
    c = Case([m + 2] * 8, [m] * 8, hq=8, hkv=2, d=64, seed=22, k_scale=1.0, v_scale=1.0)
    one, minus_one, zero, far = 0x38, 0xB8, 0, 0xFE  # 1, -1, 0, -448
    live = torch.cat([c.rows(b) for b in range(8)])
    c.v[live] = one
    c.k[live] = zero
    c.k[live, :, 0] = far
    for b in range(8):
        c.k[c.rows(b)[0], :, 0] = zero
        c.k[c.rows(b)[1], :, 0] = minus_one  # score -q / 8: a weight from 1/2 to 1
    g = torch.Generator().manual_seed(3)
    c.q.zero_()
    c.q[:, :, 0] = (torch.rand(c.q.shape[:2], generator=g) * 5.5).to(torch.bfloat16)  # ln 2 * 8 = 5.545
    seen = c.q[:, :, 0].float() > 0.7  # from there a far key's weight is exp(-448 * 0.7 / 8) at most, 1e-17
    out, _ = c.run()
    off = np.abs(out.double().numpy()[seen.numpy()] - 1.0)
    say("two parts of a weight", few, f"largest {off.max() * 2 ** 24:.2f} * 2^-24 of {int(seen.sum())} rows")
    assert off.size > 5000 and off.max() <= 6 * 2.0 ** -24
