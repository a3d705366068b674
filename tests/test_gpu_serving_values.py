"""The serving run of test_gpu_serving_run with the stored values compared with the new tokens' values themselves.

There, what the cache holds becomes the record that later steps are checked against; a value stored in another head or
row, or with another scale, would be in the record too. Values are copied, or become the nearest code of v / v_scale with
v_scale a power of two, so they are equal, not near. Attention is checked at every step.
"""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.ops_util import pages_of  # noqa: E402
from tests.test_gpu_serving_run import VS, Loop  # noqa: E402

pytestmark = pytest.mark.gpu


def stored_value(new_v, dtype):
    """What a cache of this type holds for new values, in 64 bits."""
    if dtype != "fp8":
        return new_v.double().cpu()
    return (new_v.double().cpu() / VS).clamp(-448, 448).float().to(torch.float8_e4m3fn).double() * VS


class Values(Loop):
    """The loop's buffers hold a token's queries, keys and values side by side: the values follow the keys."""

    seen = 0

    def take_new(self, r, m, new_k):
        super().take_new(r, m, new_k)
        heads, d = new_k.shape[1:]
        new_v = torch.as_strided(new_k, new_k.shape, new_k.stride(), new_k.storage_offset() + heads * d)
        got = torch.stack([v for _, v in self.kept[r][-m:]])
        assert torch.equal(got, stored_value(new_v, self.dtype)), f"V of {r}"
        self.seen += m

    def steps(self, live, count):
        for _ in range(count):  # a graph each, its first replay checked
            super().steps(live, 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [1, 16])
def test_stored_values(dtype, page):
    say("serving values", dtype, page)
    s = Values(dtype, page, rows=4, num_pages=pages_of(700, page) + 8)
    s.prompts([70, 0, 33, 0])
    s.fork([0, 2], [1, 3])
    s.steps([0, 1, 3], 7)
    n = len(s.kept[1])
    s.compact([1], [list(range(20)) + list(range(n - 21, n))])
    s.prompts([0, 18, 5, 0])
    s.steps([0, 1, 2, 3], 4)
    assert s.seen == 103 + 21 + 23 + 16
    s.release([0, 1, 2, 3])
    assert int(s.counts.abs().sum()) == 0
