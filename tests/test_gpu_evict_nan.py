"""The tests of attention weights once more, with a check that a NaN in a result fails.

test_gpu_evict's Case.check looks for elements that are too far off, and a NaN, whose comparisons are all false, is not
found to be one; its inputs hold NaN wherever a call may not look (rows of no sequence, the new tokens' prior, a workspace,
queries that saw nothing). Here an element has to be found near enough.
"""

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_evict as evict  # noqa: E402
from tests.context_util import near, weights_of  # noqa: E402
from tests.test_gpu_evict import (test_chunk, test_flat_and_peaked, test_many_tiles_and_rows,  # noqa: E402, F401
                                  test_rows_that_saw_nothing, test_shared_rows, test_step, test_strides)

pytestmark = pytest.mark.gpu


class Checked(evict.Case):
    def check(self, out, prior=None, decay=1.0, lse=None, what=""):
        want = weights_of(self.ctx, self.q, self.lse if lse is None else lse, self.new, self.scale, prior, decay)
        for b, (w, off) in enumerate(want):
            if self.new[b] > 0:
                got = out[b, :self.ctx.lens[b]].double().cpu()
                assert near(got, w, off), (what, b, int(torch.isnan(got).sum()), float(((got - w).abs() / off).max()))


@pytest.fixture(autouse=True)
def checked(monkeypatch):
    monkeypatch.setattr(evict, "Case", Checked)
