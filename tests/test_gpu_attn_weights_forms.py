"""Attention weights in every form of the kernel: tiles of 32, 64 and 96 tokens, for steps and for chunks, with eight waves a
workgroup and with four (more workgroups than compute units), a tile's query rows in one workgroup and shared by several.

Which form a call takes follows from its heads, batch and bounds alone (weights_shape in api_evict.cpp); the forms named
here are those of 256 compute units, and a kernel trace of this file has each of them.
"""

import pytest

torch = pytest.importorskip("torch")

from tests.context_util import near, weights_of  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from tests.test_gpu_evict import DEV, Case  # noqa: E402

pytestmark = pytest.mark.gpu

# form: KV heads, group, lengths, new tokens. The first sequence has the bounds; lengths lie around the tiles' ends.
STEPS = {
    "64 tokens": (2, 4, [9000, 6400, 65], [1, 1, 1]),
    "64 tokens, heads in turns": (6, 1, [8200, 63, 1], [1, 1, 1]),
    "96 tokens": (2, 4, [22000, 96, 7019], [1, 1, 1]),
    "96 tokens, one head": (1, 16, [33000, 97], [1, 1]),
    "96 tokens, heads in turns": (5, 2, [22000, 95, 1], [1, 1, 1]),
    "96 tokens, two groups of rows": (3, 2, [22000, 193, 16], [16, 7, 16]),
}
CHUNKS = {
    "32 tokens, 4 waves": (1, 2, [9000], [17]),
    "64 tokens, 8 waves": (3, 2, [9000], [64]),
    "64 tokens, 8 waves, shared": (3, 2, [3000], [300]),
    "64 tokens, 4 waves": (1, 2, [9000, 127], [17, 17]),
    "64 tokens, 4 waves, shared": (3, 2, [9000], [200]),
    "96 tokens, 8 waves": (3, 1, [9000, 97], [64, 33]),
    "96 tokens, 8 waves, heads in turns": (20, 1, [9000, 191], [40, 39]),
    "96 tokens, 8 waves, shared": (2, 16, [3000], [64]),
    "96 tokens, 4 waves": (1, 2, [33000], [17]),
    "96 tokens, 4 waves, heads in turns": (6, 1, [33000, 96], [40, 23]),
    "96 tokens, 4 waves, shared": (3, 4, [33000, 95, 500], [40, 40, 1]),
}


def run(dtype, page, d, hkv, group, lens, new, step):
    c = Case(lens, new, dtype, hkv, group, d, page, seed=len(lens) + d + page)
    prior = torch.rand((len(lens), c.bound), generator=c.gen) * 3
    for b, n in enumerate(lens):
        prior[b, n - new[b]:] = float("nan")  # the new tokens' is not read
    old = torch.full((len(lens), c.bound + 3), float("nan"))
    old[:, :c.bound] = prior
    out = torch.full((len(lens), c.bound + 3), -7.0, device=DEV)
    c.call(step=step, out=out, prior=old.to(DEV), decay=0.75)
    want = weights_of(c.ctx, c.q, c.lse, new, c.scale, prior, 0.75)
    for b, (w, off) in enumerate(want):
        got = out[b, :lens[b]].double().cpu()
        assert near(got, w, off), (b, int(torch.isnan(got).sum()), float(((got - w).abs() / off).max()))
        assert bool((out[b, lens[b]:] == -7.0).all()), b


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", STEPS)
def test_step_forms(form, d, page, dtype):
    say("weights form", form, d, page, dtype)
    hkv, group, lens, new = STEPS[form]
    run(dtype, page, d, hkv, group, lens, new, step=max(new) == 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", CHUNKS)
def test_chunk_forms(form, d, page, dtype):
    say("weights form", form, d, page, dtype)
    run(dtype, page, d, *CHUNKS[form], step=False)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv,group,lens,new", [(1, 2, [9000], [17]), (5, 2, [9000, 33], [20, 3]), (2, 4, [9000, 31], [1, 1])])
def test_float32_forms(hkv, group, lens, new, d, page):
    """Tiles of 32 tokens alone; four waves, and heads in turns."""
    say("weights form, float32", hkv, group, lens, new, d, page)
    run("f32", page, d, hkv, group, lens, new, step=max(new) == 1)
