"""Infinities and NaN in attention over blocks and in attention weights: as the decode call has them. A NaN in q or K makes
the heads that see it NaN, output and lse; a score of -inf weighs nothing; an infinity in V leaves the outputs it reaches
infinite or NaN, and the others as they were."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.context_util import Context, near, query_dtype, weights_of  # noqa: E402
from tests.gpu_util import check, say  # noqa: E402
from tests.test_gpu_block_attn import attended, ints, make_op  # noqa: E402
from tests.test_gpu_evict import DEV, Case  # noqa: E402

pytestmark = pytest.mark.gpu

FORMS = [  # dtype, page, variant, chunk, tokens of the tables (the first sequence's is the call's bound)
    ("bf16", 64, "auto", 0, [3000]), ("bf16", 16, "auto", 0, [900, 0, 40, 2000]), ("bf16", 4, "auto", 0, [900, 31]),
    ("bf16", 16, "mfma_grid", 64, [700, 31]), ("bf16", 16, "auto", 32, [6000, 31, 5000]), ("bf16", 16, "valu", 64, [700, 31]),
    ("f32", 16, "auto", 64, [700, 31]), ("fp8", 64, "auto", 0, [3000]), ("fp8", 4, "auto", 0, [900, 31])]


def draw(dtype, page, variant, chunk, tokens):
    g = torch.Generator().manual_seed(page + len(tokens))
    c = Context(tokens, dtype, 2, 64, page, g, both=True)
    op = make_op(dtype, 8, 2, 64, len(tokens), max(tokens), variant=variant, chunk_tokens=chunk)
    q = torch.randn((len(tokens), 8, 64), generator=g).to(query_dtype(dtype))
    table = c.table[:, None].expand(-1, 2, -1).contiguous()
    return c, op, q, table


def attend(c, op, q, table):
    x, lse = c.to(DEV), torch.zeros(q.shape[:2], device=DEV)
    out, _ = op.block_forward(q.to(DEV), x["k"], x["v"], table.to(DEV), x["ctx_lens"], max(c.lens), lse=lse)
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("dtype,page,variant,chunk,tokens", FORMS)
def test_a_nan_reaches_the_heads_that_see_it(dtype, page, variant, chunk, tokens):
    say("blocks, NaN", dtype, page, variant, chunk, tokens)
    c, op, q, table = draw(dtype, page, variant, chunk, tokens)
    plain, plain_lse = attend(c, op, q, table)
    for t in {0, 17, tokens[0] // 2, tokens[0] - 1}:
        at = int(c.at[0][t])
        key = c.k[at // page, at % page, 1]
        was = key[5].clone()
        key[5] = 0x7f if dtype == "fp8" else float("nan")
        out, lse = attend(c, op, q, table)
        key[5] = was
        assert bool(torch.isnan(out[0, 4:]).all()) and bool(torch.isnan(lse[0, 4:]).all()), t
        assert torch.equal(out[0, :4], plain[0, :4]) and torch.equal(lse[0, :4], plain_lse[0, :4]), t
        assert torch.equal(out[1:], plain[1:]) and torch.equal(lse[1:], plain_lse[1:]), t
    q[-1, 2, 9] = float("nan")
    out, lse = attend(c, op, q, table)
    assert bool(torch.isnan(out[-1, 2]).all()) and bool(torch.isnan(lse[-1, 2]))
    rest = [h for h in range(8) if h != 2]
    assert torch.equal(out[-1, rest], plain[-1, rest]) and torch.equal(out[:-1], plain[:-1])


@pytest.mark.parametrize("dtype,page,variant,chunk,tokens", [f for f in FORMS if f[0] != "fp8"])  # E4M3 has no infinity
def test_infinite_scores_and_values(dtype, page, variant, chunk, tokens):
    say("blocks, inf", dtype, page, variant, chunk, tokens)
    c, op, q, table = draw(dtype, page, variant, chunk, tokens)
    q[:, :, 7] = q[:, :, 7].float().abs().clamp(min=0.5).to(q.dtype)
    gone = torch.rand(tokens[0], generator=torch.Generator().manual_seed(1)) < 0.4
    gone[:300] = True  # whole tiles
    gone[-1] = False
    for t in torch.nonzero(gone)[:, 0].tolist():
        at = int(c.at[0][t])
        c.k[at // page, at % page, 0, 7] = -math.inf
    out, lse = attend(c, op, q, table)
    scale = float(np.float32(1.0 / math.sqrt(64)))
    want = [attended(c, b, q[b], [c.table[b, :-(-n // page)]] * 2, n, scale) for b, n in enumerate(tokens)]
    check(out.numpy(), lse.numpy(), np.stack([w[0] for w in want]), np.stack([w[1] for w in want]), dtype)
    at = int(c.at[0][tokens[0] - 1])
    c.v[at // page, at % page, 1, 3] = math.inf
    got, got_lse = attend(c, op, q, table)
    assert not bool(torch.isfinite(got[0, 4:, 3]).any())
    keep = [i for i in range(64) if i != 3]
    assert torch.equal(got_lse, lse) and torch.equal(got[0, :, keep], out[0, :, keep])
    assert torch.equal(got[0, :4], out[0, :4]) and torch.equal(got[1:], out[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("new", [[1, 1], [40, 7]])
def test_weights_of_infinite_scores(dtype, page, new):
    """A key that scores -inf is paid nothing by the queries that do so; one whose score is NaN makes its own weight NaN."""
    c = Case([500, 70], new, dtype, 2, 4, 64, page)
    c.q[:, :, 7] = c.q[:, :, 7].float().abs().clamp(min=0.5).to(c.q.dtype)
    for t in (0, 17, 300):
        at = int(c.ctx.at[0][t])
        (c.ctx.k[at // page, at % page] if page else c.ctx.k[at])[0, 7] = -math.inf
    out = c.call()
    lse = c.lse.clone()
    lse[:, :4] = -math.inf  # leaves those heads out
    others = weights_of(c.ctx, c.q, lse, new, c.scale)
    for b, (w, off) in enumerate(weights_of(c.ctx, c.q, c.lse, new, c.scale)):
        if b == 0:
            for t in (0, 17, 300):
                assert float(w[t]) == float(others[0][0][t])
                off[t] = others[0][1][t]  # a weight of exactly 0 is off by nothing
        assert near(out[b, :c.ctx.lens[b]].double().cpu(), w, off), b
    at = int(c.ctx.at[0][20])
    (c.ctx.k[at // page, at % page] if page else c.ctx.k[at])[1, 9] = float("nan")
    nan = c.call()
    assert bool(torch.isnan(nan[0, 20]))
    nan[0, 20] = out[0, 20]
    assert torch.equal(nan, out)
