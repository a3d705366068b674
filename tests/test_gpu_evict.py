"""Attention weights and the choice of the tokens that stay (comem_kv_evict.h) against their 64-bit forms."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.context_util import (KS, VS, Context, chosen, drawn, logsumexp_rows, query_dtype, wide,  # noqa: E402
                                weights_of)
from tests.gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def make_op(dtype, hq, hkv, d, batch, bound):
    from paper_2605_30842_amd.binding import DecodeAttention

    scales = dict(k_scale=KS, v_scale=VS) if dtype == "fp8" else {}
    return DecodeAttention(hq, hkv, d, dtype, 1.0 / math.sqrt(d), batch, bound, **scales)


class Case:
    """A drawn cache, queries of the last new[b] tokens, their lse, and the call."""

    def __init__(self, lens, new, dtype, hkv, group, d, page, seed=1, layout="dense", spread=1.0, bound=None):
        g = torch.Generator().manual_seed(seed)
        self.bound = bound or max(max(lens), 1)
        width = -(-self.bound // page) if page else None
        self.ctx = Context(lens, dtype, hkv, d, page, g, layout=layout, width=width, spread=spread)
        self.new, self.page, self.hq = list(new), page, hkv * group
        self.scale = float(np.float32(1.0 / math.sqrt(d)))
        self.q = torch.randn((sum(new), self.hq, d), generator=g).to(query_dtype(dtype))
        self.lse = logsumexp_rows(self.ctx, self.q, new, self.scale).float()
        self.op = make_op(dtype, self.hq, hkv, d, len(lens), self.bound)
        self.gen = g

    def call(self, step=False, q=None, lse=None, **kw):
        x = self.ctx.to(DEV)
        q, lse = (self.q if q is None else q).to(DEV), (self.lse if lse is None else lse).to(DEV)
        if not step:
            kw.update(q_start=torch.tensor([sum(self.new[:b]) for b in range(len(self.new))], dtype=torch.int64, device=DEV),
                      q_lens=torch.tensor(self.new, dtype=torch.int32, device=DEV), max_q_len=max(max(self.new), 1))
        if self.page:
            return self.op.attn_weights_paged(q, lse, x["k"], x["block_table"], x["ctx_lens"], self.bound, **kw)
        return self.op.attn_weights(q, lse, x["k"], x["seq_start"], x["ctx_lens"], self.bound, **kw)

    def check(self, out, prior=None, decay=1.0, lse=None, what=""):
        want = weights_of(self.ctx, self.q, self.lse if lse is None else lse, self.new, self.scale, prior, decay)
        for b, (w, off) in enumerate(want):
            if self.new[b] == 0:
                continue
            got = out[b, :self.ctx.lens[b]].double().cpu()
            over = (got - w).abs() > off
            assert not over.any(), (what, b, int(over.sum()), float(((got - w).abs() / off).max()))


SHAPES = [  # hkv, group, d
    (8, 4, 128), (2, 8, 64), (1, 1, 128), (3, 16, 64), (5, 2, 128), (1, 16, 128), (20, 4, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [0, 1, 16, 64])
@pytest.mark.parametrize("hkv,group,d", SHAPES)
def test_step(dtype, page, hkv, group, d):
    """One new token a sequence, without row lists."""
    say("weights step", dtype, page, hkv, group, d)
    lens = [1, 2, 15, 16, 17, 64, 65, 300, 129]
    c = Case(lens, [1] * len(lens), dtype, hkv, group, d, page, seed=hkv + page)
    out = torch.full((len(lens), c.bound + 5), -7.0, device=DEV)
    assert c.call(step=True, out=out) is out
    c.check(out)
    for b, n in enumerate(lens):
        assert bool((out[b, n:] == -7.0).all()), b
        # Each query row's weights add up to 1: n 2^-24 of float32 sums and the weights' own 2^-18.
        assert abs(float(out[b, :n].double().sum()) - c.hq) < c.hq * 2.0 ** -15


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("hkv,group,d", SHAPES)
def test_chunk(dtype, page, hkv, group, d):
    """Chunks of the last tokens, causal among themselves; whole contexts, none, and one."""
    say("weights chunk", dtype, page, hkv, group, d)
    lens, new = [1, 40, 90, 200, 33, 130], [1, 40, 17, 70, 0, 1]
    c = Case(lens, new, dtype, hkv, group, d, page, seed=hkv + page + 9)
    prior = torch.rand((len(lens), c.bound), generator=c.gen) * 9
    for b, n in enumerate(lens):
        prior[b, n - new[b]:] = float("nan")  # new tokens were paid nothing before
    out = torch.full((len(lens), c.bound), -7.0, device=DEV)
    c.call(out=out, prior=prior.to(DEV), decay=0.75)
    c.check(out, prior, 0.75)
    assert bool((out[4] == -7.0).all())
    plain = torch.full((len(lens), c.bound), -7.0, device=DEV)
    c.call(out=plain, prior=torch.full_like(plain, float("nan")), decay=0.0)  # not read
    c.check(plain)
    same = prior.to(DEV)
    c.call(out=same, prior=same, decay=0.75)
    for b, n in enumerate(lens):
        if new[b]:
            assert torch.equal(same[b, :n], out[b, :n])


@pytest.mark.parametrize("layout", ["fused", "heads"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_strides(layout, page, dtype):
    c = Case([100, 37], [20, 37], dtype, 4, 4, 128, page, layout=layout)
    c.check(c.call())


@pytest.mark.parametrize("spread", [0.0, 8.0])
def test_flat_and_peaked(spread):
    """All weights alike, and nearly all of them on a few tokens (the rest underflow to 0 or nearly)."""
    c = Case([500, 77], [3, 50], "bf16", 2, 4, 128, 16, spread=spread)
    c.check(c.call())


def test_many_tiles_and_rows():
    """The forms of 16, 32 and 64 tokens a workgroup, and many rows of a head."""
    for lens, new, page in ([5000], [1], 16), ([17000, 3], [1, 1], 0), ([40000], [1], 64), ([2500], [600], 0):
        say("weights tiles", lens, new)
        c = Case(lens, new, "bf16", 2, 4, 64, page)
        c.check(c.call())


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("lens,new", [([900], [900]), ([300, 1, 257], [300, 1, 100]), ([60], [3])])
def test_shared_rows(dtype, lens, new):
    """Many rows over few tokens: shared by several workgroups with a workspace, and not without a large enough one."""
    c = Case(lens, new, dtype, 2, 4, 64, 16)
    most = max(new)
    nbytes = c.op.attn_weights_workspace_bytes(len(lens), most, c.bound)
    assert (nbytes > 0) == (most > 8)
    prior = torch.rand((len(lens), c.bound), generator=c.gen)
    for ws in (None, torch.empty(1, dtype=torch.uint8, device=DEV), torch.full((nbytes // 4,), float("nan"), device=DEV)):
        out = torch.full((len(lens), c.bound + 3), -7.0, device=DEV)
        old = torch.full_like(out, float("nan"))
        old[:, :c.bound] = prior.to(DEV)
        c.call(out=out, prior=old, decay=0.5, workspace=ws if ws is None or ws.numel() else None)
        c.check(out, prior, 0.5, what=str(ws is None))
        for b, n in enumerate(lens):
            assert bool((out[b, n:] == -7.0).all())


def test_shared_rows_captured():
    """Scratch of a captured call belongs to its graph."""
    c = Case([500, 400], [200, 400], "bf16", 2, 4, 64, 0)
    x, q, lse = c.ctx.to(DEV), c.q.to(DEV), c.lse.to(DEV)
    rows = dict(q_start=torch.tensor([0, 200], dtype=torch.int64, device=DEV),
                q_lens=torch.tensor([200, 400], dtype=torch.int32, device=DEV), max_q_len=400)

    def call(**kw):
        return c.op.attn_weights(q, lse, x["k"], x["seq_start"], x["ctx_lens"], 500, **rows, **kw)

    want = call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        torch.full((1 << 20,), float("nan"), device=DEV)  # the allocator's free memory
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    stream = torch.cuda.Stream()
    other = call(stream=stream)
    stream.synchronize()
    assert torch.equal(other, want)


def test_rows_that_saw_nothing():
    """lse = -inf adds nothing, even with NaN queries; other rows as ever."""
    c = Case([70, 40], [10, 2], "bf16", 2, 4, 64, 16)
    q, lse = c.q.clone(), c.lse.clone()
    q[3], lse[3] = float("nan"), -math.inf
    lse[11, 2:5] = -math.inf
    out = c.call(q=q, lse=lse)
    c.q = torch.where(torch.isnan(q), 0.0, q.float()).to(q.dtype)
    c.check(out, lse=lse)


def test_nan_reaches_what_it_meets():
    c = Case([70], [4], "bf16", 2, 2, 64, 0)
    q = c.q.clone()
    q[2, 1] = float("nan")  # new token 2 sees the tokens 0 .. 68
    out = c.call(q=q)[0].cpu()
    assert bool(torch.isnan(out[:69]).all()) and bool(torch.isfinite(out[69:]).all())
    x = c.ctx.k[c.ctx.at[0][5], 1].clone()
    c.ctx.k[c.ctx.at[0][5], 1, 7] = float("nan")
    out = c.call()[0].cpu()
    assert bool(torch.isnan(out[5])) and int(torch.isnan(out).sum()) == 1
    c.ctx.k[c.ctx.at[0][5], 1] = x


def test_sequences_outside_their_bounds_are_left():
    c = Case([50, 60, 70, 80], [5, 5, 5, 5], "bf16", 2, 4, 64, 16, bound=80)
    x = c.ctx.to(DEV)
    out = torch.full((4, 80), -7.0, device=DEV)
    starts = torch.tensor([0, 5, 10, 15], dtype=torch.int64, device=DEV)
    for lens, counts in (([50, 81, -1, 80], [5, 5, 5, 0]), ([50, 4, 70, 2 ** 31 - 1], [5, 5, 6, 5])):
        c.op.attn_weights_paged(c.q.to(DEV), c.lse.to(DEV), x["k"], x["block_table"],
                                torch.tensor(lens, dtype=torch.int32, device=DEV), 80, q_start=starts,
                                q_lens=torch.tensor(counts, dtype=torch.int32, device=DEV), max_q_len=5, out=out)
    assert bool((out[1:] == -7.0).all())
    w, off = weights_of(c.ctx, c.q, c.lse, c.new, c.scale)[0]
    assert bool(((out[0, :50].cpu().double() - w).abs() <= off).all())


def test_bad_table_entries_read_page_0():
    c = Case([48], [2], "bf16", 2, 4, 64, 16)
    x = c.ctx.to(DEV)
    table = x["block_table"].clone()
    rows = dict(q_start=torch.zeros(1, dtype=torch.int64, device=DEV),
                q_lens=torch.tensor([2], dtype=torch.int32, device=DEV), max_q_len=2)
    got = {}
    x["k"][0] = x["k"][int(table[0, 1])] * 0.5  # finite keys there
    for bad in (0, -1, x["k"].shape[0], 2 ** 31 - 1, -2 ** 31):
        table[0, 1] = bad
        got[bad] = c.op.attn_weights_paged(c.q.to(DEV), c.lse.to(DEV), x["k"], table, x["ctx_lens"], 48, **rows)
    for bad, out in got.items():
        assert torch.equal(out, got[0]), bad


def test_same_bits_contiguous_paged_and_again():
    a = Case([700, 333], [9, 1], "bf16", 4, 4, 128, 0, seed=3)
    b = Case([700, 333], [9, 1], "bf16", 4, 4, 128, 16, seed=3)
    for s in range(2):  # the pages get the packed cache's keys
        at, to = a.ctx.at[s], b.ctx.at[s]
        b.ctx.k[to // 16, to % 16] = a.ctx.k[at]
    first = a.call()
    assert torch.equal(first, a.call()) and torch.equal(first, b.call(q=a.q, lse=a.lse))


def test_captured_and_on_another_stream():
    c = Case([260, 90], [1, 1], "fp8", 2, 8, 128, 64)
    x, q, lse = c.ctx.to(DEV), c.q.to(DEV), c.lse.to(DEV)
    sums = torch.zeros((2, 260), device=DEV)

    def step(**kw):
        return c.op.attn_weights_paged(q, lse, x["k"], x["block_table"], x["ctx_lens"], 260, **kw)

    want = step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = step(stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(prior=sums, out=sums, decay=0.5)
    eager = torch.zeros_like(sums)
    for i in range(4):
        graph.replay()
        step(prior=eager, out=eager, decay=0.5)
        torch.cuda.synchronize()
        assert torch.equal(sums, eager), i


# ------------------------------------------------------------ the tokens that stay


def keep(weights, lens, budget, first=0, last=0, rows=None, budgets=None, bound=None, **kw):
    i32 = dict(dtype=torch.int32, device=DEV)
    bound = bound or max(max(lens), 1)
    op = make_op("f32", 1, 1, 64, 1, bound)
    got = op.keep_tokens(weights.to(DEV), torch.tensor(lens, **i32), bound, budget, first, last,
                         rows=None if rows is None else torch.tensor(rows, **i32),
                         budgets=None if budgets is None else torch.tensor(budgets, **i32), **kw)
    torch.cuda.synchronize()
    return [t.cpu() for t in got]


def check_keep(weights, lens, budget, first=0, last=0, rows=None, budgets=None, bound=None):
    n = len(lens) if rows is None else len(rows)
    out = torch.full((n, budget), -5, dtype=torch.int32, device=DEV)
    vals = torch.full((n, budget), -5.0, device=DEV)
    got, start, count, kept = keep(weights, lens, budget, first, last, rows, budgets, bound, keep=out, kept=vals)
    assert start.tolist() == [i * budget for i in range(n)]
    for i, r in enumerate(range(len(lens)) if rows is None else rows):
        if not 0 <= r < len(lens) or not 0 <= lens[r] <= (bound or max(max(lens), 1)):
            assert int(count[i]) == -1 and bool((got[i] == -5).all()) and bool((kept[i] == -5.0).all())
            continue
        own = budget if budgets is None else min(max(budgets[i], first + last), budget)
        want = chosen(weights[r, :lens[r]].numpy(), min(own, lens[r]), first, last)
        assert int(count[i]) == len(want), (i, int(count[i]), len(want))
        assert got[i, :len(want)].tolist() == want, i
        assert np.array_equal(kept[i, :len(want)].numpy().view(np.int32), weights[r, want].numpy().view(np.int32))
        assert bool((got[i, len(want):] == -5).all()) and bool((kept[i, len(want):] == -5.0).all())


SIZES = [1, 2, 63, 64, 65, 255, 256, 257, 2047, 2048, 2049, 5000]


@pytest.mark.parametrize("part", [0.02, 0.4, 0.97])
def test_keep_sizes(part):
    g = torch.Generator().manual_seed(4)
    for bound in (max(SIZES), 2048, 257):
        lens = [n for n in SIZES if n <= bound] + [0]
        w = (torch.randn((len(lens), bound), generator=g) * 3).exp()
        budget = max(3, int(part * bound))
        check_keep(w, lens, budget, first=1, last=2)
        check_keep(w, lens, budget, bound=bound)


@pytest.mark.parametrize("n", [1280, 1281, 2047, 2048, 2049])
def test_keep_many_rows(n):
    """More rows than compute units, of lengths around those where the kernel changes, and few of them."""
    g = torch.Generator().manual_seed(n)
    w = (torch.randn((300, n), generator=g) * 3).exp()
    w[7] = w[7].round()
    lens = torch.randint(0, n + 1, (300,), generator=g).tolist()
    lens[:9] = [n, n - 1, 0, 1, 255, 256, 257, n, n]
    check_keep(w, lens, n // 3, first=1, last=2, bound=n)
    check_keep(w[:9].contiguous(), lens[:9], n // 3, first=1, last=2, bound=n)


@pytest.mark.parametrize("n", [32767, 32769, 65536, 65537, 100001, 150000])
def test_keep_long(n):
    say("keep", n)
    g = torch.Generator().manual_seed(n)
    w = (torch.randn((2, n), generator=g) * 3).exp()
    w[1] = w[1].round()  # many equal ones
    check_keep(w, [n, n - 7], n // 5, first=100, last=1000)
    check_keep(w, [n, n // 2], n - 1)


@pytest.mark.parametrize("n", [49152, 49153, 57344, 57345, 131073, 524288, 524289])
def test_keep_with_and_without_a_workspace(n):
    """Long rows in chunks give what one workgroup a row gives: rows that end before, in and at the end of a chunk, one
    that stays whole, one whose bound it passes, one that is forced throughout."""
    say("keep", n)
    g = torch.Generator().manual_seed(n)
    w = (torch.randn((6, n), generator=g) * 3).exp()
    w[2] = w[2].round()
    w[3] = 1.0
    lens = [n, 8193, n - 1, n - 8192, 100, n]
    full = 2 * (n // 5)
    for budget, first, last, budgets in ((n // 3, 5, 70, None), (full, n // 5, n // 5, None),
                                         (n // 2, 0, 9000, [0, 8200, 9000, 9001, 101, n // 2])):
        got = keep(w, lens, budget, first, last, budgets=budgets)
        one = keep(w, lens, budget, first, last, budgets=budgets, workspace=torch.empty(0, device=DEV))
        for i, count in enumerate(got[2].tolist()):
            assert count == int(one[2][i]) and torch.equal(got[0][i, :count], one[0][i, :count]), i
            assert torch.equal(got[3][i, :count], one[3][i, :count]), i
    check_keep(w, lens, n // 3, 5, 70)
    check_keep(w, lens, n // 4, n // 4, 0, rows=[5, 5, 1, -1, 6, 0])


def test_keep_long_captured_and_on_another_stream():
    """A graph's workspace is its own: two of them, and eager calls between."""
    n = 100000
    g = torch.Generator().manual_seed(5)
    w = [torch.randn((2, n), generator=g).to(DEV) for _ in range(2)]
    lens = torch.tensor([n, n - 9000], dtype=torch.int32, device=DEV)
    op = make_op("f32", 1, 1, 64, 1, n)
    want = [op.keep_tokens(x, lens, n, 4000, 3, 3) for x in w]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in w]
    got = []
    for graph, x in zip(graphs, w):
        with torch.cuda.graph(graph):
            got.append(op.keep_tokens(x, lens, n, 4000, 3, 3))
    for i in range(3):
        for graph, out in zip(graphs, got):
            for t in out:
                t.fill_(-7)
            torch.full((1 << 20,), -1, dtype=torch.int32, device=DEV)  # the allocator's free memory
            graph.replay()
        op.keep_tokens(w[0], lens, n, 100)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), i
    stream = torch.cuda.Stream()
    other = op.keep_tokens(w[1], lens, n, 4000, 3, 3, stream=stream)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(other, want[1]))


@pytest.mark.parametrize("n", [50, 3000, 40000, 60001])
def test_keep_equal_and_special_values(n):
    rows = [torch.zeros(n), torch.ones(n), torch.full((n,), math.inf), torch.full((n,), -math.inf), torch.full((n,), math.nan)]
    rows[0][::3] = -0.0
    g = torch.Generator().manual_seed(n)
    pick = torch.tensor([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-42, -1e-42, 3e38])
    rows.append(pick[torch.randint(len(pick), (n,), generator=g)])
    nan = torch.randn(n, generator=g)
    nan.view(torch.int32)[::7] = -1  # a negative NaN
    nan.view(torch.int32)[3::7] = 0x7f800001
    rows.append(nan)
    w = torch.stack(rows)
    for budget, first, last in (n // 2, 0, 0), (n // 10, 2, 3), (n - 1, 0, 1), (1, 0, 0), (7, 3, 4):
        check_keep(w, [n] * len(rows), budget, first, last)


def test_keep_rows_and_budgets():
    g = torch.Generator().manual_seed(8)
    w = torch.rand((6, 400), generator=g)
    lens = [400, 10, 0, 401, 77, -3]
    check_keep(w, lens, 60, 5, 6, rows=[4, 0, 3, 6, -1, 0], bound=400)
    check_keep(w, lens, 60, 5, 6, rows=[0, 1, 2, 4, 0, 5], budgets=[0, 8, 60, 11, 1000, 20], bound=400)
    check_keep(w, lens, 60, budgets=[0, -5, 3, 3, 1, 1], bound=400)
    check_keep(w, [400, 10, 0, 3, 77, 1], 0)


def test_keep_from_a_view():
    """Rows that lie apart and start anywhere."""
    g = torch.Generator().manual_seed(9)
    big = torch.rand((5, 333), generator=g)
    i32 = dict(dtype=torch.int32, device=DEV)
    op = make_op("f32", 1, 1, 64, 1, 200)
    view = big.to(DEV)[1:, 7:211]
    got, _, lens, kept = op.keep_tokens(view, torch.tensor([200, 3, 150, 60], **i32), 200, 50)
    for r, n in enumerate([200, 3, 150, 60]):
        want = chosen(big[1 + r, 7:7 + n].numpy(), min(50, n), 0, 0)
        assert got[r, :int(lens[r])].tolist() == want
        assert torch.equal(kept[r, :len(want)].cpu(), big[1 + r, 7:][want])


def test_keep_empty_call_and_capture():
    i32 = dict(dtype=torch.int32, device=DEV)
    op = make_op("f32", 1, 1, 64, 1, 300)
    w, lens = torch.rand((2, 300), device=DEV), torch.tensor([300, 120], **i32)
    got = op.keep_tokens(w, lens, 300, 10, rows=torch.zeros(0, **i32))
    assert got[0].shape == (0, 10) and got[2].shape == (0,)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        keep_g, _, lens_g, kept_g = op.keep_tokens(w, lens, 300, 10, 1, 1)
    for i in range(3):
        w.copy_(torch.rand(w.shape))
        graph.replay()
        torch.cuda.synchronize()
        a, _, n, v = op.keep_tokens(w, lens, 300, 10, 1, 1)
        assert torch.equal(a, keep_g) and torch.equal(n, lens_g) and torch.equal(v, kept_g), i


def test_two_graphs_and_eager_calls_of_shared_rows():
    """Graphs of one plan have a workspace each; a caller's own serves calls that follow each other."""
    c = Case([500, 400], [200, 400], "bf16", 2, 4, 64, 0)
    x, q = c.ctx.to(DEV), c.q.to(DEV)
    lse = [c.lse.to(DEV), (c.lse + 1).to(DEV)]
    rows = dict(q_start=torch.tensor([0, 200], dtype=torch.int64, device=DEV),
                q_lens=torch.tensor([200, 400], dtype=torch.int32, device=DEV), max_q_len=400)
    nbytes = c.op.attn_weights_workspace_bytes(2, 400, 500)
    assert nbytes > 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)

    def call(i, **kw):
        return c.op.attn_weights(q, lse[i], x["k"], x["seq_start"], x["ctx_lens"], 500, **rows, **kw)

    want = [call(0), call(1)]
    torch.cuda.synchronize()
    for given in ({}, {"workspace": ws}):
        graphs, got = [torch.cuda.CUDAGraph() for _ in lse], []
        for i, graph in enumerate(graphs):
            with torch.cuda.graph(graph):
                got.append(call(i, **given))
        for _ in range(3):
            ws.fill_(255)
            for graph in graphs:
                graph.replay()
            eager = call(0, **given)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(eager, want[0])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[call(i, stream=s) for i, s in enumerate(streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        assert torch.equal(pair[0], want[0]) and torch.equal(pair[1], want[1])
