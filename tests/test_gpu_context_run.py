"""The eviction and block operators together, as an agent's loop uses them: a prompt's attention counted, decode steps that
add theirs, the contexts cut to the most attended tokens, the sums carried along, then steps that read chosen blocks only.

The caches are those of the serving run, with its record of what every sequence should hold. A step's queries and keys are
the stored ones, so attention is held to the gates of that run. Sums of weights: lse is held to 1e-4 of its size there (at
most 8 here), which moves a weight by 8e-4 of itself; the weight's own arithmetic by less than 1e-4.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.context_util import chosen  # noqa: E402
from tests.gpu_util import say  # noqa: E402
from tests.ops_util import pages_of  # noqa: E402
from tests.test_gpu_serving_run import D, DEV, HKV, HQ, MAX, Loop  # noqa: E402

pytestmark = pytest.mark.gpu

G = HQ // HKV
SCALE = float(np.float32(1.0 / np.sqrt(D)))


class ContextLoop(Loop):
    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.sums = torch.full((self.rows, MAX), float("nan"), device=DEV)  # needs no initialisation
        self.want = [torch.zeros(0, dtype=torch.float64) for _ in range(self.rows)]
        self.ends = torch.zeros((self.k.shape[0], HKV, 2, D), dtype=self.k.dtype, device=DEV)
        self.one = torch.ones(self.rows, dtype=torch.int32, device=DEV)

    def paid(self, q, r, limit):
        """Weights of queries [hq, D] of row r over its first `limit` tokens, summed over heads, padded to its length."""
        k = torch.stack([a for a, _ in self.kept[r]])
        w = torch.zeros(len(self.kept[r]), dtype=torch.float64)
        for h in range(HQ):
            w[:limit] += torch.softmax(SCALE * (k[:limit, h // G] @ q[h]), 0)
        return w

    def check_sums(self):
        for r in range(self.rows):
            n = len(self.kept[r])
            got = self.sums[r, :n].double().cpu()
            assert bool(((got - self.want[r]).abs() <= 1e-3 * self.want[r] + 1e-30).all()), r

    def observe(self, lens, decay):
        """New tokens of some rows; the attention they pay joins the sums."""
        first = [len(k) for k in self.kept]
        i64 = dict(dtype=torch.int64, device=DEV)
        q_start = torch.tensor([sum(lens[:r]) for r in range(self.rows)], **i64)
        q_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        seen = {}
        rope, prefill = self.op.rope_append_paged, self.op.prefill_paged

        def keep_q(*a, **kw):
            seen["q"] = rope(*a, **kw)
            return seen["q"]

        self.op.rope_append_paged = keep_q
        self.prompts(lens)
        self.op.rope_append_paged = rope
        q = seen["q"]
        lse = torch.empty(q.shape[:2], device=DEV)
        if self.dtype == "f32":  # prefill takes bf16 and FP8 caches: the rows as decode steps
            for r in range(self.rows):
                for i in range(lens[r]):
                    at = int(q_start[r]) + i
                    ctx = torch.zeros_like(self.ctx)
                    ctx[r] = first[r] + i + 1
                    part = torch.empty((self.rows, HQ), device=DEV)
                    self.op.forward_paged(q[at:at + 1].expand(self.rows, -1, -1).contiguous(), self.k, self.v, self.table, ctx,
                                          MAX, lse=part)
                    lse[at] = part[r]
        else:
            prefill(q, q_start, q_lens, max(lens), self.k, self.v, self.table, self.ctx, MAX, lse=lse)
        self.op.attn_weights_paged(q, lse, self.k, self.table, self.ctx, MAX, q_start=q_start, q_lens=q_lens,
                                   max_q_len=max(lens), prior=self.sums, out=self.sums, decay=decay)
        for r in range(self.rows):
            if lens[r]:
                w = torch.zeros(len(self.kept[r]), dtype=torch.float64)
                w[:first[r]] = decay * self.want[r]
                for i in range(lens[r]):
                    w += self.paid(q[int(q_start[r]) + i].double().cpu(), r, first[r] + i + 1)
                self.want[r] = w
        self.check_sums()

    def captured(self, after):
        """A graph of one step of all rows: pages, rotation and store, then after(q)."""
        x = torch.zeros((self.rows, HQ + 2 * HKV, D), dtype=self.q_dtype, device=DEV)
        at, q = torch.zeros_like(self.ctx), torch.zeros((self.rows, HQ, D), dtype=self.q_dtype, device=DEV)
        missing = torch.ones((), dtype=torch.int32, device=DEV)

        def step():
            self.pages.reserve(self.one, missing=missing)
            self.op.rope_append_paged(x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], self.k, self.v, self.table, self.ctx,
                                      MAX, self.cos_sin, *self.weights, positions=at, q_out=q)
            return after(q)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = step()

        def run():
            x.copy_(torch.randn(x.shape, generator=self.gen).to(self.q_dtype))
            at.copy_(torch.tensor(self.where, dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            assert int(missing) == 0
            for r in range(self.rows):
                self.take_new(r, 1, x[r:r + 1, HQ:HQ + HKV])
            return q.double().cpu()

        return run, result

    def counted_steps(self, count, decay):
        lse = torch.zeros((self.rows, HQ), device=DEV)

        def after(q):
            out, _ = self.op.forward_paged(q, self.k, self.v, self.table, self.ctx, MAX, lse=lse)
            self.op.attn_weights_paged(q, lse, self.k, self.table, self.ctx, MAX, prior=self.sums, out=self.sums, decay=decay)
            return out

        run, out = self.captured(after)
        for i in range(count):
            q = run()
            for r in range(self.rows):
                n = len(self.kept[r])
                self.want[r] = torch.cat([decay * self.want[r], torch.zeros(1, dtype=torch.float64)]) + self.paid(q[r], r, n)
                self.near(out[r], self.attended(q[r], r, n), f"step {i} of {r}")
            self.check_sums()
        self.check_record()

    def cut(self, rows, budget, first, last):
        """The rows cut to their most attended tokens; their sums follow."""
        which = torch.tensor(rows, dtype=torch.int32, device=DEV)
        keep, start, lens, kept = self.op.keep_tokens(self.sums, self.ctx, MAX, budget, first, last, rows=which)
        lists = [chosen(self.sums[r, :len(self.kept[r])].cpu().numpy(), min(budget, len(self.kept[r])), first, last) for r in rows]
        for i, want in enumerate(lists):
            assert keep[i, :int(lens[i])].tolist() == want
        assert int(self.pages.compact(which, keep.view(-1), start, lens)) == 0
        self.sums[which.long(), :budget] = kept
        for r, keep in zip(rows, lists):
            self.kept[r] = [self.kept[r][t] for t in keep]
            self.want[r] = self.want[r][keep]
        self.check_record()
        self.check_sums()

    def sparse_steps(self, count, budget):
        self.op.block_bounds(self.k, self.table, self.ctx, MAX, self.ends, q_lens=self.ctx, max_q_len=MAX)
        seen = {}

        def after(q):
            self.op.block_bounds(self.k, self.table, self.ctx, MAX, self.ends)
            seen["scores"] = self.op.block_scores(q, self.ends, self.page, self.table, self.ctx, MAX)
            seen["table"], seen["lens"] = self.op.block_select(seen["scores"], self.page, self.table, self.ctx, MAX, budget, 1, 2)
            return self.op.block_forward(q, self.k, self.v, seen["table"], seen["lens"], min(MAX, budget * self.page))[0]

        run, out = self.captured(after)
        for i in range(count):
            q = run()
            for r in range(self.rows):
                n = len(self.kept[r])
                blocks = pages_of(n, self.page)
                k, v = (torch.stack([row[side] for row in self.kept[r]]) for side in (0, 1))
                want = torch.zeros(HQ, D, dtype=torch.float64)
                for h in range(HKV):
                    scores = seen["scores"][r, h, :blocks].cpu()
                    pick = chosen(scores.numpy(), min(blocks, budget), 1, 2)
                    held = seen["table"][r, h, :len(pick)].tolist()
                    assert held == [int(self.table[r, j]) for j in pick], (i, r, h)
                    t = torch.tensor([t for j in pick for t in range(j * self.page, min(n, (j + 1) * self.page))])
                    assert int(seen["lens"][r]) == len(t)
                    for j in range(h * G, (h + 1) * G):
                        s = SCALE * (k[:, h] @ q[r, j])
                        # No key scores above its block's bound (2 D float32 roundings of sums of at most |q| |k| D).
                        assert all(float(s[b * self.page:(b + 1) * self.page].max()) <= float(scores[b]) + 1e-3
                                   for b in range(blocks))
                        want[j] = torch.softmax(s[t], 0) @ v[t, h]
                self.near(out[r], want, f"sparse step {i} of {r}")
        self.check_record()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_a_context_run(dtype, page):
    say("context run", dtype, page)
    s = ContextLoop(dtype, page, rows=3, num_pages=pages_of(900, page) + 12, norm=page != 64)
    s.observe([90, 41, 7], 1.0)
    s.counted_steps(6, 0.9)
    s.cut([0, 1], 40, 4, 10)
    s.observe([0, 20, 33], 0.5)     # observations on the cut contexts
    s.counted_steps(4, 1.0)
    s.cut([2, 0, 1], 30, 0, 5)
    s.sparse_steps(5, 3)
    s.release([0, 1, 2])
    assert int(s.counts.abs().sum()) == 0


@pytest.mark.parametrize("dtype,page", [("bf16", 4), ("fp8", 16)])
def test_pools_past_32_bits(dtype, page):
    """Every call over pages whose bytes, and whose bounds' bytes, lie past 2^32 gives what it gives over a small pool."""
    from tests.test_gpu_block_attn import make_op

    say("pools past 32 bits", dtype, page)
    hkv, d, lens = 8, 128, [203, 64, 1]
    g = torch.Generator().manual_seed(12)
    width = -(-max(lens) // page)
    few = 3 * width
    kind = torch.float8_e4m3fn if dtype == "fp8" else torch.bfloat16
    size = 1 if dtype == "fp8" else 2
    small = torch.randn((few, page, hkv, d), generator=g).to(kind).to(DEV)
    base = 2 ** 32 // (2 * hkv * d * size) + 100  # bounds of a page: 2 hkv d elements
    assert base * 2 * hkv * d * size > 2 ** 32 and base * page * hkv * d * size > 2 ** 32
    big = torch.empty((base + few, page, hkv, d), dtype=torch.uint8 if dtype == "fp8" else kind, device=DEV).view(kind)
    big[base:] = small
    ends = {0: torch.empty((few, hkv, 2, d), dtype=kind, device=DEV)}
    ends[base] = torch.empty((base + few, hkv, 2, d), dtype=torch.uint8 if dtype == "fp8" else kind, device=DEV).view(kind)
    table = torch.randperm(few, generator=g).view(3, width).to(torch.int32).to(DEV)
    ctx = torch.tensor(lens, dtype=torch.int32, device=DEV)
    op = make_op(dtype, 32, hkv, d, 3, 203)
    q = torch.randn((3, 32, d), generator=g).to(torch.bfloat16).to(DEV)
    got = {}
    for shift, pool in ((0, small), (base, big)):
        at, e = table + shift, ends[shift]
        op.block_bounds(pool, at, ctx, 203, e, q_lens=ctx, max_q_len=203)
        scores = op.block_scores(q, e, page, at, ctx, 203, scores=torch.zeros((3, hkv, width), device=DEV))
        chosen, count = op.block_select(scores, page, at, ctx, 203, 5, table=torch.full((3, hkv, 5), shift, dtype=torch.int32,
                                                                                       device=DEV))
        out, lse = op.block_forward(q, pool, pool, chosen, count, 5 * page, lse=torch.empty((3, 32), device=DEV))
        _, all_lse = op.forward_paged(q, pool, pool, at, ctx, 203, lse=torch.empty((3, 32), device=DEV))
        paid = op.attn_weights_paged(q, all_lse, pool, at, ctx, 203)
        got[shift] = (e[shift:][table[0].long()].view(torch.uint8), scores, chosen - shift, count, out, lse, paid)
    for i, (a, b) in enumerate(zip(got[0], got[base])):
        assert torch.equal(a, b), i
    # One long cache without pages: the sequence begins past 2^32 bytes.
    flat, start = big.view(-1, hkv, d), (base + few - width) * page
    begin = torch.tensor([start], dtype=torch.int64, device=DEV)
    own = flat[start:start + 203].view(torch.uint8).clone().view(kind)
    a, b = (op.attn_weights(q[:1], all_lse[:1], k, s, ctx[:1], 203) for k, s in ((flat, begin), (own, begin * 0)))
    assert torch.equal(a, b)


def test_rows_of_weights_past_32_bits():
    """Rows of weights further apart than 2^32 bytes."""
    say("weights past 32 bits")
    from tests.test_gpu_evict import make_op

    g = torch.Generator().manual_seed(13)
    n, stride = 3000, 2 ** 30 + 64
    wide = torch.empty((2 * stride,), device=DEV).view(2, stride)
    near = torch.rand((2, n), generator=g).to(DEV)
    wide[:, :n] = near
    ctx = torch.tensor([n, n - 1], dtype=torch.int32, device=DEV)
    op = make_op("bf16", 8, 2, 64, 2, n)
    got = [op.keep_tokens(w, ctx, n, 700, 3, 5) for w in (wide, near)]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][3], got[1][3])
    k = torch.randn((2 * n, 2, 64), generator=g).to(torch.bfloat16).to(DEV)
    q = torch.randn((2, 8, 64), generator=g).to(torch.bfloat16).to(DEV)
    lse, start = torch.full((2, 8), 9.0, device=DEV), torch.tensor([0, n], dtype=torch.int64, device=DEV)
    for w in (wide, near):
        op.attn_weights(q, lse, k, start, ctx, n, prior=w, decay=0.5, out=w)
    assert torch.equal(wide[:, :n], near)
