"""The operators together, as a serving loop uses them: pages for prompts, keys rotated into the cache, prefill, a fork,
captured decode steps that take their pages as they go, the contexts cut, more steps, the pages given back.

Beside it goes a record of what every sequence should hold: for each token the K and V rows that the rotation stored
when it was new. Attention is checked in 64 bits over the recorded rows, with the gates of the decode and prefill tests
(gpu_util.check: 1e-4 of the largest output; queries and rows are the stored ones, so no rounding of them counts).
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.ops_util import pages_of, rotated  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, HKV, D, MAX = 8, 2, 128, 400
KS, VS = 2.0 ** -5, 2.0 ** -5


class Loop:
    def __init__(self, dtype, page, rows, num_pages, norm=True, seed=1):
        from paper_2605_30842_amd.binding import DecodeAttention, KVPages

        scales = dict(k_scale=KS, v_scale=VS) if dtype == "fp8" else {}
        self.dtype, self.page, self.rows = dtype, page, rows
        self.op = DecodeAttention(HQ, HKV, D, dtype, 1.0 / math.sqrt(D), rows, MAX, **scales)
        self.q_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        cache = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}[dtype]
        self.k = torch.zeros((num_pages, page, HKV, D), dtype=cache, device=DEV)
        self.v = torch.zeros_like(self.k)
        self.table = torch.full((rows, pages_of(MAX, page)), -1, dtype=torch.int32, device=DEV)
        self.ctx = torch.zeros(rows, dtype=torch.int32, device=DEV)
        self.counts = torch.zeros(num_pages, dtype=torch.int32, device=DEV)
        self.pages = KVPages(self.op, self.k, self.v, self.table, self.ctx, self.counts, MAX)
        self.gen = torch.Generator().manual_seed(seed)
        a = torch.arange(2 * MAX, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
        self.cos_sin = torch.cat([a.cos(), a.sin()], 1).float().to(DEV)
        w = [(1 + 0.2 * torch.randn(D, generator=self.gen)).to(self.q_dtype).to(DEV) for _ in range(2)]
        self.weights = w if norm else [None, None]
        self.kept = [[] for _ in range(rows)]  # (K row, V row) of each token, as stored
        self.where = [0] * rows                # position of the next token

    def wide(self, t, scale):
        x = t.view(torch.float8_e4m3fn).double() * scale if self.dtype == "fp8" else t.double()
        return x.cpu()

    def stored(self, r):
        """The rows that the cache holds for sequence r, through its table."""
        n = int(self.ctx[r])
        t = torch.arange(n, device=DEV)
        at = self.table[r].long()[t // self.page] * self.page + t % self.page
        return (self.wide(self.k.view(-1, HKV, D)[at], KS), self.wide(self.v.view(-1, HKV, D)[at], VS))

    def check_record(self):
        for r in range(self.rows):
            assert int(self.ctx[r]) == len(self.kept[r])
            if self.kept[r]:
                k, v = self.stored(r)
                assert torch.equal(k, torch.stack([a for a, _ in self.kept[r]])), f"K of {r}"
                assert torch.equal(v, torch.stack([b for _, b in self.kept[r]])), f"V of {r}"

    def take_new(self, r, m, new_k):
        """Record the m newest tokens of r; their keys are near the formula's."""
        k, v = self.stored(r)
        self.kept[r] += list(zip(k[-m:], v[-m:]))
        at = np.arange(self.where[r], self.where[r] + m)
        w = self.weights[1]
        z, _ = rotated(new_k.double().cpu().numpy(), None if w is None else w.double().cpu().numpy(), 1e-6,
                       self.cos_sin.double().cpu().numpy(), at, False)
        half = {"f32": 2.0 ** -18, "bf16": 2.0 ** -7.9, "fp8": 2.0 ** -3.9}[self.dtype]
        assert np.all(np.abs(k[-m:].numpy() - z) <= half * np.abs(z) + 2e-4 + (KS * 2.0 ** -10 if self.dtype == "fp8" else 0))
        self.where[r] += m

    def attended(self, q, r, limit):
        k = torch.stack([a for a, _ in self.kept[r][:limit]])
        v = torch.stack([b for _, b in self.kept[r][:limit]])
        scale = float(np.float32(1.0 / math.sqrt(D)))
        out = torch.zeros(HQ, D, dtype=torch.float64)
        for h in range(HQ):
            s = torch.softmax(scale * (k[:, h // (HQ // HKV)] @ q[h]), 0)
            out[h] = s @ v[:, h // (HQ // HKV)]
        return out

    def near(self, got, want, what):
        err = float((got.double().cpu() - want).abs().max())
        assert err <= 1e-4 * max(1.0, float(want.abs().max())), (what, err)

    def prompts(self, lens):
        """Pages, rotation and prefill of new tokens; lens[r] may be 0."""
        assert int(self.pages.reserve(torch.tensor(lens, dtype=torch.int32, device=DEV))) == 0
        starts = [sum(lens[:r]) for r in range(self.rows)]
        x = torch.randn((sum(lens), HQ + 2 * HKV, D), generator=self.gen).to(self.q_dtype).to(DEV)
        more = dict(q_start=torch.tensor(starts, dtype=torch.int64, device=DEV),
                    q_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), max_q_len=max(lens))
        at = [self.where[r] + i for r in range(self.rows) for i in range(lens[r])]
        q = self.op.rope_append_paged(x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], self.k, self.v, self.table, self.ctx, MAX,
                                      self.cos_sin, *self.weights, positions=torch.tensor(at, dtype=torch.int32, device=DEV),
                                      **more)
        for r in range(self.rows):
            if lens[r]:
                self.take_new(r, lens[r], x[starts[r]:starts[r] + lens[r], HQ:HQ + HKV])
        self.check_record()
        if self.dtype == "f32":
            return
        out, _ = self.op.prefill_paged(q, more["q_start"], more["q_lens"], max(lens), self.k, self.v, self.table, self.ctx, MAX)
        for r in range(self.rows):
            for i in sorted({0, lens[r] // 2, lens[r] - 1} if lens[r] else ()):
                row, limit = starts[r] + i, len(self.kept[r]) - lens[r] + i + 1
                self.near(out[row], self.attended(q[row].double().cpu(), r, limit), f"prefill of {r}, token {i}")

    def steps(self, live, count):
        """Decode steps of the rows in `live`, captured once and replayed."""
        one = torch.tensor([1 if r in live else 0 for r in range(self.rows)], dtype=torch.int32, device=DEV)
        x = torch.zeros((self.rows, HQ + 2 * HKV, D), dtype=self.q_dtype, device=DEV)
        at = torch.zeros(self.rows, dtype=torch.int32, device=DEV)
        q = torch.zeros((self.rows, HQ, D), dtype=self.q_dtype, device=DEV)
        out = torch.zeros((self.rows, HQ, D), device=DEV)
        missing = torch.ones((), dtype=torch.int32, device=DEV)

        q_lens = torch.tensor([1 if r in live else 0 for r in range(self.rows)], dtype=torch.int32, device=DEV)
        q_start = torch.arange(self.rows, dtype=torch.int64, device=DEV)

        def step():
            self.pages.reserve(one, missing=missing)
            self.op.rope_append_paged(x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], self.k, self.v, self.table, self.ctx,
                                      MAX, self.cos_sin, *self.weights, positions=at, q_start=q_start, q_lens=q_lens,
                                      max_q_len=1, q_out=q)
            self.op.forward_paged(q, self.k, self.v, self.table, self.ctx, MAX, out=out)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(count):
            x.copy_(torch.randn(x.shape, generator=self.gen).to(self.q_dtype))
            at.copy_(torch.tensor(self.where, dtype=torch.int32))
            graph.replay()
            torch.cuda.synchronize()
            assert int(missing) == 0
            for r in live:
                self.take_new(r, 1, x[r:r + 1, HQ:HQ + HKV])
            if i % 5 == 0 or i == count - 1:
                self.check_record()
                for r in live:
                    self.near(out[r], self.attended(q[r].double().cpu(), r, len(self.kept[r])), f"step {i} of {r}")

    def fork(self, parents, children):
        i32 = dict(dtype=torch.int32, device=DEV)
        assert int(self.pages.fork(torch.tensor(parents, **i32), torch.tensor(children, **i32))) == 0
        for p, c in zip(parents, children):
            self.kept[c], self.where[c] = list(self.kept[p]), self.where[p]
        self.check_record()

    def compact(self, rows, keeps):
        i32 = dict(dtype=torch.int32, device=DEV)
        starts = [sum(len(k) for k in keeps[:i]) for i in range(len(keeps))]
        assert int(self.pages.compact(torch.tensor(rows, **i32), torch.tensor([p for k in keeps for p in k], **i32),
                                      torch.tensor(starts, dtype=torch.int64, device=DEV),
                                      torch.tensor([len(k) for k in keeps], **i32))) == 0
        for r, keep in zip(rows, keeps):
            self.kept[r] = [self.kept[r][t] for t in keep]
        self.check_record()

    def release(self, rows):
        self.pages.release(torch.tensor(rows, dtype=torch.int32, device=DEV))
        for r in rows:
            self.kept[r], self.where[r] = [], 0
        self.check_record()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_a_serving_run(dtype, page):
    say("serving run", dtype, page)
    s = Loop(dtype, page, rows=5, num_pages=pages_of(1000, page) + 12, norm=page != 64)
    s.prompts([100, 0, 37, 0, 0])
    s.fork([0, 0, 2], [1, 3, 4])             # several continuations of a history
    s.steps([0, 1, 2, 4], 20)                # they part ways, row 3 waits
    n = len(s.kept[1])
    s.compact([1, 4], [list(range(33)) + list(range(n - 40, n)), [0] + list(range(5, 50))])
    s.prompts([0, 25, 0, 60, 1])             # a summary's tokens after the cut; an observation
    s.steps([1, 3], 18)
    s.release([0, 2])
    s.prompts([64, 0, 16, 0, 0])             # new sequences on the pages that came back
    s.steps([0, 1, 2, 3, 4], 6)
    s.release([0, 1, 2, 3, 4])
    assert int(s.counts.abs().sum()) == 0 and bool((s.table == -1).all())
