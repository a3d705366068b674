"""Pages that run out inside a captured loop: what reserve grants is the q_lens of the calls that store and read.

A row that gets no room keeps its length, so a fixed q_lens would store a step's token over the row's last one, which
lies in a full page that forks may share. Here every stored row is compared bit for bit.
"""

import random

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.ops_util import PagesModel, pages_of  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, HKV, D = 8, 2, 64


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


class State:
    def __init__(self, rows, num_pages, page, max_ctx, dtype="bf16"):
        from paper_2605_30842_amd.binding import DecodeAttention, KVPages

        self.op = DecodeAttention(HQ, HKV, D, dtype, 0.125, rows, max_ctx)
        shape = (num_pages, page, HKV, D)
        self.k = torch.randint(0, 100, shape, device=DEV).to(torch.uint8 if dtype == "fp8" else torch.bfloat16)
        self.v = self.k.clone()
        width = pages_of(max_ctx, page)
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
        self.ctx, self.counts = _i32([0] * rows), _i32([0] * num_pages)
        self.max_ctx = max_ctx
        self.p = KVPages(self.op, self.k, self.v, self.table, self.ctx, self.counts, max_ctx)
        self.m = PagesModel(rows, width, num_pages, page, max_ctx)

    def granted(self, add):
        """What the model says, which is changed by the call."""
        was = list(self.m.ctx)
        missing = self.m.reserve(add)
        return [n - w for n, w in zip(self.m.ctx, was)], missing

    def check(self):
        assert self.ctx.tolist() == self.m.ctx and self.table.tolist() == self.m.table
        assert self.counts.tolist() == self.m.counts


@pytest.mark.parametrize("rows,num_pages", [(1, 2), (7, 12), (1500, 3000), (900, 20000), (2600, 9000)])
def test_granted_lengths(rows, num_pages):
    """Pools of one chunk of the counts and of several; refused rows, and calls that lack pages."""
    say("granted", rows, num_pages)
    rng = random.Random(rows)
    s = State(rows, num_pages, 4, 40)
    got, lacked = torch.empty(rows, dtype=torch.int32, device=DEV), 0
    for _ in range(12):
        most = rng.choice([2, 9, 30])
        add = [rng.choice([0, 1, rng.randint(0, most), rng.randint(0, most), -2, 41]) for _ in range(rows)]
        got.fill_(77)
        missing = s.p.reserve(_i32(add), granted=got)
        want, lack = s.granted(add)
        assert int(missing) == lack and got.tolist() == want
        s.check()
        lacked += lack > 0
        if lack:
            gone = rng.sample(range(rows), (rows + 1) // 2)
            s.p.release(_i32(gone))
            s.m.release(gone)
    assert lacked or rows * 10 < num_pages


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("end", ["pool", "max_ctx_len"])
def test_a_captured_loop_without_room_stores_nothing(dtype, end):
    """Three rows on a history of two whole pages, and a fourth that ends earlier. Replays run into the end of the
    pool, or of max_ctx_len; then a row gives its pages back and the loop goes on."""
    page, max_ctx = 16, 64 if end == "pool" else 40
    s = State(4, 4 if end == "pool" else 30, page, max_ctx, dtype)
    say("captured loop", dtype, end)
    assert int(s.p.reserve(_i32([32, 0, 0, 5]))) == s.m.reserve([32, 0, 0, 5]) == 0
    assert int(s.p.fork(_i32([0, 0]), _i32([1, 2]))) == s.m.fork([0, 0], [1, 2]) == 0
    add = [0, 1, 1, 1]
    one, granted, missing = _i32(add), _i32([9] * 4), _i32([0])
    x = torch.randn((4, HQ + 2 * HKV, D), device=DEV).to(torch.bfloat16)
    angles = torch.zeros((1, 0), device=DEV)
    start = torch.arange(4, dtype=torch.int64, device=DEV)
    q = torch.zeros((4, HQ, D), dtype=torch.bfloat16, device=DEV)

    def step():
        s.p.reserve(one, missing=missing, granted=granted)
        s.op.rope_append_paged(x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], s.k, s.v, s.table, s.ctx, max_ctx, angles,
                               q_start=start, q_lens=granted, max_q_len=1, q_out=q)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()

    def refused_and_stored(i):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))
        before = s.k.clone(), s.v.clone()
        graph.replay()
        want, lack = s.granted(add)
        torch.cuda.synchronize()
        assert granted.tolist() == want and int(missing) == lack
        s.check()
        for pool, was, first in ((s.k, before[0], HQ), (s.v, before[1], HQ + HKV)):
            new = x[:, first:first + HKV]
            if dtype == "fp8":
                new = new.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            for r in range(4):
                if want[r]:
                    t = s.m.ctx[r] - 1
                    was[s.m.table[r][t // page], t % page] = new[r]
            assert torch.equal(pool, was), f"replay {i}"
        return sum(want), lack

    full = [refused_and_stored(i) for i in range(14)]
    if end == "pool":  # one page is left for the first step's two rows: none of its rows grows, nor of any other
        assert all(f == (0, 1) for f in full)
    else:
        assert full[:8] == [(3, 0)] * 8 and full[8:] == [(1, 0)] * 6
    s.p.release(_i32([2]))
    s.m.release([2])
    add[2] = 0
    one.copy_(torch.tensor(add, dtype=torch.int32))
    assert [refused_and_stored(100 + i)[0] for i in range(6)] == [2 if end == "pool" else 1] * 6


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_prefill_of_granted_lengths(dtype):
    """Rows without room have no new token: prefill leaves their output rows as they were."""
    s = State(3, 12, 16, 64, dtype)
    s.p.reserve(_i32([20, 60, 3]))
    granted, lens = _i32([9] * 3), [5, 7, 4]
    assert int(s.p.reserve(_i32(lens), granted=granted)) == 0 and granted.tolist() == [5, 0, 4]
    q = torch.randn((16, HQ, D), device=DEV).to(torch.bfloat16)
    start = torch.tensor([0, 5, 12], dtype=torch.int64, device=DEV)
    out = torch.full((16, HQ, D), 3.0, device=DEV)
    s.op.prefill_paged(q, start, granted, 7, s.k, s.v, s.table, s.ctx, 64, out=out)
    want, _ = s.op.prefill_paged(q, start, _i32([5, 0, 4]), 7, s.k, s.v, s.table, s.ctx, 64)
    torch.cuda.synchronize()
    assert bool((out[5:12] == 3).all()) and torch.equal(out[:5], want[:5]) and torch.equal(out[12:], want[12:])
