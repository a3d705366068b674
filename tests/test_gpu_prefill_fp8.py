"""Prefill over FP8 caches: the HIP path against softmax attention in 64 bits over the codes' values.

Tolerances. Scores: the products of bf16 queries and codes are exact in float32, their sums are not, and neither are the
exponential's argument and the exponential; the weights are carried as two f16 values, 2^-21 of each off at most. For
N(0, 1) queries and values of 1/sqrt(d) scaled scores these errors are independent from key to key and at most about
1e-6 of a weight each (sums of 128 in float32 3e-7, argument 5e-7, split 5e-7), so the outputs' error is about 1e-6 of
their norm; four times that is the gate (NORM). Every element also meets the bound that check_prefill in gpu_util holds
for bf16 caches: 2^-14 of sum_t w_t |v_t|, 1e-5 of the value, 1e-6.
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import check_prefill, say  # noqa: E402
from tests.ops_util import pages_of  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NORM = 4e-6
NAN = 0x7F


def attend(q, k, v, scale, limits):
    """softmax(scale q k^T) v in 64 bits; row i sees the keys 0 .. limits[i]."""
    s = (q @ k.t()) * scale
    s = torch.where(torch.arange(k.shape[0])[None, :] <= limits[:, None], s, -math.inf)
    lse = torch.logsumexp(s, 1)
    w = torch.exp(s - lse[:, None])
    return w @ v, w @ v.abs(), lse


class Case:
    def __init__(self, lens, new, hq=8, hkv=2, d=128, page=0, k_scale=2.0 ** -6, v_scale=2.0 ** -6, seed=1, bound=None,
                 spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.hq, self.hkv, self.d, self.page = list(lens), list(new), hq, hkv, d, page
        self.k_scale, self.v_scale, self.scale = k_scale, v_scale, 1.0 / math.sqrt(d)
        self.bound = bound or max(max(lens), 1)
        if page:
            counts = [pages_of(n, page) for n in lens]
            total = sum(counts) + 2
            order = torch.randperm(total, generator=g).tolist()
            self.where = torch.full((len(lens), max(1, pages_of(self.bound, page))), -1, dtype=torch.int32)
            for b, n in enumerate(counts):
                self.where[b, :n] = torch.tensor(order[sum(counts[:b]):sum(counts[:b]) + n], dtype=torch.int32)
            shape = (total, page, hkv, d)
        else:
            self.where = torch.tensor([3 + sum(lens[:b]) + 2 * b for b in range(len(lens))], dtype=torch.int64)
            shape = (sum(lens) + 2 * len(lens) + 6, hkv, d)

        def codes(scale):
            x = torch.randn(shape, generator=g) * spread
            return (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

        self.k, self.v = codes(k_scale), codes(v_scale)
        live = torch.zeros(math.prod(shape[:-2]), dtype=torch.bool)
        for b, n in enumerate(lens):
            live[self.rows(b)] = True
        self.k.view(-1, hkv, d)[~live] = NAN  # whatever no context covers
        self.v.view(-1, hkv, d)[~live] = NAN
        self.starts = [sum(new[:b]) for b in range(len(new))]
        self.q = torch.randn((max(sum(new), 1), hq, d), generator=g).to(torch.bfloat16)[:sum(new)]

    def rows(self, b):
        t = torch.arange(self.lens[b])
        if self.page:
            return self.where[b].long()[t // self.page] * self.page + t % self.page
        return int(self.where[b]) + t

    def context(self, b, hk):
        def wide(t, scale):
            return t.view(-1, self.hkv, self.d)[self.rows(b), hk].view(torch.float8_e4m3fn).double() * float(np.float32(scale))

        return wide(self.k, self.k_scale), wide(self.v, self.v_scale)

    def op(self):
        from paper_2605_30842_amd.binding import DecodeAttention

        return DecodeAttention(self.hq, self.hkv, self.d, "fp8", self.scale, len(self.lens), self.bound,
                               k_scale=self.k_scale, v_scale=self.v_scale)

    def run(self, op=None, **kw):
        op = op or self.op()
        i32 = torch.int32
        lse = torch.full(self.q.shape[:2], float("nan"), device=DEV)
        args = (self.q.to(DEV), torch.tensor(self.starts, dtype=torch.int64, device=DEV),
                torch.tensor(self.new, dtype=i32, device=DEV), max(self.new), self.k.to(DEV), self.v.to(DEV),
                self.where.to(DEV), torch.tensor(self.lens, dtype=i32, device=DEV), self.bound)
        out, lse = (op.prefill_paged if self.page else op.prefill)(*args, lse=lse, **kw)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    def want(self):
        out = torch.zeros(self.q.shape, dtype=torch.float64)
        size, lse = out.clone(), out[..., 0].clone()
        scale = float(np.float32(self.scale))
        for b, (n, m, s) in enumerate(zip(self.lens, self.new, self.starts)):
            for h in range(self.hq if m else 0):
                k, v = self.context(b, h // (self.hq // self.hkv))
                o, a, l = attend(self.q[s:s + m, h].double(), k, v, scale, n - m + torch.arange(m))
                out[s:s + m, h], size[s:s + m, h], lse[s:s + m, h] = o, a, l
        return out, lse, size

    def check(self, what, **kw):
        say("fp8 prefill", what, "L", self.lens[:8], "M", self.new[:8], "G", self.hq // self.hkv, "D", self.d, "page",
            self.page)
        out, lse = self.run(**kw)
        ref, ref_lse, size = self.want()
        check_prefill(out.numpy(), lse.numpy(), ref.numpy(), ref_lse.numpy(), size.numpy(), what)
        err = float((out.double() - ref).norm() / ref.norm())
        say(f"  error {err:.2e} of the norm")
        assert err <= NORM, what
        return out, lse


RAGGED_L = [40, 7, 1, 0, 64, 300, 1000, 129, 700]
RAGGED_M = [5, 7, 1, 0, 16, 129, 1000, 33, 70]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 1, 2, 8, 16, 64, 128])
def test_ragged(page, d):
    Case(RAGGED_L, RAGGED_M, d=d, page=page, seed=page + d, bound=1010).check("ragged")


@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
def test_groups(group, d):
    Case([200, 77, 500], [200, 3, 150], hq=2 * group, d=d, seed=group).check("groups")


@pytest.mark.parametrize("page", [0, 16, 1])
def test_more_workgroups_than_units(page):
    rng = np.random.default_rng(59)
    lens = [1, 64, 65, 700, 300, 129] + rng.integers(1, 300, size=42).tolist()
    new = [1, 64, 33, 31, 150, 2] + [int(min(n, m)) for n, m in zip(lens[6:], rng.integers(1, 33, size=42))]
    Case(lens, new, hq=16, hkv=8, page=page, seed=7).check("many")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,lens,new", [(0, [9000], [40]), (64, [5000, 12000], [17, 130]), (8, [6001], [1])])
def test_keys_shared_by_workgroups(page, lens, new, d):
    """Few new tokens over long prefixes: with scratch the keys of a block are split, without they are not."""
    c = Case(lens, new, hq=32, hkv=8, d=d, page=page, seed=3)
    op = c.op()
    assert op.prefill_workspace_bytes(len(lens), max(new), max(lens)) > 0
    split, split_lse = c.check("split", op=op)
    whole, whole_lse = c.run(op=op, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    assert float((split - whole).abs().max()) <= 1e-5 and float((split_lse - whole_lse).abs().max()) <= 1e-5
    assert not torch.equal(split, whole)


@pytest.mark.parametrize("most", [0, 1])
@pytest.mark.parametrize("page", [0, 16, 2])
@pytest.mark.parametrize("group,d", [(1, 128), (4, 128), (8, 128), (4, 64), (16, 64)])
def test_few_rows(group, d, page, most):
    """Blocks of at most 64 rows and, with one more token, of more: contexts whose last tile ends in its first or its
    second 32 keys, sequences without a new token, single tokens, and rows that see no key of a tile's second part."""
    m = 64 // group + most
    lens = [m, 32, 33, 63, 64, 65, 96 + m, 97, 1000, 0, 5, 2048 + m // 2]
    new = [min(n, k) for n, k in zip(lens, [m, 1, m, m, 2, m, m, 1, m, 0, 1, m])]
    Case(lens, new, hq=2 * group, d=d, page=page, seed=10 * group + most).check("few rows")


@pytest.mark.parametrize("d", [64, 128])
def test_one_new_token_is_a_decode_step(d):
    c = Case([700, 1, 64, 3000], [1, 1, 1, 1], d=d, page=16, k_scale=0.011, v_scale=0.03, seed=5)
    out, lse = c.check("decode")
    op = c.op()
    want, _ = op.forward_paged(c.q.to(DEV), c.k.to(DEV), c.v.to(DEV), c.where.to(DEV),
                               torch.tensor(c.lens, dtype=torch.int32, device=DEV), c.bound)
    assert float((out - want.cpu()).abs().max()) <= 2e-5 * max(1.0, float(want.abs().max()))


@pytest.mark.parametrize("k_scale,v_scale", [(1.0, 1.0), (0.0173, 3.7), (2.0 ** -6, 2.0 ** -20)])
def test_scales(k_scale, v_scale):
    Case([300, 90], [300, 20], k_scale=k_scale, v_scale=v_scale, spread=min(1.0, v_scale * 100), seed=6).check("scales")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("new", [90, 13])  # 13: few rows, a tile's keys shared by waves
def test_scores_around_the_lazy_bound(d, split, new):
    """Tiles of equal scores: below the running maximum, a little above it (no rescale), far above (rescale), and far
    below, in both halves of a workgroup's tiles and, shared, in every split."""
    steps = [0.0, -3.0, 5.0, 5.5, 30.0, 10.0, 37.9, 38.1, -60.0, 60.0, 59.0, 0.0, 64.0, 60.0, 80.0, 75.0]
    n = 64 * len(steps) - 10
    c = Case([n], [new], hq=4, hkv=1, d=d, seed=8)
    c.q.zero_()
    c.q[:, :, 0] = 1.0
    kv = c.k.view(torch.float8_e4m3fn)[3:3 + n]
    c.k[3:3 + n] = 0
    width = 64 if new == 90 else 32  # few rows: other steps for the two parts of a tile too
    scores = torch.tensor(steps * (64 // width)).repeat_interleave(width)[:n] + (torch.arange(n) % 3) * 0.25
    codes = (scores / (math.log2(math.e) * c.scale) / 16).clamp(-448, 448).to(torch.float8_e4m3fn)
    c.q[:, :, 0] = 16.0 * c.k_scale ** 0
    c.k_scale = 1.0
    kv[:, 0, 0] = codes
    if not split:
        c.check("lazy bound")
        return
    op = c.op()
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    c.check("lazy bound, workspace", op=op, workspace=ws)


def test_many_small_weights_count():
    """One key of weight 1 among 30000 of weight 2^-20.2: together they are 2.4% of the sum, and their values are what
    the output is made of.

    The weights enter as two f16 values, 2^9 times as large. 2^-11.2 has the f16 neighbours 2^-22 apart, so the first
    value is off by at most 2^-23, and the second one, a multiple of 2^-24, by at most 2^-25 of what is left: 2^-34 of
    the weight 1. All 30000 are the same and may be off the same way, 30000 * 2^-34 = 1.7e-6 in an output of 0.024. To
    that come the exponent's argument (scale, log2(e) and their product rounded, 2^-23 of 20.2, times ln 2: 1.7e-6 of a
    weight) and the sums (1e-6), as in every form of the kernel.
    """
    n, d = 30001, 64
    c = Case([n], [3], hq=2, hkv=1, d=d, seed=9, k_scale=1.0, v_scale=1.0)
    c.q.zero_()
    c.q[:, :, 0] = 1.0
    c.k[3:3 + n] = 0
    kf = c.k.view(torch.float8_e4m3fn)
    kf[3:3 + n, 0, 0] = -112.0   # score -14 = -20.2 in log2 units
    kf[3, 0, 0] = 0.0
    vf = c.v.view(torch.float8_e4m3fn)
    vf[3:3 + n] = torch.tensor(1.0).to(torch.float8_e4m3fn)
    vf[3] = torch.tensor(0.0).to(torch.float8_e4m3fn)
    ref, _, _ = c.want()
    assert 0.02 < float(ref[0, 0, 0]) < 0.03
    for ws in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
        out, _ = c.run() if ws is None else c.run(workspace=ws)
        err = float((out.double() - ref).abs().max())
        assert err <= 30000 * 2.0 ** -34 + 4e-6 * float(ref.max()), err


def test_smallest_and_largest_codes():
    """Subnormal codes and 448 are values like any other."""
    c = Case([500], [64], d=64, seed=10, k_scale=1.0, v_scale=1.0)
    g = torch.Generator().manual_seed(4)
    small = torch.randint(0, 8, c.k.shape, generator=g, dtype=torch.uint8) | (torch.randint(0, 2, c.k.shape, generator=g, dtype=torch.uint8) << 7)
    live = torch.zeros(c.k.shape[0], dtype=torch.bool)
    live[c.rows(0)] = True
    c.k[live] = small[live]
    c.v[live] = torch.where(torch.rand(c.v.shape, generator=g) < 0.5, 0x7E, 0xFE).to(torch.uint8)[live]
    c.check("smallest keys, largest values")
    c.v[live] = small[live]
    c.check("smallest values")


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("few", [False, True])
def test_nan_codes(split, few):
    """A NaN key: every row that sees it is NaN, out and lse, and no other. A NaN value in the prefix: the outputs at
    its head_dim entry."""
    n, m = (3000, 40) if split else (200, 120)
    m = 14 if few else m
    for where in ("k", "v"):
        c = Case([n, n], [m, m], hq=8, hkv=2, seed=11)
        clean, clean_lse = c.run()
        t = n - 10 if where == "k" else 20
        row = int(c.where[0]) + t
        (c.k if where == "k" else c.v)[row, 1, 5] = NAN
        out, lse = c.run()
        assert torch.equal(out[m:], clean[m:]) and torch.equal(out[:m, :4], clean[:m, :4])
        if where == "k":
            first = m - 10
            assert bool(torch.isnan(out[first:m, 4:]).all()) and bool(torch.isnan(lse[first:m, 4:]).all())
            assert torch.equal(out[:first, 4:], clean[:first, 4:]) and torch.equal(lse[:first], clean_lse[:first])
        else:
            assert bool(torch.isnan(out[:m, 4:, 5]).all()) and torch.equal(lse, clean_lse)
            keep = [i for i in range(c.d) if i != 5]
            assert torch.equal(out[:m, 4:][..., keep], clean[:m, 4:][..., keep])


def test_rows_of_no_sequence_stay():
    c = Case([50, 20], [3, 20], seed=12)
    c.starts = [1, 7]
    q = torch.randn((30, c.hq, c.d)).to(torch.bfloat16)
    q[1:4], q[7:27] = c.q[:3], c.q[3:]
    want, _ = Case([50, 20], [3, 20], seed=12).run()
    c.q = q
    out = torch.full(q.shape, 5.0, device=DEV)
    got, lse = c.run(out=out)
    assert torch.equal(got[1:4], want[:3]) and torch.equal(got[7:27], want[3:])
    for rows in (got[:1], got[4:7], got[27:]):
        assert bool((rows == 5).all())
    assert bool(torch.isnan(lse[4:7]).all())


def test_bad_entries_and_lengths_stay_inside():
    """As for bf16 caches: entries outside the pool are read as page 0, lengths are clamped to the call's bounds."""
    c = Case([100, 64, 90], [20, 64, 10], page=16, seed=13)
    good, _ = c.run()
    c.where[0, 2] = 10 ** 6
    c.where[0, 3] = -7
    out, _ = c.run()
    assert torch.equal(out[20:], good[20:])
    c.where[0, 2] = c.where[0, 3] = 0
    want, _ = c.run()
    assert torch.equal(torch.nan_to_num(out, 9.0), torch.nan_to_num(want, 9.0))
    c2 = Case([100, 64, 90], [20, 64, 10], page=16, seed=13)
    op = c2.op()
    c2.lens[1] = 10 ** 6
    c2.where[1] = c2.where[0, :c2.where.shape[1]]
    out, _ = c2.run(op=op)
    assert torch.equal(out[:20], good[:20]) and torch.equal(out[84:], good[84:])


def test_captured_and_other_stream():
    c = Case([5000], [60], hq=32, hkv=8, page=16, seed=14)
    op = c.op()
    want, _ = c.run(op=op)
    i32 = torch.int32
    q, k, v, table = (t.to(DEV) for t in (c.q, c.k, c.v, c.where))
    args = (q, torch.zeros(1, dtype=torch.int64, device=DEV), torch.tensor([60], dtype=i32, device=DEV), 60, k, v, table,
            torch.tensor([5000], dtype=i32, device=DEV), 5000)
    out = torch.zeros(q.shape, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    op.prefill_paged(*args, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out.cpu(), want)
    got, _ = op.prefill_paged(*args, stream=side)  # its own output: memory of that stream
    side.synchronize()
    assert torch.equal(got.cpu(), want)
    owner = [s["stream"] for s in torch.cuda.memory_snapshot() if 0 <= got.data_ptr() - s["address"] < s["total_size"]]
    assert owner == [side.cuda_stream]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.prefill_paged(*args, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want)
        torch.empty(1 << 24, dtype=torch.uint8, device=DEV).fill_(255)


def test_cache_past_4_gib():
    """A sequence in the last pages of a pool whose offsets pass 32 bits."""
    pages, page, n = 4200, 1024, 3000  # 1 MB a page
    g = torch.Generator().manual_seed(15)
    c = Case([n], [50], hq=16, hkv=8, page=page, seed=15)
    k = torch.full((pages, page, 8, 128), NAN, dtype=torch.uint8, device=DEV)
    v = torch.full_like(k, NAN)
    new = torch.tensor([[pages - 2, pages - 4, pages - 1]], dtype=torch.int32)
    for i in range(3):
        k[int(new[0, i])], v[int(new[0, i])] = c.k[int(c.where[0, i])].to(DEV), c.v[int(c.where[0, i])].to(DEV)
    want, _ = c.run()
    op = c.op()
    i32 = torch.int32
    out, _ = op.prefill_paged(c.q.to(DEV), torch.zeros(1, dtype=torch.int64, device=DEV),
                              torch.tensor([50], dtype=i32, device=DEV), 50, k, v, new.to(DEV),
                              torch.tensor([n], dtype=i32, device=DEV), n)
    assert torch.equal(out.cpu(), want)
