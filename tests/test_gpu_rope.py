"""Rotate-and-store on the GPU against the plain 64-bit form, through the wrapper.

Tolerances. Before its last rounding an element z = y_a c - y_b s carries: the sum of at most 128 squares, all positive,
in a tree of at most 12 additions after one rounded product each (13 steps of 2^-24, halved by the root), the mean's eps
and the root (2), its product with x and the weight (3), the product with the table and the addition (3): less than
16 * 2^-24 = 2^-20 of |y_a c| + |y_b s|. The last rounding is half a step: 2^-8 (bf16) or 2^-24 (f32) of the value. An FP8
code is off by 2^-4 of the value, or half of the smallest step, 2^-10, where it is subnormal; what is rounded is the
value times the rounded reciprocal of the scale, two roundings more (2^-22 covers both).
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402
from tests.ops_util import FP8_MAX, pages_of, rotated  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
KS, VS = 0.013, 2.0 ** -5  # FP8 scales, one of them no power of two
F32_STEPS = 2.0 ** -20


def _op(dtype, hq, hkv, d, batch, max_ctx):
    from paper_2605_30842_amd.binding import DecodeAttention

    scales = dict(k_scale=KS, v_scale=VS) if dtype == "fp8" else {}
    return DecodeAttention(hq, hkv, d, dtype, 1.0 / math.sqrt(d), batch, max_ctx, **scales)


def _np(t):
    return t.to(torch.float64).cpu().numpy()


class Case:
    """A cache filled with a pattern, the new tokens in one buffer, and what should come out."""

    def __init__(self, dtype="bf16", hq=8, hkv=2, d=128, page=16, lens=(5, 0, 40), new=None, rot=None, norm=(True, True),
                 interleaved=False, positions=None, spare_rows=3, seed=1, fused=True, table_rows=None, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.d, self.page = dtype, hq, hkv, d, page
        self.lens = list(lens)
        self.step = new is None
        self.new = [min(1, n) for n in lens] if self.step else list(new)
        self.rot = d if rot is None else rot
        self.interleaved, self.eps = interleaved, 1e-5
        self.max_ctx = max(max(lens), 1)
        self.q_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        cache_dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}[dtype]
        self.starts = [sum(self.new[:b]) + b for b in range(len(lens))]  # a row between sequences belongs to nobody
        rows = len(lens) if self.step else self.starts[-1] + self.new[-1] + spare_rows
        if self.step:
            self.starts = list(range(len(lens)))
        x = torch.randn((rows, hq + 2 * hkv, d), generator=g) * scale
        self.qkv = x.to(self.q_dtype).to(DEV)
        parts = (self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:])
        self.q, self.new_k, self.new_v = parts if fused else tuple(p.contiguous() for p in parts)
        w = [(1 + 0.3 * torch.randn(d, generator=g)).to(self.q_dtype).to(DEV) if n else None for n in norm]
        self.q_weight, self.k_weight = w
        table_rows = table_rows or self.max_ctx + 7
        a = torch.rand((table_rows, self.rot // 2), generator=g, dtype=torch.float64) * 6.3
        self.cos_sin = torch.cat([a.cos(), a.sin()], 1).float().contiguous().to(DEV)
        self.positions = None
        if positions is not None:
            self.positions = torch.tensor([positions(r) for r in range(rows)], dtype=torch.int32, device=DEV)
        self.ctx = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.q_start = torch.tensor(self.starts, dtype=torch.int64, device=DEV)
        self.q_lens = torch.tensor(self.new, dtype=torch.int32, device=DEV)
        if page:
            counts = [pages_of(n, page) for n in lens]
            total = sum(counts) + 2
            order = torch.randperm(total, generator=g).tolist()
            self.table = torch.full((len(lens), max(max(counts), 1)), -1, dtype=torch.int32)
            for b, n in enumerate(counts):
                self.table[b, :n] = torch.tensor(order[sum(counts[:b]):sum(counts[:b]) + n], dtype=torch.int32)
            shape = (total, page, hkv, d)
            self.block_table = self.table.to(DEV)
        else:
            self.seq_start = torch.tensor([sum(lens[:b]) + 2 * b for b in range(len(lens))], dtype=torch.int64,
                                          device=DEV)
            shape = (sum(lens) + 2 * len(lens) + 3, hkv, d)
        fill = torch.randint(0, 120, shape, generator=g)
        self.k, self.v = fill.to(cache_dtype).to(DEV), (fill + 1).to(cache_dtype).to(DEV)
        self.op = _op(dtype, hq, hkv, d, len(lens), self.max_ctx)

    def call(self, **kw):
        more = dict(q_weight=self.q_weight, k_weight=self.k_weight, eps=self.eps, positions=self.positions,
                    interleaved=self.interleaved)
        if not self.step:
            more.update(q_start=self.q_start, q_lens=self.q_lens, max_q_len=max(max(self.new), 1))
        more.update(kw)
        head = (self.q, self.new_k, self.new_v, self.k, self.v)
        if self.page:
            return self.op.rope_append_paged(*head, self.block_table, self.ctx, self.max_ctx, self.cos_sin, **more)
        return self.op.rope_append(*head, self.seq_start, self.ctx, self.max_ctx, self.cos_sin, **more)

    def slot(self, b, t):
        if self.page:
            return int(self.table[b, t // self.page]) * self.page + t % self.page
        return int(self.seq_start[b]) + t

    def tokens(self):
        """(row, cache row, cache index) of every new token."""
        out = []
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            out += [(self.starts[b] + i, self.slot(b, n - m + i), n - m + i) for i in range(m)]
        return out

    def check(self, q_out, before_k, before_v, before_q):
        rows = [r for r, _, _ in self.tokens()]
        at = [t if self.positions is None else int(self.positions[r]) for r, _, t in self.tokens()]
        slots = [s for _, s, _ in self.tokens()]
        cos_sin = _np(self.cos_sin)

        def made(x, w):
            return rotated(_np(x)[rows], None if w is None else _np(w), self.eps, cos_sin, np.array(at, dtype=np.int64),
                           self.interleaved)

        zq, size = made(self.q, self.q_weight)
        half = 2.0 ** (-24 if self.dtype == "f32" else -8)
        err = np.abs(_np(q_out)[rows] - zq)
        assert np.all(err <= half * np.abs(zq) + (1 + half) * F32_STEPS * size), (err - half * np.abs(zq)).max()
        others = np.setdiff1d(np.arange(q_out.shape[0]), rows)
        assert torch.equal(q_out[others].view(torch.uint8), before_q[others].view(torch.uint8))
        zk, ksize = made(self.new_k, self.k_weight)
        zv = _np(self.new_v)[rows]
        for cache, before, z, size, scale in ((self.k, before_k, zk, ksize, KS), (self.v, before_v, zv, np.abs(zv), VS)):
            flat, was = cache.view(-1, self.hkv, self.d), before.view(-1, self.hkv, self.d)
            if self.dtype == "fp8":
                got = _np(flat.view(torch.float8_e4m3fn).float())[slots]
                want = np.clip(z / scale, -FP8_MAX, FP8_MAX)
                slack = (F32_STEPS + 2.0 ** -22) * size / scale
                assert np.all(np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + (1 + 2.0 ** -4) * slack)
            else:
                tol = half * np.abs(z) + (1 + half) * F32_STEPS * size
                assert np.all(np.abs(_np(flat)[slots] - z) <= (0 if cache is self.v else tol))
            keep = np.setdiff1d(np.arange(flat.shape[0]), slots)
            assert torch.equal(flat[keep].view(torch.uint8), was[keep].view(torch.uint8))


def _run(c, **kw):
    q_out = torch.full((c.q.shape[0], c.hq, c.d), float("nan"), dtype=c.q_dtype, device=DEV)
    before = c.k.clone(), c.v.clone(), q_out.clone()
    got = c.call(q_out=q_out, **kw)
    torch.cuda.synchronize()
    assert got is q_out
    c.check(q_out, *before)
    return q_out


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("d,hq,hkv", [(128, 32, 8), (64, 2, 2), (128, 3 * 16, 3), (64, 8, 1)])
@pytest.mark.parametrize("page", [0, 1, 16])
def test_chunks(dtype, d, hq, hkv, page):
    say("rope chunk", dtype, d, hq, hkv, page)
    _run(Case(dtype, hq, hkv, d, page, lens=(37, 0, 5, 70, 1), new=(9, 0, 5, 33, 1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("rot,interleaved,norm", [(128, True, (True, True)), (64, False, (False, True)),
                                                  (48, True, (True, False)), (16, False, (False, False)),
                                                  (0, False, (True, True))])
def test_kinds(dtype, page, rot, interleaved, norm):
    say("rope kind", dtype, page, rot, interleaved, norm)
    c = Case(dtype, 8, 4, 128, page, lens=(20, 90), new=(20, 7), rot=rot, interleaved=interleaved, norm=norm)
    _run(c)


@pytest.mark.parametrize("batch", [1, 3, 64, 700])
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("fp8", 64), ("f32", 0)])
def test_steps(batch, dtype, page):
    say("rope step", batch, dtype, page)
    _run(Case(dtype, 16, 4, 128, page, lens=[1 + 7 * b % 50 for b in range(batch)]))


def test_step_skips_an_empty_sequence():
    _run(Case("bf16", 8, 2, 64, 16, lens=(4, 0, 9)))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_long_chunk_many_waves_per_part(dtype):
    """Enough tokens that a wave takes all heads of a token, and a token count that is no multiple of anything."""
    _run(Case(dtype, 32, 8, 128, 16, lens=(3001, 2000), new=(3001, 777)))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_more_than_the_caches_hold(dtype):
    """Over 256 MB written: the same values as for each part of the tokens alone."""
    n, hq, hkv = 17000, 64, 8
    a = Case(dtype, hq, hkv, 128, 0, lens=(n,), new=(n,))
    whole = a.call()[:n].clone()
    k, v = a.k.clone(), a.v.clone()
    a.k.fill_(3)
    a.v.fill_(3)
    for first in range(0, n, 4096):
        last = min(first + 4096, n)
        part = a.op.rope_append(a.q[first:last], a.new_k[first:last], a.new_v[first:last], a.k, a.v, a.seq_start,
                                torch.tensor([last], dtype=torch.int32, device=DEV), n, a.cos_sin, a.q_weight, a.k_weight,
                                a.eps, torch.zeros(1, dtype=torch.int64, device=DEV),
                                torch.tensor([last - first], dtype=torch.int32, device=DEV), last - first)
        assert torch.equal(part, whole[first:last])
    assert torch.equal(a.k[:n], k[:n]) and torch.equal(a.v[:n], v[:n])


def test_positions_and_their_bounds():
    c = Case("bf16", 8, 2, 64, 16, lens=(30, 12), new=(30, 5), positions=lambda r: (r * 7919) % 41 - 2, table_rows=33)
    _run(c)


def test_positions_of_single_tokens():
    _run(Case("bf16", 8, 2, 128, 16, lens=(30, 12, 5), positions=lambda r: 20 + r, table_rows=64))


def test_fused_and_separate_inputs_agree():
    a, b = (Case("fp8", 8, 2, 128, 16, lens=(30, 12), new=(9, 12), fused=f) for f in (True, False))
    qa, qb = _run(a), _run(b)
    assert torch.equal(qa.view(torch.uint8), qb.view(torch.uint8))
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)


def test_step_equals_chunk_of_one():
    a = Case("bf16", 32, 8, 128, 16, lens=[11 * b + 1 for b in range(9)])
    b = Case("bf16", 32, 8, 128, 16, lens=[11 * b + 1 for b in range(9)])
    qa, qb = a.call(), b.call(q_start=b.q_start, q_lens=b.q_lens, max_q_len=1)
    assert torch.equal(qa, qb) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_queries(dtype):
    c = Case(dtype, 8, 2, 128, 16, lens=(300, 12), new=(290, 12), fused=False)
    want = c.call()
    got = c.call(q_out=c.q)
    assert got is c.q
    rows = [r for r, _, _ in c.tokens()]
    assert torch.equal(got[rows], want[rows])


def test_cache_of_other_strides():
    """K and V interleaved in one buffer, heads padded apart."""
    c = Case("bf16", 8, 4, 64, 0, lens=(20, 31), new=(3, 31))
    wide = torch.zeros((c.k.shape[0], 2, 4, 96), dtype=torch.bfloat16, device=DEV)
    want_k, want_v = c.k.clone(), c.v.clone()
    wide[:, 0, :, :64], wide[:, 1, :, :64] = c.k, c.v
    c.call()
    dense_k, dense_v = c.k.clone(), c.v.clone()
    c.k, c.v = wide[:, 0, :, :64], wide[:, 1, :, :64]
    c.call()
    assert torch.equal(c.k, dense_k) and torch.equal(c.v, dense_v) and not torch.equal(dense_k, want_k)
    assert not torch.equal(dense_v, want_v) and float(wide[..., 64:].abs().max()) == 0


def test_head_major_cache():
    c = Case("bf16", 8, 4, 64, 0, lens=(20, 31), new=(20, 1))
    k, v = c.k.clone(), c.v.clone()
    c.call()
    want_k, want_v = c.k.clone(), c.v.clone()
    c.k, c.v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (k, v))
    c.call()
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v)


def test_sequences_outside_the_contract_are_skipped():
    c = Case("bf16", 8, 2, 128, 16, lens=(30, 12, 25, 8, 16), new=(3, 2, 4, 5, 6))
    good = c.call().clone()
    ref_k = c.k.clone()
    for b, (ctx, m) in {0: (31, 3), 1: (-1, 2), 2: (25, 26), 3: (8, -1)}.items():
        c.ctx[b], c.q_lens[b] = ctx, m
    c2 = Case("bf16", 8, 2, 128, 16, lens=(30, 12, 25, 8, 16), new=(3, 2, 4, 5, 6))
    c2.ctx, c2.q_lens = c.ctx, c.q_lens
    q_out = torch.full_like(good, 7.0)
    before = c2.k.clone()
    c2.call(q_out=q_out, max_q_len=27)
    first = c2.starts[4]
    assert torch.equal(q_out[first:first + 6], good[first:first + 6])
    assert bool((q_out[:first] == 7).all()) and bool((q_out[first + 6:] == 7).all())
    flat, want, old = (t.view(-1, 2, 128) for t in (c2.k, ref_k, before))
    slots = [s for _, s, _ in c2.tokens()[-6:]]
    rest = np.setdiff1d(np.arange(flat.shape[0]), slots)
    assert torch.equal(flat[slots], want[slots]) and torch.equal(flat[rest], old[rest])


@pytest.mark.parametrize("bad", [-1, 1000])
def test_token_without_a_page_is_not_stored(bad):
    c = Case("fp8", 8, 2, 128, 16, lens=(40, 20), new=(40, 20))
    want = c.call().clone()
    fresh = Case("fp8", 8, 2, 128, 16, lens=(40, 20), new=(40, 20))
    lost = int(fresh.table[0, 1])
    before = fresh.k[lost].clone(), fresh.v[lost].clone()
    fresh.block_table[0, 1] = bad
    got = fresh.call()
    rows = [r for r, _, _ in c.tokens()]
    assert torch.equal(got[rows], want[rows])
    assert torch.equal(fresh.k[lost], before[0]) and torch.equal(fresh.v[lost], before[1])
    keep = [p for p in range(c.k.shape[0]) if p != lost]
    assert torch.equal(fresh.k[keep], c.k[keep]) and torch.equal(fresh.v[keep], c.v[keep])


def test_fp8_codes_of_large_values_and_nan():
    c = Case("fp8", 2, 2, 64, 16, lens=(8,), new=(8,), norm=(False, False), rot=0)
    values = torch.tensor([0.0, 448.0, 449.0, 464.0, 465.0, 1e6, float("inf"), float("nan")]) * VS
    for t in range(8):
        c.new_v[t] = values[t]
        c.new_v[t, 0, ::2] = -values[t]
    c.call()
    got = c.v.view(-1, 2, 64).view(torch.float8_e4m3fn).float()[[s for _, s, _ in c.tokens()]].cpu()
    want = [0, 448, 448, 448, 448, 448, 448]
    for t, w in enumerate(want):
        assert bool((got[t].abs() == w).all()) and (w == 0 or bool((got[t, 0, ::2] == -w).all()))
    assert bool(torch.isnan(got[7]).all())


def test_nan_and_infinity_stay_in_their_head():
    c = Case("bf16", 4, 2, 64, 16, lens=(6,), new=(6,))
    clean = c.call().clone()
    c.q[2, 1, 5] = float("nan")
    c.q[4, 3, 9] = float("inf")
    got = c.call()
    assert bool(torch.isnan(got[2, 1]).all())
    assert bool((~torch.isfinite(got[4, 3])).any())
    mask = torch.ones((got.shape[0], 4), dtype=torch.bool)
    mask[2, 1] = mask[4, 3] = False
    mask[6:] = False
    assert torch.equal(got[mask.to(DEV)], clean[mask.to(DEV)])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d,rot", [("bf16", 128, 32), ("bf16", 64, 16), ("f32", 128, 80), ("bf16", 128, 0)])
def test_infinity_beside_the_rotation_stays_in_its_place(dtype, d, rot, interleaved):
    """An element that is not rotated meets no other one: an infinity or a NaN there is passed on alone."""
    c = Case(dtype=dtype, d=d, lens=(40,), new=[9], rot=rot, norm=(False, False), interleaved=interleaved, page=0)
    clean = c.call()
    k = c.k.clone()
    for at, x in ((rot, float("inf")), (rot + 3, float("nan")), (d - 1, float("-inf"))):
        c.q[:, :, at] = x
        c.new_k[:, :, at] = x
        clean[:9, :, at] = x
        k[[s for _, s, _ in c.tokens()], :, at] = x
    got = c.call()
    for out, want in ((got[:9], clean[:9]), (c.k, k)):
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(1.0), want.nan_to_num(1.0))


def test_zero_rows_and_zero_heads():
    """A head of zeros stays zero (eps > 0)."""
    c = Case("f32", 4, 2, 64, 0, lens=(6,), new=(6,))
    c.qkv.zero_()
    assert float(c.call()[:6].abs().max()) == 0 and float(c.k.view(-1, 2, 64)[:6].abs().max()) == 0


def test_other_stream_and_its_memory():
    c = Case("bf16", 32, 8, 128, 16, lens=(500, 40), new=(500, 40))
    want = c.call().clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = c.call(stream=side)
    side.synchronize()
    rows = [r for r, _, _ in c.tokens()]
    assert torch.equal(got[rows], want[rows])


def test_captured_step():
    c = Case("bf16", 32, 8, 128, 16, lens=[30 + b for b in range(6)])
    q_out = c.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(q_out=q_out)
    for i in range(3):
        c.qkv.copy_(torch.randn(c.qkv.shape, generator=torch.Generator().manual_seed(i)).to(c.qkv.dtype))
        want, want_k = c.call().clone(), c.k.clone()
        q_out.zero_()
        c.k.view(-1, 8, 128)[[s for _, s, _ in c.tokens()]] = 0
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want) and torch.equal(c.k, want_k)


def test_page_offsets_past_4_gib():
    """One token in the last page of a pool of 4.5 GB."""
    from paper_2605_30842_amd.binding import DecodeAttention

    pages = 540  # of 4096 tokens, 8 MB each
    k = torch.zeros((pages, 4096, 8, 128), dtype=torch.bfloat16, device=DEV)
    op = DecodeAttention(8, 8, 128, "bf16", 0.1, 1, 4096)
    x = torch.randn((3, 1, 8, 128), device=DEV).to(torch.bfloat16)
    v = k  # K then V of the token go to one pool: V stays
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV)
    ctx = torch.tensor([4096], dtype=torch.int32, device=DEV)
    angles = torch.cat([torch.ones(4096, 64), torch.zeros(4096, 64)], 1).to(DEV)
    k2 = torch.zeros_like(k)
    op.rope_append_paged(x[0], x[1], x[2], k, k2, table, ctx, 4096, angles)
    assert torch.equal(k[pages - 1, 4095], x[1, 0]) and torch.equal(k2[pages - 1, 4095], x[2, 0])
    assert int(torch.count_nonzero(v)) == int(torch.count_nonzero(x[1]))
