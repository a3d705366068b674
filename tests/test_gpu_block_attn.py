"""Block bounds, scores, selection and attention over selected blocks (comem_block_attn.h) against their 64-bit forms."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.context_util import (KS, VS, Context, chosen, drawn, ends_of, patterns, query_dtype, reach, wide)  # noqa: E402
from tests.gpu_util import check, say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def make_op(dtype, hq, hkv, d, batch, bound, **kw):
    from paper_2605_30842_amd.binding import DecodeAttention

    scales = dict(k_scale=KS, v_scale=VS) if dtype == "fp8" else {}
    return DecodeAttention(hq, hkv, d, dtype, 1.0 / math.sqrt(d), batch, bound, **scales, **kw)


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


# ------------------------------------------------------------ bounds


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("hkv,d,page", [(8, 128, 64), (2, 64, 16), (1, 64, 1), (3, 128, 32), (40, 128, 8), (5, 64, 128),
                                        (1, 128, 512)])
@pytest.mark.parametrize("layout", ["dense", "fused", "heads"])
def test_bounds(dtype, hkv, d, page, layout):
    """Every bit pattern there is, in pages that the new tokens reach; the other pages stay."""
    say("bounds", dtype, hkv, d, page, layout)
    g = torch.Generator().manual_seed(page + hkv)
    lens = [1, page, page + 1, 3 * page - 1, 0, 2 * page]
    new = [1, 1, 2, 2 * page, 0, 2 * page]
    c = Context(lens, dtype, hkv, d, page, g, layout=layout)
    for b, n in enumerate(lens):
        if n:
            at = c.at[b]
            raw = torch.randint(0, 256, (n, hkv, d, c.k.element_size()), generator=g, dtype=torch.uint8)
            x = raw.view(c.k.dtype)[..., 0] if c.k.dtype != torch.uint8 else raw[..., 0]
            c.k[at // page, at % page] = x
    x = c.to(DEV)
    op = make_op(dtype, hkv, hkv, d, len(lens), max(lens))
    ends = drawn((c.k.shape[0], hkv, 2, d), dtype, g).to(DEV)
    before = ends.clone()
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], max(lens), ends, q_lens=ints(new), max_q_len=max(new))
    torch.cuda.synchronize()
    want = patterns(before.cpu())[0]
    for b, (n, m) in enumerate(zip(lens, new)):
        for i in range((n - m) // page, -(-n // page)) if m else ():
            p = int(c.table[b, i])
            want[p] = ends_of(c.k[p, :min(page, n - i * page)])
    assert torch.equal(patterns(ends.cpu())[0], want)
    # One token each: the last page alone.
    ends = before.clone()
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], max(lens), ends)
    want = patterns(before.cpu())[0]
    for b, n in enumerate(lens):
        if n:
            p = int(c.table[b, (n - 1) // page])
            want[p] = ends_of(c.k[p, :(n - 1) % page + 1])
    assert torch.equal(patterns(ends.cpu())[0], want)


def test_bounds_leave_out_what_is_outside():
    g = torch.Generator().manual_seed(2)
    c = Context([40, 40, 40, 40, 40], "bf16", 2, 64, 16, g)
    x, op = c.to(DEV), make_op("bf16", 2, 2, 64, 5, 40)
    table = x["block_table"].clone()
    table[4, 1], table[4, 0] = -1, x["k"].shape[0]
    ends = torch.zeros((x["k"].shape[0], 2, 2, 64), dtype=torch.bfloat16, device=DEV)
    op.block_bounds(x["k"], table, ints([41, -1, 40, 3, 40]), 40, ends, q_lens=ints([1, 1, 41, 4, 40]), max_q_len=40)
    torch.cuda.synchronize()
    want = torch.zeros(ends.shape, dtype=torch.int64)
    p = int(c.table[4, 2])
    want[p] = ends_of(c.k[p, :8])
    assert torch.equal(patterns(ends.cpu())[0], want)
    ends.zero_()
    op.block_bounds(x["k"], table, ints([40] * 5), 40, ends, q_lens=ints([3, 2, 0, 9, 0]), max_q_len=2)
    torch.cuda.synchronize()
    p = int(c.table[1, 2])
    want.zero_()
    want[p] = ends_of(c.k[p, :8])
    assert torch.equal(patterns(ends.cpu())[0], want)


# ------------------------------------------------------------ scores


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("hkv,group,d,page", [(8, 4, 128, 64), (2, 8, 64, 16), (1, 1, 128, 1), (3, 16, 64, 4), (5, 2, 128, 256)])
def test_scores(dtype, hkv, group, d, page):
    """The bound's value, within the float32 sums of 2 D products; and a bound it is."""
    say("scores", dtype, hkv, group, d, page)
    g = torch.Generator().manual_seed(page)
    lens = [0, 1, page, page + 1, 15 * page, 16 * page + 1, 33 * page]
    c = Context(lens, dtype, hkv, d, page, g)
    x, op = c.to(DEV), make_op(dtype, hkv * group, hkv, d, len(lens), max(lens))
    q = torch.randn((len(lens), hkv * group, d), generator=g).to(query_dtype(dtype))
    ends = drawn((c.k.shape[0], hkv, 2, d), dtype, g).to(DEV)
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], max(lens), ends, q_lens=x["ctx_lens"], max_q_len=max(lens))
    blocks = -(-max(lens) // page)
    scores = torch.full((len(lens), hkv, blocks), -7.0, device=DEV)
    op.block_scores(q.to(DEV), ends, page, x["block_table"], x["ctx_lens"], max(lens), scores=scores)
    torch.cuda.synchronize()
    scale = float(np.float32(1.0 / math.sqrt(d)))
    got, wide_ends = scores.cpu().double(), wide(ends, dtype)
    for b, n in enumerate(lens):
        nb = -(-n // page)
        assert bool((got[b, :, nb:] == -7.0).all())
        if not n:
            continue
        k = c.keys(b)
        for h in range(hkv):
            qh = q[b, h * group:(h + 1) * group].double()
            want, size = reach(qh, wide_ends[c.table[b, :nb].long(), h], scale)
            off = 2 * d * 2.0 ** -23 * size + 2.0 ** -22 * want.abs()
            assert bool(((got[b, h, :nb] - want).abs() <= off).all()), (b, h)
            top = scale * (qh @ k[:, h].T).max(0).values
            each = torch.nn.functional.pad(top, (0, nb * page - n), value=-math.inf).view(nb, page).max(1).values
            assert bool((got[b, h, :nb] >= each - off).all()), (b, h)


def test_scores_of_special_values():
    """NaN in a query or a bound, and infinities that a query's sign meets; no sequence but theirs is touched."""
    g = torch.Generator().manual_seed(5)
    hkv, d, page = 2, 64, 16
    c = Context([64, 64, 64], "bf16", hkv, d, page, g)
    x, op = c.to(DEV), make_op("bf16", 4, hkv, d, 3, 64)
    q = torch.randn((3, 4, d), generator=g).to(torch.bfloat16)
    q[q == 0] = 1.0
    ends = torch.zeros((c.k.shape[0], hkv, 2, d), dtype=torch.bfloat16, device=DEV)
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], 64, ends, q_lens=x["ctx_lens"], max_q_len=64)
    plain = op.block_scores(q.to(DEV), ends, page, x["block_table"], x["ctx_lens"], 64).cpu()
    table = c.table.long()
    ends[table[0, 1], 1, 0, 7] = float("nan")
    ends[table[0, 2], 0, 1, 9] = -float("nan")
    bad = q.clone()
    bad[1, 2, 5] = float("nan")
    got = op.block_scores(bad.to(DEV), ends, page, x["block_table"], x["ctx_lens"], 64).cpu()
    nan = torch.zeros(got.shape, dtype=torch.bool)
    nan[0, 1, 1] = nan[0, 0, 2] = True
    nan[1, 1, :] = True
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], plain[~nan])
    # Entries outside the pool are read as page 0's.
    ends[0] = ends[table[2, 3]]
    outside = c.table.clone()
    outside[2] = torch.tensor([-1, c.k.shape[0], 2 ** 31 - 1, 0])
    got = op.block_scores(q.to(DEV), ends, page, outside.to(DEV), x["ctx_lens"], 64).cpu()
    assert torch.equal(got[2], plain[2, :, 3:].expand(hkv, 4))


def test_scores_lengths_are_clamped():
    g = torch.Generator().manual_seed(6)
    c = Context([64, 64, 64], "bf16", 2, 64, 16, g)
    x, op = c.to(DEV), make_op("bf16", 4, 2, 64, 3, 64)
    ends = drawn((c.k.shape[0], 2, 2, 64), "bf16", g).to(DEV)
    q = torch.randn((3, 4, 64), generator=g).to(torch.bfloat16).to(DEV)
    want = op.block_scores(q, ends, 16, x["block_table"], x["ctx_lens"], 64)
    got = torch.full((3, 2, 4), -7.0, device=DEV)
    op.block_scores(q, ends, 16, x["block_table"], ints([2 ** 31 - 1, -5, 64]), 64, scores=got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and bool((got[1] == -7.0).all())


# ------------------------------------------------------------ selection


def check_select(scores, table, lens, page, bound, budget, first, last):
    batch, hkv, _ = scores.shape
    op = make_op("f32", hkv, hkv, 64, batch, max(bound, 1))
    out = torch.full((batch, hkv, budget), -5, dtype=torch.int32, device=DEV)
    got, count = op.block_select(scores.to(DEV), page, table.to(DEV), ints(lens), bound, budget, first, last, table=out)
    torch.cuda.synchronize()
    assert got is out
    got = got.cpu()
    for b, n in enumerate(lens):
        n = min(max(n, 0), bound)
        nb = -(-n // page)
        k = min(nb, budget)
        assert int(count[b]) == (0 if n == 0 else (k - 1) * page + n - (nb - 1) * page)
        for h in range(hkv):
            want = chosen(scores[b, h, :nb].numpy(), k, first, last)
            assert got[b, h, :k].tolist() == table[b, want].tolist(), (b, h)
            assert bool((got[b, h, k:] == -5).all())


@pytest.mark.parametrize("page,budget,first,last", [(16, 1, 0, 1), (16, 7, 1, 2), (1, 40, 3, 5), (64, 300, 1, 1), (8, 20, 0, 20)])
def test_select(page, budget, first, last):
    g = torch.Generator().manual_seed(budget)
    lens = [0, 1, page, page + 1, 5 * page - 1, 64 * page, 257 * page, 300 * page - 3, 10 ** 6, -1]
    bound = 300 * page
    blocks = -(-bound // page)
    scores = torch.randn((len(lens), 3, blocks), generator=g)
    scores[:, 1] = scores[:, 1].round()
    scores[:, 2, ::5] = float("nan")
    table = torch.randint(-3, 10 ** 6, (len(lens), blocks + 2), generator=g, dtype=torch.int32)
    check_select(scores, table, lens, page, bound, budget, first, last)


@pytest.mark.parametrize("blocks", [2047, 2048, 2049, 33000])
def test_select_many_blocks(blocks):
    g = torch.Generator().manual_seed(blocks)
    scores = torch.randn((2, 2, blocks), generator=g)
    scores[1] = scores[1].round()
    table = torch.randperm(2 * blocks, generator=g).view(2, blocks).to(torch.int32)
    check_select(scores, table, [blocks * 4, blocks * 4 - 5], 4, blocks * 4, 600, 2, 3)


# ------------------------------------------------------------ attention


def attended(c, b, q, pages, tokens, scale):
    """out, lse of sequence b's queries [hq, d] over the first `tokens` of each KV head's pages."""
    group = q.shape[0] // c.hkv
    out, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    for j in range(q.shape[0]) if tokens else ():
        h = j // group
        rows = lambda t: wide(t[pages[h].long(), :, h].flatten(0, 1)[:tokens], c.dtype)  # noqa: E731
        s = scale * (rows(c.k) @ q[j].double())
        lse[j] = torch.logsumexp(s, 0)
        out[j] = torch.softmax(s, 0) @ rows(c.v)
    return out.numpy(), lse.numpy()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("hkv,group,d,page", [(8, 4, 128, 64), (2, 8, 64, 16), (3, 1, 128, 1), (4, 16, 64, 4), (2, 2, 128, 32)])
def test_attention_over_blocks(dtype, hkv, group, d, page):
    """Each head its own pages, in any order; lengths that end in a page; an empty sequence."""
    say("block attention", dtype, hkv, group, d, page)
    g = torch.Generator().manual_seed(page + d)
    lens = [900, 5, 333]
    c = Context(lens, dtype, hkv, d, page, g, both=True)
    x, op = c.to(DEV), make_op(dtype, hkv * group, hkv, d, 4, 1024)
    width = -(-200 // page) + 1
    tokens = [200, 5, 0, 97]
    table = torch.full((4, hkv, width), -9, dtype=torch.int32)
    for b, src in ((0, 0), (1, 1), (3, 2)):
        whole = lens[src] // page
        for h in range(hkv):
            n = -(-tokens[b] // page)
            pick = torch.randperm(max(whole, 1), generator=g)[:n]
            table[b, h, :n] = c.table[src][pick]
    q = torch.randn((4, hkv * group, d), generator=g).to(query_dtype(dtype))
    lse = torch.zeros((4, hkv * group), device=DEV)
    out, _ = op.block_forward(q.to(DEV), x["k"], x["v"], table.to(DEV), ints(tokens), 200, lse=lse)
    torch.cuda.synchronize()
    scale = float(np.float32(1.0 / math.sqrt(d)))
    want = [attended(c, b, q[b], [table[b, h, :-(-t // page)] for h in range(hkv)], t, scale) for b, t in enumerate(tokens)]
    check(out.cpu().numpy(), lse.cpu().numpy(), np.stack([w[0] for w in want]), np.stack([w[1] for w in want]), dtype)


def near_decode(got, want, v, exact):
    """The decode call's results: its bits where both take the weights in float32; else within what its weights are off by
    (two bf16 parts, 2^-17 of a weight, so 2^-17 of the largest value; as much again for the float32 sums)."""
    if exact:
        assert torch.equal(got, want)
    else:
        assert float((got - want).abs().max()) <= 2.0 ** -16 * max(1.0, v)


@pytest.mark.parametrize("dtype,variant,chunk", [("bf16", "auto", 0), ("fp8", "auto", 0), ("f32", "auto", 0), ("bf16", "valu", 0),
                                                 ("bf16", "mfma_grid", 0), ("bf16", "mfma", 64)])
@pytest.mark.parametrize("page", [1, 16])
def test_one_table_for_all_heads_is_the_decode_call(dtype, variant, chunk, page):
    """... in every form of the kernels: split, balanced (long calls), queue, vector."""
    g = torch.Generator().manual_seed(7)
    for lens in ([700], [3000, 1, 0, 2500], [4000] * 6 if dtype != "f32" else [400] * 6):
        c = Context(lens, dtype, 2, 64, page, g, both=True)
        x, op = c.to(DEV), make_op(dtype, 8, 2, 64, len(lens), max(lens), variant=variant, chunk_tokens=chunk)
        q = torch.randn((len(lens), 8, 64), generator=g).to(query_dtype(dtype)).to(DEV)
        a, b = (torch.zeros((len(lens), 8), device=DEV) for _ in range(2))
        want, _ = op.forward_paged(q, x["k"], x["v"], x["block_table"], x["ctx_lens"], max(lens), lse=a)
        table = x["block_table"][:, None].expand(-1, 2, -1).contiguous()
        got, _ = op.block_forward(q, x["k"], x["v"], table, x["ctx_lens"], max(lens), lse=b)
        torch.cuda.synchronize()
        near_decode(got, want, 5.0, dtype == "f32" or variant == "valu")
        assert torch.equal(a, b), (lens, variant)
        again, _ = op.block_forward(q, x["k"], x["v"], table, x["ctx_lens"], max(lens))
        assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("page", [4, 64])
def test_the_weights_keep_float32s_precision(dtype, page):
    """Errors against 64 bits stay below 2^-20 of the outputs' norm: weights in three bf16 parts (2^-26), products exact,
    float32 sums of at most 128 products in a row (a few 2^-24 of the norm, at random signs), lse likewise."""
    g = torch.Generator().manual_seed(3)
    c = Context([4096, 1000], dtype, 2, 128, page, g, both=True)
    x, op = c.to(DEV), make_op(dtype, 8, 2, 128, 2, 4096)
    q = torch.randn((2, 8, 128), generator=g).to(query_dtype(dtype))
    table = x["block_table"][:, None].expand(-1, 2, -1).contiguous()
    got, _ = op.block_forward(q.to(DEV), x["k"], x["v"], table, x["ctx_lens"], 4096)
    scale = float(np.float32(1.0 / math.sqrt(128)))
    for b, n in enumerate([4096, 1000]):
        want, _ = attended(c, b, q[b], [c.table[b, :-(-n // page)]] * 2, n, scale)
        off = np.linalg.norm(got[b].cpu().double().numpy() - want) / np.linalg.norm(want)
        assert off <= 2.0 ** -20, off


def test_heads_tables_are_their_own():
    """A head's result is that of a call with its table for all heads, whatever the other heads' say; bad entries read
    page 0 and are reported."""
    g = torch.Generator().manual_seed(8)
    c = Context([640, 500], "bf16", 4, 64, 16, g, both=True)
    x, op = c.to(DEV), make_op("bf16", 16, 4, 64, 2, 640, debug_checks=True)
    x["k"][0], x["v"][0] = 0.25, 0.5
    q = torch.randn((2, 16, 64), generator=g).to(torch.bfloat16).to(DEV)
    lens = ints([150, 90])
    table = torch.stack([torch.stack([c.table[b, torch.randperm(30, generator=g)[:10]] for _ in range(4)]) for b in range(2)])
    got, _ = op.block_forward(q, x["k"], x["v"], table.to(DEV), lens, 160)
    for h in range(4):
        one, _ = op.block_forward(q, x["k"], x["v"], table[:, h:h + 1].expand(-1, 4, -1).contiguous().to(DEV), lens, 160)
        assert torch.equal(got[:, 4 * h:4 * h + 4], one[:, 4 * h:4 * h + 4]), h
    assert op.device_errors() == 0
    bad = table.clone()
    bad[1, 2, 3] = 10 ** 6
    out, _ = op.block_forward(q, x["k"], x["v"], bad.to(DEV), lens, 160)
    assert op.device_errors() == 2
    bad[1, 2, 3] = 0
    zero, _ = op.block_forward(q, x["k"], x["v"], bad.to(DEV), lens, 160)
    assert torch.equal(out, zero)
    keep = [i for i in range(16) if i // 4 != 2]
    assert torch.equal(out[0], got[0]) and torch.equal(out[1, keep], got[1, keep])


def test_all_blocks_selected_is_dense_attention():
    """With a budget for every block the step is the dense one."""
    g = torch.Generator().manual_seed(9)
    lens = [1000, 16, 333]
    c = Context(lens, "bf16", 2, 128, 16, g, both=True)
    x, op = c.to(DEV), make_op("bf16", 8, 2, 128, 3, 1000)
    q = torch.randn((3, 8, 128), generator=g).to(torch.bfloat16).to(DEV)
    ends = torch.zeros((c.k.shape[0], 2, 2, 128), dtype=torch.bfloat16, device=DEV)
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], 1000, ends, q_lens=x["ctx_lens"], max_q_len=1000)
    scores = op.block_scores(q, ends, 16, x["block_table"], x["ctx_lens"], 1000)
    table, count = op.block_select(scores, 16, x["block_table"], x["ctx_lens"], 1000, 63)
    assert torch.equal(count, x["ctx_lens"])
    got, _ = op.block_forward(q, x["k"], x["v"], table, count, 1000)
    want, _ = op.forward_paged(q, x["k"], x["v"], x["block_table"], x["ctx_lens"], 1000)
    near_decode(got, want, 5.0, False)


def test_a_needle_is_found():
    """A block with a key near the queries is among the selected, and its value dominates the output."""
    g = torch.Generator().manual_seed(10)
    c = Context([4000], "bf16", 2, 128, 16, g, both=True)
    q = torch.randn((1, 8, 128), generator=g).to(torch.bfloat16)
    at = {0: 1234, 1: 77}
    for h, t in at.items():
        c.k[c.at[0][t] // 16, c.at[0][t] % 16, h] = (q[0, 4 * h].float() * 3).to(torch.bfloat16)
    x, op = c.to(DEV), make_op("bf16", 8, 2, 128, 1, 4000)
    ends = torch.zeros((c.k.shape[0], 2, 2, 128), dtype=torch.bfloat16, device=DEV)
    op.block_bounds(x["k"], x["block_table"], x["ctx_lens"], 4000, ends, q_lens=x["ctx_lens"], max_q_len=4000)
    scores = op.block_scores(q.to(DEV), ends, 16, x["block_table"], x["ctx_lens"], 4000)
    table, count = op.block_select(scores, 16, x["block_table"], x["ctx_lens"], 4000, 12)
    got, _ = op.block_forward(q.to(DEV), x["k"], x["v"], table, count, 12 * 16)
    for h, t in at.items():
        assert int(c.table[0, t // 16]) in table[0, h].tolist()
        v = c.v[c.at[0][t] // 16, c.at[0][t] % 16, h].double()
        # s = 3 |q|^2 / sqrt(D), about 34 above the rest: what 192 others weigh is below 1e-8.
        assert float((got[0, 4 * h].cpu().double() - v).abs().max()) < 1e-4


def test_the_chain_captured():
    """Bounds, scores, selection and attention of a step in one graph, replayed as the context grows."""
    g = torch.Generator().manual_seed(11)
    lens, page, bound = [500, 37], 16, 600
    c = Context([600, 600], "bf16", 2, 64, page, g, both=True)
    x, op = c.to(DEV), make_op("bf16", 8, 2, 64, 2, bound)
    q = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device=DEV)
    ctx, out = ints(lens), torch.zeros((2, 8, 64), device=DEV)

    def all_bounds():
        e = torch.zeros((c.k.shape[0], 2, 2, 64), dtype=torch.bfloat16, device=DEV)
        return op.block_bounds(x["k"], x["block_table"], ctx, bound, e, q_lens=ctx, max_q_len=bound)

    ends = all_bounds()

    def step(ends, out):
        op.block_bounds(x["k"], x["block_table"], ctx, bound, ends)
        s = op.block_scores(q, ends, page, x["block_table"], ctx, bound)
        table, count = op.block_select(s, page, x["block_table"], ctx, bound, 6, 1, 2)
        return op.block_forward(q, x["k"], x["v"], table, count, 6 * page, out=out)[0]

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ends, out)
    for i in range(20):
        ctx.add_(1)
        q.copy_(torch.randn(q.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = step(all_bounds(), torch.zeros_like(out))
        assert torch.equal(out, want), i
