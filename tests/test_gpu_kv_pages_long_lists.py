"""Forks of more pairs than one workgroup has threads, up to the most that a call may have, on a pool of one chunk."""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("n", [1024, 1025, 4097, 65535])
def test_fork_of_many_pairs(n):
    """Children of a parent of one whole page, and of one of a page and a token; the last pair names the first pair's
    child again and the one before it an empty parent."""
    from paper_2605_30842_amd.binding import DecodeAttention, KVPages

    say("fork of", n)
    i32 = dict(dtype=torch.int32, device=DEV)
    rows = min(n + 2, 65535)
    k = torch.randint(0, 100, (8000, 16, 1, 64), device=DEV).to(torch.uint8)
    v = k + 1
    table, ctx = torch.full((rows, 2), -1, **i32), torch.zeros(rows, **i32)
    counts = torch.zeros(8000, **i32)
    p = KVPages(DecodeAttention(1, 1, 64, "fp8", 0.1, 1, 32), k, v, table, ctx, counts, 32)
    assert int(p.reserve(torch.tensor([16, 17] + [0] * (rows - 2), **i32))) == 0
    children = torch.arange(2, n + 2, **i32)
    parents = torch.zeros(n, **i32)
    parents[::50] = 1
    parents[0], parents[-1], children[-1] = 0, 1, 2
    parents[-2] = n  # the child of the pair before it, empty
    children = children.clamp(max=rows - 1)
    assert int(p.fork(parents, children)) == 0
    torch.cuda.synchronize()
    want_ctx, want = torch.zeros(rows, dtype=torch.int64), torch.full((rows, 2), -1, dtype=torch.int64)
    want_ctx[0], want_ctx[1], want[0, 0], want[1] = 16, 17, 0, torch.tensor([1, 2])
    next_page, held = 3, torch.zeros(8000, dtype=torch.int64)
    par, chi = parents.tolist(), children.tolist()
    seen = set()
    for a, c in zip(par, chi):
        if c in seen or c == a:
            seen.add(c)
            continue
        seen.add(c)
        if a == 0:
            want_ctx[c], want[c, 0] = 16, 0
        elif a == 1:
            want_ctx[c], want[c, 0], want[c, 1] = 17, 1, next_page
            next_page += 1
    for e in want.flatten().tolist():
        if e >= 0:
            held[e] += 1
    assert torch.equal(ctx.cpu().long(), want_ctx) and torch.equal(table.cpu().long(), want)
    assert torch.equal(counts.cpu().long(), held) and next_page < 8000
    for pool in (k, v):
        assert bool((pool[3:next_page, 0] == pool[2, 0]).all())
