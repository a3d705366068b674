"""Streams that are not torch's objects: anything with a cuda_stream, as the attention calls take it."""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Handle:
    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


def test_page_calls_and_rotation():
    from paper_2605_30842_amd.binding import DecodeAttention, KVPages

    say("stream objects")
    i32 = dict(dtype=torch.int32, device=DEV)
    op = DecodeAttention(2, 1, 64, "bf16", 0.1, 2, 64)
    k = torch.zeros((8, 16, 1, 64), dtype=torch.bfloat16, device=DEV)
    v, table, ctx = torch.zeros_like(k), torch.full((2, 4), -1, **i32), torch.zeros(2, **i32)
    p = KVPages(op, k, v, table, ctx, torch.zeros(8, **i32), 64)
    add, none, pair = torch.tensor([20, 0], **i32), torch.zeros(0, **i32), (torch.zeros(1, **i32), torch.ones(1, **i32))
    keep, start = torch.arange(7, **i32), torch.zeros(1, dtype=torch.int64, device=DEV)
    granted = torch.full((2,), 9, **i32)
    missing = [torch.full((), 9, **i32) for _ in range(5)]
    x = torch.randn((2, 4, 64), device=DEV).to(torch.bfloat16)
    angles = torch.zeros((1, 0), device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s = Handle(side)
    p.reserve(add, missing=missing[0], granted=granted, stream=s)
    p.fork(*pair, missing=missing[1], stream=s)
    p.fork(none, none, missing=missing[2], stream=s)
    p.compact(pair[1], keep, start, torch.tensor([7], **i32), missing=missing[3], stream=s)
    p.compact(none, none, none.long(), none, missing=missing[4], stream=s)
    q = op.rope_append_paged(x[:, :2], x[:, 2:3], x[:, 3:], k, v, table, ctx, 64, angles, stream=s)
    side.synchronize()
    assert [int(m) for m in missing] == [0] * 5 and granted.tolist() == [20, 0] and ctx.tolist() == [20, 7]
    assert torch.equal(q, x[:, :2]) and torch.equal(v[table[1, 0].long(), 6], x[1, 3:])
    p.release(pair[1], stream=s)
    side.synchronize()
    assert ctx.tolist() == [20, 0]
