"""Outputs that the wrapper makes for a call on another stream: read on the caller's own stream and dropped there, their
memory must not be handed to the next call before the reading is done."""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, HKV, D, L, M = 8, 2, 128, 600, 300


def _setup(dtype):
    from paper_2605_30842_amd.binding import DecodeAttention

    g = torch.Generator().manual_seed(1)
    op = DecodeAttention(HQ, HKV, D, dtype, 0.09, 1, L)
    q = torch.randn((M, HQ, D), generator=g).to(torch.bfloat16).to(DEV)
    k, v = (torch.randint(0, 90, (L, HKV, D), generator=g).to(torch.uint8 if dtype == "fp8" else torch.bfloat16).to(DEV)
            for _ in range(2))
    i64, i32 = dict(dtype=torch.int64, device=DEV), dict(dtype=torch.int32, device=DEV)
    start, lens, ctx = torch.zeros(1, **i64), torch.tensor([M], **i32), torch.tensor([L], **i32)
    new = torch.randn((2, M, HKV, D), generator=g).to(torch.bfloat16).to(DEV)
    angles = torch.randn((L, 64), generator=g).to(DEV)

    def prefill(stream=None):
        return op.prefill(q, start, lens, M, k, v, start, ctx, L, stream=stream)[0]

    def rope(stream=None):
        return op.rope_append(q, new[0], new[1], k.clone(), v.clone(), start, ctx, L, angles, q_start=start, q_lens=lens,
                              max_q_len=M, stream=stream)

    return prefill, rope


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("which", [0, 1], ids=["prefill", "rope"])
def test_a_result_read_on_the_callers_stream_may_be_dropped(dtype, which):
    say("output memory", dtype, which)
    call = _setup(dtype)[which]
    want = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = torch.randn((8192, 8192), device=DEV).to(torch.bfloat16)
    out = call(side)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(60):  # tens of milliseconds, so that the reading is still to come
        b = a @ a
    read = torch.empty_like(out)
    read.copy_(out)
    done = torch.cuda.Event()
    done.record()
    was = out.data_ptr()
    del out
    again = call(side)
    assert not done.query()
    assert again.data_ptr() != was
    torch.cuda.synchronize()
    assert torch.equal(read, want) and torch.equal(again, want) and bool(torch.isfinite(b).all())
    del again
    torch.cuda.synchronize()
    last = call(side)  # and now it may be taken again
    side.synchronize()
    assert torch.equal(last, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_captured_on_a_second_stream(dtype):
    """An output made, read and dropped inside a capture, the call on a stream that joins it."""
    prefill, _ = _setup(dtype)
    want = prefill()
    side, res = torch.cuda.Stream(), torch.zeros_like(want)
    prefill(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            side.wait_stream(torch.cuda.current_stream())
            out = prefill(side)
            torch.cuda.current_stream().wait_stream(side)
            res.copy_(out)
            del out
    for _ in range(3):
        res.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, want)
        again = prefill(side)
        side.synchronize()
        assert torch.equal(again, want)
