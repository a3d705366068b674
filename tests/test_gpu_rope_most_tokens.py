"""Rotate-and-store at the most tokens that a call may have: 2^26 - 1, one workgroup for every four."""

import pytest

torch = pytest.importorskip("torch")

from tests.gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST = (1 << 26) - 1


def _lists(length, new):
    return dict(seq_start=torch.zeros(1, dtype=torch.int64, device=DEV),
                ctx_lens=torch.tensor([length], dtype=torch.int32, device=DEV),
                q_start=torch.zeros(1, dtype=torch.int64, device=DEV),
                q_lens=torch.tensor([new], dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("bound", [MOST - 3, MOST - 2, MOST])
def test_bound_far_above_the_new_tokens(bound):
    """The bounds on either side of the last whole launch; the sequence has 5 new tokens of 40."""
    from paper_2605_30842_amd.binding import DecodeAttention

    say("rope, max_q_len", bound)
    op = DecodeAttention(4, 2, 64, "bf16", 0.1, 1, 1 << 27)
    x = torch.randn((5, 8, 64), device=DEV).to(torch.bfloat16)
    angles = torch.randn((64, 32), device=DEV)
    got = []
    for most in (5, bound):
        k = torch.zeros((40, 2, 64), dtype=torch.bfloat16, device=DEV)
        v = torch.zeros_like(k)
        q = op.rope_append(x[:, :4], x[:, 4:6], x[:, 6:], k, v, max_ctx_len=bound, cos_sin=angles, max_q_len=most,
                           **_lists(40, 5))
        torch.cuda.synchronize()
        got.append((q, k, v))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(got[0][2][35:], x[:, 6:])


def test_every_token_of_the_longest_call():
    """One head of 64, nothing rotated (34 GB): all zeros are stored over a pattern, and rows around the ends of the
    grid's parts arrive in their places."""
    from paper_2605_30842_amd.binding import DecodeAttention

    say("rope of", MOST, "tokens")
    op = DecodeAttention(1, 1, 64, "bf16", 0.1, 1, MOST)
    shape = (MOST, 1, 64)
    q, new = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rows = torch.tensor([0, 1, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, MOST - 5, MOST - 4, MOST - 3, MOST - 2, MOST - 1],
                        device=DEV)
    q[rows] = torch.rand((len(rows), 1, 64), device=DEV).to(torch.bfloat16) + 1
    new[rows] = q[rows] * 2
    k = torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV)
    v = torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV)
    want = q[rows].clone()
    got = op.rope_append(q, new, new, k, v, max_ctx_len=MOST, cos_sin=torch.zeros((1, 0), device=DEV), max_q_len=MOST,
                         q_out=q, **_lists(MOST, MOST))
    torch.cuda.synchronize()
    assert got is q
    for t, rest in ((q, want), (k, want * 2), (v, want * 2)):
        assert torch.equal(t[rows], rest)
        t[rows] = 0
        assert not bool(t.view(torch.int32).any())
