"""Integers that the library's arguments do not hold are refused, not taken modulo 2^32 or 2^64 (no device)."""

import numpy as np
import pytest
import torch

from paper_2605_30842_amd import binding as B

BF, I32, I64 = torch.bfloat16, torch.int32, torch.int64
W = 1 << 32


@pytest.fixture
def op():
    o = object.__new__(B.DecodeAttention)
    o.plan, _ = B.comem_decode_attn_init(B.Config(num_q_heads=8, num_kv_heads=2, head_dim=64, dtype=B.BF16, scale=0.1,
                                                  max_batch=4, max_ctx_len=64), B.NO_DEVICE)
    o.dtype, o.device = "bf16", 0
    o.num_q_heads, o.num_kv_heads, o.head_dim = 8, 2, 64
    o._torch_device = torch.device("cpu")
    o._q_dtypes, o._kv_dtypes = B._torch_dtypes("bf16")
    o._stream = lambda s: 0
    o.workspace, o.workspace_bytes = torch.zeros(512, dtype=torch.uint8)[:256], 0
    return o


def calls(op):
    """Every call with host integers: (function, its integers that the plan takes)."""
    q, lse = torch.zeros(3, 8, 64, dtype=BF), torch.zeros(3, 8)
    k, pool = torch.zeros(40, 2, 64, dtype=BF), torch.zeros(9, 16, 2, 64, dtype=BF)
    start, lens, table = torch.zeros(3, dtype=I64), torch.zeros(3, dtype=I32), torch.zeros(3, 4, dtype=I32)
    ends = torch.zeros(9, 2, 2, 64, dtype=BF)
    new, cos = torch.zeros(3, 2, 64, dtype=BF), torch.zeros(64, 64)
    return {
        "attn_weights": (lambda **n: op.attn_weights(q, lse, k, start, lens, q_start=start, q_lens=lens, **n),
                         dict(max_ctx_len=20, max_q_len=2)),
        "attn_weights_paged": (lambda **n: op.attn_weights_paged(q, lse, pool, table, lens, q_start=start, q_lens=lens, **n),
                               dict(max_ctx_len=20, max_q_len=2)),
        "keep_tokens": (lambda **n: op.keep_tokens(torch.zeros(3, 32), lens, **n),
                        dict(max_ctx_len=20, budget=8, first=1, last=2)),
        "block_bounds": (lambda **n: op.block_bounds(pool, table, lens, bounds=ends, q_lens=lens, **n),
                         dict(max_ctx_len=64, max_q_len=2)),
        "block_scores": (lambda **n: op.block_scores(q, ends, block_table=table, ctx_lens=lens, **n),
                         dict(page_size=16, max_ctx_len=64)),
        "block_select": (lambda **n: op.block_select(torch.zeros(3, 2, 4), block_table=table, ctx_lens=lens, **n),
                         dict(page_size=16, max_ctx_len=64, budget=3, first=1, last=1)),
        "block_forward": (lambda **n: op.block_forward(q, pool, pool, torch.zeros(3, 2, 4, dtype=I32), lens, **n),
                          dict(max_len=64)),
        "prefill": (lambda **n: op.prefill(q, start, lens, k=k, v=k, seq_start=start, ctx_lens=lens, **n),
                    dict(max_q_len=2, max_ctx_len=20)),
        "rope_append": (lambda **n: op.rope_append(q, new, new, k, k.clone(), start, lens, cos_sin=cos, q_start=start,
                                                   q_lens=lens, **n), dict(max_ctx_len=20, max_q_len=2)),
    }


NAMES = ["attn_weights", "attn_weights_paged", "keep_tokens", "block_bounds", "block_scores", "block_select",
         "block_forward", "prefill", "rope_append"]


@pytest.mark.parametrize("name", NAMES)
def test_what_an_argument_does_not_hold_is_refused(op, name):
    call, good = calls(op)[name]
    for kind in (int, np.int64, np.int32):  # reaches the library, which has no device
        with pytest.raises(B.ComemError):
            call(**{k: kind(v) for k, v in good.items()})
    for k, v in good.items():
        period = W * W if k in ("max_ctx_len", "max_len") else W
        for bad in (v + period, v - period, period // 2, -period // 2 - 1):
            with pytest.raises(ValueError):
                call(**dict(good, **{k: bad}))
    if name not in ("block_bounds", "block_forward", "prefill", "rope_append"):
        k = "budget" if "budget" in good else "max_ctx_len"
        with pytest.raises(ValueError):  # a dimension of the results
            call(**dict(good, **{k: -64}))
