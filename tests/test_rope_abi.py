"""comem_rope.h without a GPU: exported symbols, host-side validation, and the wrapper's checks of tensors."""

import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2605_30842_amd import binding as B
from tests.ops_util import rotated

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an aligned address that is never dereferenced


def test_header_and_library():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "comem_rope.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(comem_[a-z_]+)\s*\(", text))) == sorted(B.ROPE_EXPORTED)
    for name in B.ROPE_EXPORTED:
        assert hasattr(B.load_library(), name)


def _plan(**kw):
    cfg = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, dtype=B.BF16, scale=0.088, max_batch=4, max_ctx_len=4096,
               chunk_tokens=0, variant=B.VARIANT_AUTO, k_scale=1.0, v_scale=1.0)
    cfg.update(kw)
    return B.comem_decode_attn_init(B.Config(**cfg), B.NO_DEVICE)[0]


@pytest.fixture
def plan():
    p = _plan()
    yield p
    B.comem_decode_attn_destroy(p)


def _call(plan, paged=False, **kw):
    cfg = dict(q_weight=A, k_weight=A, cos_sin=A, num_positions=4096, rot_dim=128, eps=1e-6, flags=0)
    cfg.update({k: kw.pop(k) for k in list(kw) if k in cfg})
    rope = kw.pop("rope", ctypes.byref(B.RopeConfig(**cfg)))
    a = dict(q=A, q_stride=48 * 128, new_k=A, k_stride=48 * 128, new_v=A, v_stride=48 * 128, q_start=A, q_lens=A,
             max_q_len=64, positions=None, q_out=2 * A, k=A, v=A, stride_token=1024, stride_head=128, ctx_lens=A,
             batch=2, max_ctx_len=4096)
    p = dict(stride_page=16 * 1024, page_size=16, num_pages=100, block_table=A, max_pages=256, seq_start=A)
    for k, val in kw.items():
        (a if k in a else p)[k] = val
    head = (plan, rope, a["q"], a["q_stride"], a["new_k"], a["k_stride"], a["new_v"], a["v_stride"], a["q_start"],
            a["q_lens"], a["max_q_len"], a["positions"], a["q_out"], a["k"], a["v"])
    lib = B.load_library()
    if paged:
        return lib.comem_rope_append_paged(*head, p["stride_page"], a["stride_token"], a["stride_head"], p["page_size"],
                                           p["num_pages"], p["block_table"], p["max_pages"], a["ctx_lens"], a["batch"],
                                           a["max_ctx_len"], None)
    return lib.comem_rope_append(*head, a["stride_token"], a["stride_head"], p["seq_start"], a["ctx_lens"], a["batch"],
                                 a["max_ctx_len"], None)


GOOD = [dict(), dict(positions=A), dict(q_weight=None, k_weight=None), dict(rot_dim=64), dict(flags=1),
        dict(rot_dim=0, cos_sin=None, num_positions=0), dict(q_start=None, q_lens=None, max_q_len=1),
        dict(q_out=A, q_stride=32 * 128), dict(eps=0.0)]


@pytest.mark.parametrize("kw", GOOD, ids=str)
@pytest.mark.parametrize("paged", [False, True])
def test_good_calls_stop_at_the_device(plan, paged, kw):
    assert _call(plan, paged, **kw) == B.ERR_NO_DEVICE


BAD = [
    (dict(rope=None), B.ERR_NULL_POINTER), (dict(q=None), B.ERR_NULL_POINTER), (dict(new_k=None), B.ERR_NULL_POINTER),
    (dict(new_v=None), B.ERR_NULL_POINTER), (dict(q_out=None), B.ERR_NULL_POINTER), (dict(k=None), B.ERR_NULL_POINTER),
    (dict(v=None), B.ERR_NULL_POINTER), (dict(ctx_lens=None), B.ERR_NULL_POINTER),
    (dict(q_start=None), B.ERR_NULL_POINTER), (dict(q_lens=None), B.ERR_NULL_POINTER),
    (dict(cos_sin=None), B.ERR_NULL_POINTER), (dict(q_start=None, q_lens=None), B.ERR_INVALID_SHAPE),
    (dict(num_positions=0), B.ERR_INVALID_SHAPE), (dict(num_positions=1 << 31), B.ERR_INVALID_SHAPE),
    (dict(rot_dim=24), B.ERR_INVALID_SHAPE), (dict(rot_dim=144), B.ERR_INVALID_SHAPE),
    (dict(rot_dim=-16), B.ERR_INVALID_SHAPE), (dict(eps=-1.0), B.ERR_INVALID_SHAPE),
    (dict(eps=float("nan")), B.ERR_INVALID_SHAPE), (dict(flags=2), B.ERR_UNSUPPORTED),
    (dict(batch=-1), B.ERR_INVALID_SHAPE), (dict(batch=5), B.ERR_INVALID_SHAPE),
    (dict(max_ctx_len=4097), B.ERR_INVALID_SHAPE), (dict(max_q_len=-1), B.ERR_INVALID_SHAPE),
    (dict(max_q_len=4097), B.ERR_INVALID_SHAPE), (dict(q_stride=32 * 128 - 8), B.ERR_INVALID_SHAPE),
    (dict(k_stride=8 * 128 - 8), B.ERR_INVALID_SHAPE), (dict(v_stride=0), B.ERR_INVALID_SHAPE),
    (dict(q_out=A), B.ERR_INVALID_SHAPE), (dict(stride_token=0), B.ERR_INVALID_SHAPE),
    (dict(stride_token=1 << 40), B.ERR_INVALID_SHAPE), (dict(stride_head=0), B.ERR_INVALID_SHAPE),
    (dict(q=A + 8), B.ERR_MISALIGNED), (dict(new_k=A + 8), B.ERR_MISALIGNED), (dict(q_out=2 * A + 8), B.ERR_MISALIGNED),
    (dict(cos_sin=A + 4), B.ERR_MISALIGNED), (dict(q_weight=A + 2), B.ERR_MISALIGNED),
    (dict(q_stride=48 * 128 + 4), B.ERR_MISALIGNED), (dict(stride_token=1028), B.ERR_MISALIGNED),
    (dict(positions=A + 2), B.ERR_MISALIGNED), (dict(q_start=A + 4), B.ERR_MISALIGNED),
]


@pytest.mark.parametrize("kw,status", BAD, ids=str)
@pytest.mark.parametrize("paged", [False, True])
def test_refusals(plan, paged, kw, status):
    assert _call(plan, paged, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(block_table=None), B.ERR_NULL_POINTER), (dict(page_size=24), B.ERR_INVALID_SHAPE),
    (dict(num_pages=0), B.ERR_INVALID_SHAPE), (dict(max_pages=255), B.ERR_INVALID_SHAPE),
    (dict(stride_page=4), B.ERR_MISALIGNED)])
def test_paged_refusals(plan, kw, status):
    assert _call(plan, True, **kw) == status


def test_contiguous_needs_seq_start(plan):
    assert _call(plan, seq_start=None) == B.ERR_NULL_POINTER


def test_empty_calls_and_bad_handle(plan):
    nothing = dict(rope=None, q=None, new_k=None, new_v=None, q_out=None, k=None, v=None, ctx_lens=None)
    for paged in (False, True):
        assert _call(plan, paged, batch=0, **nothing) == B.OK
        assert _call(plan, paged, max_q_len=0, **nothing) == B.OK
        assert _call(None, paged) == B.ERR_BAD_HANDLE


def test_fp8_scale_without_reciprocal():
    p = _plan(dtype=B.FP8_E4M3, k_scale=1e-40)
    assert _call(p) == B.ERR_UNSUPPORTED
    B.comem_decode_attn_destroy(p)


# ------------------------------------------------------------ the wrapper


class Reached(Exception):
    pass


@pytest.fixture
def op(monkeypatch):
    def sentinel(*a, **k):
        raise Reached()

    for name in B.ROPE_EXPORTED:
        monkeypatch.setattr(B, name, sentinel)
    o = object.__new__(B.DecodeAttention)
    o.plan, o.dtype, o.device = None, "bf16", 0
    o.num_q_heads, o.num_kv_heads, o.head_dim = 8, 2, 64
    o._torch_device = torch.device("cpu")
    o._q_dtypes, o._kv_dtypes = B._torch_dtypes("bf16")
    o._stream = lambda s: 0
    return o


def _good(rows=3, paged=False):
    bf = torch.bfloat16
    qkv = torch.zeros(rows, 12, 64, dtype=bf)
    d = dict(q=qkv[:, :8], new_k=qkv[:, 8:10], new_v=qkv[:, 10:], ctx_lens=torch.ones(3, dtype=torch.int32),
             max_ctx_len=64, cos_sin=torch.zeros(64, 64), q_weight=torch.zeros(64, dtype=bf),
             k_weight=torch.zeros(64, dtype=bf))
    if paged:
        d.update(k_pages=torch.zeros(6, 16, 2, 64, dtype=bf), v_pages=torch.zeros(6, 16, 2, 64, dtype=bf),
                 block_table=torch.zeros(3, 4, dtype=torch.int32))
    else:
        d.update(k=torch.zeros(40, 2, 64, dtype=bf), v=torch.zeros(40, 2, 64, dtype=bf),
                 seq_start=torch.zeros(3, dtype=torch.int64))
    return d


def test_wrapper_passes_good_tensors(op):
    with pytest.raises(Reached):
        op.rope_append(**_good())
    with pytest.raises(Reached):
        op.rope_append_paged(**_good(paged=True))
    chunk = dict(q_start=torch.zeros(3, dtype=torch.int64), q_lens=torch.ones(3, dtype=torch.int32), max_q_len=4)
    with pytest.raises(Reached):
        op.rope_append(**_good(rows=7), **chunk, positions=torch.zeros(7, dtype=torch.int32))


@pytest.mark.parametrize("change", [
    dict(q=torch.zeros(3, 8, 64)), dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3, 8, 128, dtype=torch.bfloat16)[..., ::2]),
    dict(q=torch.zeros(8, 3, 64, dtype=torch.bfloat16).transpose(0, 1)), dict(q=None),
    dict(new_k=torch.zeros(4, 2, 64, dtype=torch.bfloat16)), dict(new_v=torch.zeros(3, 2, 64)),
    dict(ctx_lens=torch.ones(2, dtype=torch.int32)), dict(ctx_lens=torch.ones(3)),
    dict(cos_sin=torch.zeros(64, 64, dtype=torch.float64)), dict(cos_sin=torch.zeros(64)),
    dict(cos_sin=torch.zeros(64, 128)[:, ::2]), dict(q_weight=torch.zeros(64)),
    dict(k_weight=torch.zeros(32, dtype=torch.bfloat16)), dict(q_start=torch.zeros(3, dtype=torch.int64)),
    dict(q_lens=torch.ones(3, dtype=torch.int32)), dict(positions=torch.zeros(3, dtype=torch.int64)),
    dict(positions=torch.zeros(2, dtype=torch.int32)), dict(max_ctx_len=1.5), dict(max_q_len=True),
    dict(q_out=torch.zeros(3, 8, 64)), dict(q_out=torch.zeros(2, 8, 64, dtype=torch.bfloat16)),
    dict(k=torch.zeros(40, 2, 64)), dict(seq_start=torch.zeros(3, dtype=torch.int32)),
], ids=lambda c: next(iter(c)))
def test_wrapper_refuses(op, change):
    with pytest.raises(ValueError):
        op.rope_append(**dict(_good(), **change))


@pytest.mark.parametrize("change", [
    dict(q_start=None), dict(q_lens=None), dict(q_start=torch.zeros(3, dtype=torch.int32)),
    dict(q_lens=torch.ones(3, dtype=torch.int64)), dict(q_start=torch.zeros(2, dtype=torch.int64)),
    dict(q_lens=torch.ones(4, dtype=torch.int32)), dict(q_lens=torch.ones(6, dtype=torch.int32)[::2]),
    dict(q_start=torch.zeros(3, 1, dtype=torch.int64)), dict(q_lens=[1, 1, 1]), dict(ctx_lens=None),
    dict(ctx_lens=torch.tensor(1, dtype=torch.int32)), dict(ctx_lens=torch.ones(3, 1, dtype=torch.int32)),
    dict(positions=torch.zeros(3, dtype=torch.int32)), dict(new_k=torch.zeros(3, 2, 64, dtype=torch.bfloat16)),
    dict(q_out=torch.zeros(3, 8, 64, dtype=torch.bfloat16)),
], ids=lambda c: next(iter(c)))
def test_wrapper_refuses_chunks(op, change):
    chunk = dict(q_start=torch.zeros(3, dtype=torch.int64), q_lens=torch.ones(3, dtype=torch.int32), max_q_len=4)
    with pytest.raises(ValueError):
        op.rope_append(**dict(_good(rows=7), **dict(chunk, **change)))


# ------------------------------------------------------------ the plain form


def test_plain_form_is_a_rotation():
    """By hand: a quarter turn maps (a, b) to (-b, a), keeps norms, and two turns add up."""
    x = np.zeros((1, 1, 64))
    x[0, 0, :4] = [1, 2, 3, 4]
    quarter = np.concatenate([np.zeros((1, 2)), np.ones((1, 2))], axis=1)
    assert rotated(x, None, 0, quarter, [0], True)[0][0, 0, :4].tolist() == [-2, 1, -4, 3]
    assert rotated(x, None, 0, quarter, [0], False)[0][0, 0, :4].tolist() == [-3, -4, 1, 2]
    rng = np.random.default_rng(3)
    x, a = rng.normal(size=(5, 2, 64)), rng.normal(size=(5, 16))
    once = np.concatenate([np.cos(a), np.sin(a)], axis=1)
    twice = np.concatenate([np.cos(2 * a), np.sin(2 * a)], axis=1)
    for inter in (False, True):
        y = rotated(rotated(x, None, 0, once, np.arange(5), inter)[0], None, 0, once, np.arange(5), inter)[0]
        assert np.allclose(y, rotated(x, None, 0, twice, np.arange(5), inter)[0], atol=1e-14)
        assert np.array_equal(y[..., 32:], x[..., 32:])
    z, _ = rotated(x, np.ones(64), 0.0, once[:, :0], np.arange(5), False)
    assert np.allclose((z * z).mean(-1), 1.0)


def test_most_tokens_of_a_launch():
    p = _plan(max_ctx_len=1 << 27)
    for tokens, status in (((1 << 26) - 1, B.ERR_NO_DEVICE), (1 << 26, B.ERR_INVALID_SHAPE)):
        assert _call(p, max_q_len=tokens, max_ctx_len=1 << 27) == status
    B.comem_decode_attn_destroy(p)
