"""comem_block_attn.h without a GPU: exported symbols, host-side validation, the wrapper's checks."""

import os
import re

import pytest
import torch

from paper_2605_30842_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20


def test_header_and_library():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "comem_block_attn.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(comem_block_[a-z_]+)\s*\(", text))) == sorted(B.BLOCK_EXPORTED)
    for name in B.BLOCK_EXPORTED:
        assert hasattr(B.load_library(), name)


@pytest.fixture
def plan():
    p, _ = B.comem_decode_attn_init(B.Config(num_q_heads=32, num_kv_heads=8, head_dim=128, dtype=B.BF16, scale=0.088,
                                             max_batch=4, max_ctx_len=4096), B.NO_DEVICE)
    yield p
    B.comem_decode_attn_destroy(p)


def _bounds(plan, **kw):
    a = dict(k_pages=A, stride_page=16 * 1024, stride_token=1024, stride_head=128, page_size=16, num_pages=100,
             block_table=A, max_pages=256, ctx_lens=A, q_lens=A, max_q_len=5, batch=3, max_ctx_len=4096, bounds=A)
    a.update(kw)
    return B.load_library().comem_block_bounds(plan, *a.values(), None)


def _scores(plan, **kw):
    a = dict(q=A, bounds=A, page_size=16, num_pages=100, block_table=A, max_pages=256, ctx_lens=A, batch=3,
             max_ctx_len=4096, scores=A, scores_stride=256)
    a.update(kw)
    return B.load_library().comem_block_scores(plan, *a.values(), None)


def _select(plan, **kw):
    a = dict(scores=A, scores_stride=256, page_size=16, block_table=A, max_pages=256, ctx_lens=A, batch=3,
             max_ctx_len=4096, budget=32, first=1, last=2, table=A, max_blocks=32, lens=A)
    a.update(kw)
    return B.load_library().comem_block_select(plan, *a.values(), None)


def _attn(plan, **kw):
    a = dict(q=A, k_pages=A, v_pages=A, stride_page=16 * 1024, stride_token=1024, stride_head=128, page_size=16,
             num_pages=100, table=A, max_blocks=32, lens=A, batch=3, max_len=512, out=A, lse=A, workspace=A, nbytes=1 << 30)
    a.update(kw)
    return B.load_library().comem_block_attn(plan, *a.values(), None)


CALLS = (_bounds, _scores, _select, _attn)


def test_good_calls_stop_at_the_device(plan):
    for call in CALLS:
        assert call(plan) == B.ERR_NO_DEVICE
    assert _bounds(plan, q_lens=None, max_q_len=1) == B.ERR_NO_DEVICE
    assert _select(plan, budget=5000, max_blocks=256) == B.ERR_NO_DEVICE
    assert _select(plan, first=0, last=32) == B.ERR_NO_DEVICE
    assert _attn(plan, lse=None) == B.ERR_NO_DEVICE
    assert _scores(plan, max_ctx_len=0, scores=None) == B.ERR_NO_DEVICE
    assert _select(plan, max_ctx_len=0, scores=None, table=None) == B.ERR_NO_DEVICE


def test_empty_calls_look_at_nothing(plan):
    none = dict(block_table=None, ctx_lens=None, batch=0)
    assert _bounds(plan, k_pages=None, bounds=None, **none) == B.OK
    assert _bounds(plan, k_pages=None, bounds=None, max_q_len=0) == B.OK
    assert _scores(plan, q=None, bounds=None, scores=None, **none) == B.OK
    assert _select(plan, scores=None, table=None, lens=None, **none) == B.OK
    assert _attn(plan, q=None, table=None, lens=None, out=None, batch=0) == B.OK


def test_a_bad_plan(plan):
    assert {call(None) for call in CALLS} == {B.ERR_BAD_HANDLE}


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), B.ERR_INVALID_SHAPE), (dict(batch=5), B.ERR_INVALID_SHAPE),
    (dict(max_ctx_len=4097), B.ERR_INVALID_SHAPE), (dict(max_ctx_len=-1), B.ERR_INVALID_SHAPE),
    (dict(page_size=0), B.ERR_INVALID_SHAPE), (dict(page_size=24), B.ERR_INVALID_SHAPE),
    (dict(page_size=8192), B.ERR_INVALID_SHAPE), (dict(max_pages=255), B.ERR_INVALID_SHAPE),
    (dict(block_table=None), B.ERR_NULL_POINTER), (dict(ctx_lens=None), B.ERR_NULL_POINTER),
    (dict(block_table=A + 2), B.ERR_MISALIGNED), (dict(ctx_lens=A + 2), B.ERR_MISALIGNED)], ids=str)
def test_refusals_of_all(plan, kw, status):
    for call in CALLS[:3]:
        assert call(plan, **kw) == status


@pytest.mark.parametrize("call,kw,status", [
    (_bounds, dict(k_pages=None), B.ERR_NULL_POINTER), (_bounds, dict(bounds=None), B.ERR_NULL_POINTER),
    (_bounds, dict(q_lens=None), B.ERR_INVALID_SHAPE), (_bounds, dict(max_q_len=-1), B.ERR_INVALID_SHAPE),
    (_bounds, dict(max_q_len=4097), B.ERR_INVALID_SHAPE), (_bounds, dict(num_pages=0), B.ERR_INVALID_SHAPE),
    (_bounds, dict(stride_page=0), B.ERR_INVALID_SHAPE), (_bounds, dict(stride_token=0), B.ERR_INVALID_SHAPE),
    (_bounds, dict(stride_token=1 << 40), B.ERR_INVALID_SHAPE), (_bounds, dict(stride_head=0), B.ERR_INVALID_SHAPE),
    (_bounds, dict(stride_page=16 * 1024 + 4), B.ERR_MISALIGNED), (_bounds, dict(stride_token=1028), B.ERR_MISALIGNED),
    (_bounds, dict(stride_head=132), B.ERR_MISALIGNED), (_bounds, dict(k_pages=A + 8), B.ERR_MISALIGNED),
    (_bounds, dict(bounds=A + 8), B.ERR_MISALIGNED), (_bounds, dict(q_lens=A + 2), B.ERR_MISALIGNED),
    (_scores, dict(q=None), B.ERR_NULL_POINTER), (_scores, dict(bounds=None), B.ERR_NULL_POINTER),
    (_scores, dict(scores=None), B.ERR_NULL_POINTER), (_scores, dict(num_pages=0), B.ERR_INVALID_SHAPE),
    (_scores, dict(scores_stride=255), B.ERR_INVALID_SHAPE), (_scores, dict(q=A + 8), B.ERR_MISALIGNED),
    (_scores, dict(bounds=A + 8), B.ERR_MISALIGNED), (_scores, dict(scores=A + 2), B.ERR_MISALIGNED),
    (_select, dict(scores=None), B.ERR_NULL_POINTER), (_select, dict(table=None), B.ERR_NULL_POINTER),
    (_select, dict(lens=None), B.ERR_NULL_POINTER), (_select, dict(first=-1), B.ERR_INVALID_SHAPE),
    (_select, dict(last=0), B.ERR_INVALID_SHAPE), (_select, dict(budget=2), B.ERR_INVALID_SHAPE),
    (_select, dict(first=2 ** 31 - 1, last=2 ** 31 - 1), B.ERR_INVALID_SHAPE),
    (_select, dict(scores_stride=255), B.ERR_INVALID_SHAPE), (_select, dict(max_blocks=31), B.ERR_INVALID_SHAPE),
    (_select, dict(budget=5000, max_blocks=255), B.ERR_INVALID_SHAPE), (_select, dict(scores=A + 2), B.ERR_MISALIGNED),
    (_select, dict(table=A + 2), B.ERR_MISALIGNED), (_select, dict(lens=A + 2), B.ERR_MISALIGNED),
    (_attn, dict(q=None), B.ERR_NULL_POINTER), (_attn, dict(table=None), B.ERR_NULL_POINTER),
    (_attn, dict(lens=None), B.ERR_NULL_POINTER), (_attn, dict(max_blocks=31), B.ERR_INVALID_SHAPE),
    (_attn, dict(max_len=4097), B.ERR_INVALID_SHAPE), (_attn, dict(num_pages=0), B.ERR_INVALID_SHAPE),
    (_attn, dict(page_size=24), B.ERR_INVALID_SHAPE), (_attn, dict(table=A + 2), B.ERR_MISALIGNED),
    (_attn, dict(out=A + 8), B.ERR_MISALIGNED), (_attn, dict(workspace=A + 64), B.ERR_MISALIGNED)],
    ids=lambda v: getattr(v, "__name__", str(v)))
def test_refusals(plan, call, kw, status):
    assert call(plan, **kw) == status


def test_select_fits_a_launch():
    """Items beyond what one launch holds are refused, not cut."""
    p, _ = B.comem_decode_attn_init(B.Config(num_q_heads=65535, num_kv_heads=65535, head_dim=64, dtype=B.BF16, scale=0.1,
                                             max_batch=65535, max_ctx_len=64), B.NO_DEVICE)
    assert _select(p, batch=65535, max_ctx_len=64) == B.ERR_INVALID_SHAPE
    assert _select(p, batch=200, max_ctx_len=64) == B.ERR_NO_DEVICE
    B.comem_decode_attn_destroy(p)


# ------------------------------------------------------------ the wrapper


class Reached(Exception):
    pass


@pytest.fixture
def op(monkeypatch):
    def sentinel(*a, **k):
        raise Reached()

    for name in B.BLOCK_EXPORTED:
        monkeypatch.setattr(B, name, sentinel)
    o = object.__new__(B.DecodeAttention)
    o.plan = None
    o.dtype, o.device = "bf16", 0
    o.num_q_heads, o.num_kv_heads, o.head_dim = 8, 2, 64
    o._torch_device = torch.device("cpu")
    o._q_dtypes, o._kv_dtypes = B._torch_dtypes("bf16")
    o._stream = lambda s: 0
    o.workspace, o.workspace_bytes = torch.zeros(256, dtype=torch.uint8), 256
    return o


BF, I32 = torch.bfloat16, torch.int32


def _args(name, **kw):
    pool, table, lens = torch.zeros(10, 16, 2, 64, dtype=BF), torch.zeros(3, 4, dtype=I32), torch.zeros(3, dtype=I32)
    q, ends = torch.zeros(3, 8, 64, dtype=BF), torch.zeros(10, 2, 2, 64, dtype=BF)
    d = dict(
        block_bounds=dict(k_pages=pool, block_table=table, ctx_lens=lens, max_ctx_len=64, bounds=ends,
                          q_lens=lens.clone(), max_q_len=5),
        block_scores=dict(q=q, bounds=ends, page_size=16, block_table=table, ctx_lens=lens, max_ctx_len=60,
                          scores=torch.zeros(3, 2, 4)),
        block_select=dict(scores=torch.zeros(3, 2, 4), page_size=16, block_table=table, ctx_lens=lens, max_ctx_len=60,
                          budget=3, first=1, last=1, table=torch.zeros(3, 2, 3, dtype=I32), lens=lens.clone()),
        block_forward=dict(q=q, k_pages=pool, v_pages=pool.clone(), table=torch.zeros(3, 2, 3, dtype=I32),
                           lens=lens, max_len=48, out=torch.zeros(3, 8, 64), lse=torch.zeros(3, 8)))[name]
    d.update(kw)
    return d


@pytest.mark.parametrize("name,kw", [
    ("block_bounds", {}), ("block_bounds", dict(q_lens=None, max_q_len=1)), ("block_scores", {}),
    ("block_scores", dict(scores=None)), ("block_select", {}), ("block_select", dict(table=None, lens=None)),
    ("block_forward", {}), ("block_forward", dict(out=None, lse=None))], ids=str)
def test_wrapper_good_calls(op, name, kw):
    with pytest.raises(Reached):
        getattr(op, name)(**_args(name, **kw))


@pytest.mark.parametrize("name,kw", [
    ("block_bounds", dict(k_pages=torch.zeros(10, 16, 2, 32, dtype=BF))), ("block_bounds", dict(bounds=torch.zeros(10, 2, 2, 64))),
    ("block_bounds", dict(bounds=torch.zeros(9, 2, 2, 64, dtype=BF))), ("block_bounds", dict(bounds=torch.zeros(10, 2, 64, dtype=BF))),
    ("block_bounds", dict(q_lens=torch.zeros(2, dtype=I32))), ("block_bounds", dict(max_q_len=1.5)),
    ("block_bounds", dict(ctx_lens=torch.zeros(3))), ("block_bounds", dict(block_table=torch.zeros(2, 4, dtype=I32))),
    ("block_scores", dict(q=torch.zeros(2, 8, 64, dtype=BF))), ("block_scores", dict(q=torch.zeros(3, 8, 64))),
    ("block_scores", dict(bounds=torch.zeros(10, 2, 2, 64))), ("block_scores", dict(bounds=None)),
    ("block_scores", dict(bounds=torch.zeros(10, 2, 2, 32, dtype=BF))), ("block_scores", dict(page_size=0)),
    ("block_scores", dict(page_size=16.0)), ("block_scores", dict(scores=torch.zeros(3, 2, 5))),
    ("block_scores", dict(scores=torch.zeros(3, 2, 4).half())), ("block_select", dict(scores=torch.zeros(3, 2, 5))),
    ("block_select", dict(budget=None)), ("block_select", dict(table=torch.zeros(3, 2, 4, dtype=I32))),
    ("block_select", dict(table=torch.zeros(3, 2, 3))), ("block_select", dict(lens=torch.zeros(2, dtype=I32))),
    ("block_forward", dict(table=torch.zeros(3, 3, dtype=I32))), ("block_forward", dict(table=None)),
    ("block_forward", dict(table=torch.zeros(3, 1, 3, dtype=I32))), ("block_forward", dict(lens=torch.zeros(3))),
    ("block_forward", dict(lse=torch.zeros(3, 7))), ("block_forward", dict(max_len="48"))],
    ids=lambda v: v if isinstance(v, str) else str(list(v)))
def test_wrapper_refusals(op, name, kw):
    with pytest.raises(ValueError):
        getattr(op, name)(**_args(name, **kw))
