"""comem_kv_evict.h without a GPU: exported symbols, host-side validation, the wrapper's checks."""

import os
import re

import pytest
import torch

from paper_2605_30842_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20


def test_header_and_library():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "comem_kv_evict.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(comem_(?:attn|keep)_[a-z_]+)\s*\(", text))) == sorted(B.EVICT_EXPORTED)
    for name in B.EVICT_EXPORTED:
        assert hasattr(B.load_library(), name)


@pytest.fixture
def plan():
    p, _ = B.comem_decode_attn_init(B.Config(num_q_heads=32, num_kv_heads=8, head_dim=128, dtype=B.BF16, scale=0.088,
                                             max_batch=4, max_ctx_len=4096), B.NO_DEVICE)
    yield p
    B.comem_decode_attn_destroy(p)


def _weights(plan, **kw):
    a = dict(q=A, lse=A, q_start=A, q_lens=A, max_q_len=7, k=A, stride_token=1024, stride_head=128, seq_start=A,
             ctx_lens=A, batch=3, max_ctx_len=4096, prior=A, decay=0.5, weights=A, weights_stride=4096, workspace=None, nbytes=0)
    a.update(kw)
    return B.load_library().comem_attn_weights(plan, *a.values(), None)


def _paged(plan, **kw):
    a = dict(q=A, lse=A, q_start=A, q_lens=A, max_q_len=7, k=A, stride_page=16 * 1024, stride_token=1024,
             stride_head=128, page_size=16, num_pages=100, block_table=A, max_pages=256, ctx_lens=A, batch=3,
             max_ctx_len=4096, prior=A, decay=0.5, weights=A, weights_stride=4096, workspace=None, nbytes=0)
    a.update(kw)
    return B.load_library().comem_attn_weights_paged(plan, *a.values(), None)


def _keep(plan, **kw):
    a = dict(weights=A, weights_stride=4096, ctx_lens=A, num_rows=8, rows=A, n=5, max_ctx_len=4096, budget=100,
             budgets=A, first=10, last=20, keep=A, keep_stride=100, keep_start=A, keep_lens=A, kept=A,
             workspace=None, nbytes=0)
    a.update(kw)
    return B.load_library().comem_keep_tokens(plan, *a.values(), None)


def test_good_calls_stop_at_the_device(plan):
    for call in (_weights, _paged):
        assert call(plan) == B.ERR_NO_DEVICE
        assert call(plan, prior=None, decay=float("nan")) == B.ERR_NO_DEVICE
        assert call(plan, q_start=None, q_lens=None, max_q_len=1) == B.ERR_NO_DEVICE
        assert call(plan, decay=0.0) == B.ERR_NO_DEVICE
    for kw in ({}, dict(rows=None, budgets=None, keep_start=None, kept=None), dict(budget=0, first=0, last=0),
               dict(budget=5000, keep_stride=4096), dict(first=0, last=100), dict(budget=0, first=0, last=0, keep=None),
               dict(max_ctx_len=0, weights=None, keep=None)):
        assert _keep(plan, **kw) == B.ERR_NO_DEVICE


def test_empty_calls_look_at_nothing(plan):
    for call in (_weights, _paged):
        for kw in (dict(batch=0), dict(max_q_len=0)):
            assert call(plan, q=None, lse=None, k=None, ctx_lens=None, weights=None, **kw) == B.OK
    assert _keep(plan, n=0, weights=None, ctx_lens=None, keep=None, keep_lens=None) == B.OK


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), B.ERR_NULL_POINTER), (dict(lse=None), B.ERR_NULL_POINTER), (dict(k=None), B.ERR_NULL_POINTER),
    (dict(ctx_lens=None), B.ERR_NULL_POINTER), (dict(weights=None), B.ERR_NULL_POINTER),
    (dict(q_start=None), B.ERR_NULL_POINTER), (dict(q_lens=None), B.ERR_NULL_POINTER),
    (dict(q_start=None, q_lens=None), B.ERR_INVALID_SHAPE), (dict(batch=-1), B.ERR_INVALID_SHAPE),
    (dict(batch=5), B.ERR_INVALID_SHAPE), (dict(max_ctx_len=4097), B.ERR_INVALID_SHAPE),
    (dict(max_ctx_len=-1), B.ERR_INVALID_SHAPE), (dict(max_q_len=-1), B.ERR_INVALID_SHAPE),
    (dict(max_q_len=4097), B.ERR_INVALID_SHAPE), (dict(weights_stride=4095), B.ERR_INVALID_SHAPE),
    (dict(decay=-0.5), B.ERR_INVALID_SHAPE), (dict(decay=float("inf")), B.ERR_INVALID_SHAPE),
    (dict(decay=float("nan")), B.ERR_INVALID_SHAPE), (dict(stride_token=0), B.ERR_INVALID_SHAPE),
    (dict(stride_token=1 << 40), B.ERR_INVALID_SHAPE), (dict(stride_head=0), B.ERR_INVALID_SHAPE),
    (dict(stride_head=-128), B.ERR_INVALID_SHAPE), (dict(stride_token=1028), B.ERR_MISALIGNED),
    (dict(stride_head=132), B.ERR_MISALIGNED), (dict(q=A + 8), B.ERR_MISALIGNED), (dict(k=A + 8), B.ERR_MISALIGNED),
    (dict(lse=A + 2), B.ERR_MISALIGNED), (dict(q_start=A + 4), B.ERR_MISALIGNED), (dict(q_lens=A + 2), B.ERR_MISALIGNED),
    (dict(ctx_lens=A + 2), B.ERR_MISALIGNED), (dict(prior=A + 2), B.ERR_MISALIGNED),
    (dict(weights=A + 2), B.ERR_MISALIGNED), (dict(workspace=A + 64, nbytes=1 << 20), B.ERR_MISALIGNED)], ids=str)
def test_weights_refusals(plan, kw, status):
    assert _weights(plan, **kw) == status
    assert _paged(plan, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(block_table=None), B.ERR_NULL_POINTER), (dict(page_size=0), B.ERR_INVALID_SHAPE),
    (dict(page_size=24), B.ERR_INVALID_SHAPE), (dict(page_size=8192), B.ERR_INVALID_SHAPE),
    (dict(num_pages=0), B.ERR_INVALID_SHAPE), (dict(stride_page=0), B.ERR_INVALID_SHAPE),
    (dict(max_pages=255), B.ERR_INVALID_SHAPE), (dict(stride_page=16 * 1024 + 4), B.ERR_MISALIGNED),
    (dict(block_table=A + 2), B.ERR_MISALIGNED)], ids=str)
def test_paged_refusals(plan, kw, status):
    assert _paged(plan, **kw) == status


def test_workspace(plan):
    """None for a step and for what fills the chip; a sum for each token and part otherwise; the call's own bounds hold."""
    size = lambda *a: B.comem_attn_weights_workspace(plan, *a)  # noqa: E731
    assert size(4, 1, 4096) == size(0, 5, 4096) == size(4, 0, 4096) == 0
    assert size(1, 300, 4096) >= 2 * 4096 * 4 and size(1, 300, 4096) % 256 == 0
    for a in ((5, 1, 4096), (-1, 1, 4096), (1, -1, 4096), (1, 5, 4), (1, 1, 4097), (1, 1, -1)):
        with pytest.raises(B.ComemError) as e:
            size(*a)
        assert e.value.status == B.ERR_INVALID_SHAPE
    with pytest.raises(B.ComemError):
        B.comem_attn_weights_workspace(None, 1, 1, 1)
    assert B.load_library().comem_attn_weights_workspace(plan, 1, 1, 1, None) == B.ERR_NULL_POINTER
    for nbytes in (0, 1, 1 << 30):
        assert _weights(plan, workspace=A, nbytes=nbytes) == _paged(plan, workspace=A, nbytes=nbytes) == B.ERR_NO_DEVICE


def test_contiguous_refusals(plan):
    assert _weights(plan, seq_start=None) == B.ERR_NULL_POINTER
    assert _weights(plan, seq_start=A + 4) == B.ERR_MISALIGNED
    assert _weights(None) == _paged(None) == _keep(None) == B.ERR_BAD_HANDLE


@pytest.mark.parametrize("kw,status", [
    (dict(num_rows=0), B.ERR_INVALID_SHAPE), (dict(num_rows=65536), B.ERR_INVALID_SHAPE),
    (dict(n=-1), B.ERR_INVALID_SHAPE), (dict(n=9), B.ERR_INVALID_SHAPE), (dict(max_ctx_len=4097), B.ERR_INVALID_SHAPE),
    (dict(max_ctx_len=-1), B.ERR_INVALID_SHAPE), (dict(first=-1), B.ERR_INVALID_SHAPE),
    (dict(last=-1), B.ERR_INVALID_SHAPE), (dict(first=90), B.ERR_INVALID_SHAPE), (dict(budget=-1), B.ERR_INVALID_SHAPE),
    (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), B.ERR_INVALID_SHAPE), (dict(weights_stride=4095), B.ERR_INVALID_SHAPE),
    (dict(keep_stride=99), B.ERR_INVALID_SHAPE), (dict(budget=5000, keep_stride=4095), B.ERR_INVALID_SHAPE),
    (dict(weights=None), B.ERR_NULL_POINTER), (dict(ctx_lens=None), B.ERR_NULL_POINTER),
    (dict(keep=None), B.ERR_NULL_POINTER), (dict(keep_lens=None), B.ERR_NULL_POINTER),
    (dict(weights=A + 2), B.ERR_MISALIGNED), (dict(ctx_lens=A + 2), B.ERR_MISALIGNED), (dict(rows=A + 2), B.ERR_MISALIGNED),
    (dict(budgets=A + 2), B.ERR_MISALIGNED), (dict(keep=A + 2), B.ERR_MISALIGNED),
    (dict(keep_start=A + 4), B.ERR_MISALIGNED), (dict(keep_lens=A + 2), B.ERR_MISALIGNED),
    (dict(kept=A + 2), B.ERR_MISALIGNED), (dict(workspace=A + 64, nbytes=1 << 20), B.ERR_MISALIGNED)], ids=str)
def test_keep_refusals(plan, kw, status):
    assert _keep(plan, **kw) == status


def test_keep_workspace():
    """None for rows that one workgroup takes, and for too many rows or chunks; else counts and lists of every entry."""
    p, _ = B.comem_decode_attn_init(B.Config(num_q_heads=8, num_kv_heads=8, head_dim=64, dtype=B.BF16, scale=0.1,
                                             max_batch=4, max_ctx_len=1 << 30), B.NO_DEVICE)
    size = lambda *a: B.comem_keep_tokens_workspace(p, *a)  # noqa: E731
    assert size(0, 100000) == size(5, 49152) == size(5, 0) == size(5, 1 << 30) == 0
    assert size(33, 50000) == size(17, 500000) == 0
    assert size(1, 49153) >= 4 * 49153 and size(3, 131072) == 3 * size(1, 131072) and size(1, 131072) % 256 == 0
    for a in ((-1, 5), (65536, 5), (1, -1), (1, (1 << 30) + 1)):
        with pytest.raises(B.ComemError) as e:
            size(*a)
        assert e.value.status == B.ERR_INVALID_SHAPE
    assert B.load_library().comem_keep_tokens_workspace(p, 1, 1, None) == B.ERR_NULL_POINTER
    assert B.load_library().comem_keep_tokens_workspace(None, 1, 1, None) == B.ERR_BAD_HANDLE
    for nbytes in (0, 5, 1 << 30):
        assert _keep(p, max_ctx_len=100000, weights_stride=100000, workspace=A, nbytes=nbytes) == B.ERR_NO_DEVICE
    B.comem_decode_attn_destroy(p)


# ------------------------------------------------------------ the wrapper


class Reached(Exception):
    pass


@pytest.fixture
def op(monkeypatch):
    def sentinel(*a, **k):
        raise Reached()

    for name in ("comem_attn_weights", "comem_attn_weights_paged", "comem_keep_tokens"):
        monkeypatch.setattr(B, name, sentinel)
    o = object.__new__(B.DecodeAttention)
    o.plan, _ = B.comem_decode_attn_init(B.Config(num_q_heads=8, num_kv_heads=2, head_dim=64, dtype=B.BF16, scale=0.1,
                                                  max_batch=4, max_ctx_len=64), B.NO_DEVICE)
    o.dtype, o.device = "bf16", 0
    o.num_q_heads, o.num_kv_heads, o.head_dim = 8, 2, 64
    o._torch_device = torch.device("cpu")
    o._q_dtypes, o._kv_dtypes = B._torch_dtypes("bf16")
    o._stream = lambda s: 0
    return o


def _tensors(**kw):
    bf = torch.bfloat16
    d = dict(q=torch.zeros(5, 8, 64, dtype=bf), lse=torch.zeros(5, 8), k=torch.zeros(40, 2, 64, dtype=bf),
             seq_start=torch.zeros(3, dtype=torch.int64), ctx_lens=torch.zeros(3, dtype=torch.int32), max_ctx_len=20,
             q_start=torch.zeros(3, dtype=torch.int64), q_lens=torch.zeros(3, dtype=torch.int32), max_q_len=2,
             prior=torch.zeros(3, 32), decay=0.5, out=torch.zeros(3, 32))
    d.update(kw)
    return d


def test_wrapper_good_calls(op):
    for kw in ({}, dict(out=None), dict(out=None, prior=None), dict(prior=None),
               dict(q_start=None, q_lens=None, max_q_len=1, q=torch.zeros(3, 8, 64, dtype=torch.bfloat16),
                    lse=torch.zeros(3, 8)),
               dict(out=torch.zeros(3, 64)[:, :32], prior=torch.zeros(3, 64)[:, 5:37]),
               dict(workspace=torch.zeros(256, dtype=torch.uint8))):
        if kw.get("out", 1) is None and "prior" not in kw:
            kw = dict(kw, prior=torch.zeros(3, 20))
        with pytest.raises(Reached):
            op.attn_weights(**_tensors(**kw))
    t = _tensors(block_table=torch.zeros(3, 2, dtype=torch.int32), k_pages=torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16))
    del t["k"], t["seq_start"]
    with pytest.raises(Reached):
        op.attn_weights_paged(**t)


@pytest.mark.parametrize("kw", [
    dict(q=torch.zeros(5, 8, 64)), dict(lse=None), dict(lse=torch.zeros(5, 7)), dict(lse=torch.zeros(5, 8).double()),
    dict(k=torch.zeros(40, 2, 32, dtype=torch.bfloat16)), dict(k=torch.zeros(40, 2, 64)),
    dict(q_start=None), dict(q_lens=None), dict(q_start=None, q_lens=None), dict(q_lens=torch.zeros(3)),
    dict(seq_start=torch.zeros(3, dtype=torch.int32)), dict(ctx_lens=torch.zeros(3)), dict(max_ctx_len=20.0),
    dict(max_q_len=True), dict(out=torch.zeros(3, 19)), dict(out=torch.zeros(2, 32)),
    dict(out=torch.zeros(32, 3).T), dict(prior=torch.zeros(3, 19)), dict(prior=torch.zeros(3, 31)),
    dict(prior=torch.zeros(3, 32).half()), dict(workspace=torch.zeros(64, 64)[:, 1]), dict(workspace=5), dict(out=torch.zeros(1, 32).expand(3, 32))], ids=lambda kw: str(list(kw)))
def test_wrapper_refusals(op, kw):
    with pytest.raises(ValueError):
        op.attn_weights(**_tensors(**kw))


def _keep_tensors(**kw):
    d = dict(weights=torch.zeros(6, 32), ctx_lens=torch.zeros(6, dtype=torch.int32), max_ctx_len=20, budget=8, first=1,
             last=2, rows=torch.zeros(3, dtype=torch.int32), budgets=torch.zeros(3, dtype=torch.int32),
             keep=torch.zeros(3, 8, dtype=torch.int32), kept=torch.zeros(3, 8))
    d.update(kw)
    return d


def test_wrapper_keep(op):
    for kw in ({}, dict(keep=None, kept=None), dict(rows=None, budgets=None, keep=None, kept=None)):
        with pytest.raises(Reached):
            op.keep_tokens(**_keep_tensors(**kw))
    for kw in (dict(weights=torch.zeros(6, 19)), dict(weights=torch.zeros(5, 32)), dict(ctx_lens=torch.zeros(6)),
               dict(budget=8.0), dict(first=None), dict(rows=torch.zeros(3)), dict(budgets=torch.zeros(2, dtype=torch.int32)),
               dict(keep=torch.zeros(3, 9, dtype=torch.int32)), dict(kept=torch.zeros(2, 8)), dict(kept=torch.zeros(3, 8).int())):
        with pytest.raises(ValueError):
            op.keep_tokens(**_keep_tensors(**kw))
