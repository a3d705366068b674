"""comem_prefill_fp8.h without a GPU: exported symbols, host-side validation, and which entry the wrapper takes."""

import ctypes
import os
import re

import pytest
import torch

from paper_2605_30842_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20


def test_header_and_library():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "comem_prefill_fp8.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(comem_prefill_fp8_[a-z_]+)\s*\(", text))) == sorted(B.PREFILL_FP8_EXPORTED)
    for name in B.PREFILL_FP8_EXPORTED:
        assert hasattr(B.load_library(), name)


def _plan(dtype=B.FP8_E4M3, **kw):
    cfg = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, dtype=dtype, scale=0.088, max_batch=4, max_ctx_len=40960,
               k_scale=0.5, v_scale=0.5)
    cfg.update(kw)
    return B.comem_decode_attn_init(B.Config(**cfg), B.NO_DEVICE)[0]


@pytest.fixture
def plan():
    p = _plan()
    yield p
    B.comem_decode_attn_destroy(p)


def _call(plan, paged, **kw):
    a = dict(q=A, q_start=A, q_lens=A, max_q_len=64, k=A, v=A, stride_token=1024, stride_head=128, ctx_lens=A, batch=2,
             max_ctx_len=4096, out=A, lse=A, workspace=A, workspace_bytes=1 << 20, seq_start=A, stride_page=16 * 1024,
             page_size=16, num_pages=100, block_table=A, max_pages=256)
    a.update(kw)
    head = (plan, a["q"], a["q_start"], a["q_lens"], a["max_q_len"], a["k"], a["v"])
    tail = (a["ctx_lens"], a["batch"], a["max_ctx_len"], a["out"], a["lse"], a["workspace"], a["workspace_bytes"], None)
    lib = B.load_library()
    if paged:
        return lib.comem_prefill_fp8_attn_paged(*head, a["stride_page"], a["stride_token"], a["stride_head"],
                                                a["page_size"], a["num_pages"], a["block_table"], a["max_pages"], *tail)
    return lib.comem_prefill_fp8_attn(*head, a["stride_token"], a["stride_head"], a["seq_start"], *tail)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(), B.ERR_NO_DEVICE), (dict(workspace=None, workspace_bytes=0), B.ERR_NO_DEVICE), (dict(lse=None), B.ERR_NO_DEVICE),
    (dict(batch=0, q=None, k=None, out=None), B.OK), (dict(max_q_len=0, q=None, q_lens=None), B.OK),
    (dict(q=None), B.ERR_NULL_POINTER), (dict(q_start=None), B.ERR_NULL_POINTER), (dict(q_lens=None), B.ERR_NULL_POINTER),
    (dict(k=None), B.ERR_NULL_POINTER), (dict(out=None), B.ERR_NULL_POINTER), (dict(batch=5), B.ERR_INVALID_SHAPE),
    (dict(max_q_len=4097), B.ERR_INVALID_SHAPE), (dict(max_ctx_len=40961), B.ERR_INVALID_SHAPE),
    (dict(stride_token=0), B.ERR_INVALID_SHAPE), (dict(stride_token=1032), B.ERR_MISALIGNED),
    (dict(k=A + 8), B.ERR_MISALIGNED), (dict(workspace=A + 64), B.ERR_MISALIGNED),
], ids=str)
def test_validation(plan, paged, kw, status):
    assert _call(plan, paged, **kw) == status


def test_layout_arguments(plan):
    assert _call(plan, False, seq_start=None) == B.ERR_NULL_POINTER
    assert _call(plan, True, block_table=None) == B.ERR_NULL_POINTER
    assert _call(plan, True, max_pages=255) == B.ERR_INVALID_SHAPE
    assert _call(None, True) == B.ERR_BAD_HANDLE


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_other_plans_are_refused(dtype):
    p = _plan(dtype, **(dict(head_dim=64) if dtype == B.F32 else {}))
    n = ctypes.c_size_t()
    assert _call(p, False) == _call(p, True) == B.ERR_UNSUPPORTED
    assert B.load_library().comem_prefill_fp8_workspace(p, 1, 16, 4096, ctypes.byref(n)) == B.ERR_UNSUPPORTED
    B.comem_decode_attn_destroy(p)


def test_workspace(plan):
    assert B.comem_prefill_fp8_workspace(plan, 1, 16, 32768) > 0
    assert B.comem_prefill_fp8_workspace(plan, 1, 4096, 4096) == 0
    assert B.comem_prefill_fp8_workspace(plan, 1, 0, 4096) == 0
    bf16 = _plan(B.BF16)
    assert B.comem_prefill_fp8_workspace(plan, 1, 16, 32768) == B.comem_prefill_attn_workspace(bf16, 1, 16, 32768)
    B.comem_decode_attn_destroy(bf16)
    assert B.load_library().comem_prefill_fp8_workspace(plan, 1, 16, 4096, None) == B.ERR_NULL_POINTER


@pytest.mark.parametrize("dtype,names", [("fp8", ("comem_prefill_fp8_attn", "comem_prefill_fp8_attn_paged")),
                                         ("bf16", ("comem_prefill_attn", "comem_prefill_attn_paged"))])
def test_wrapper_takes_the_entry_of_its_cache(monkeypatch, dtype, names):
    called = []
    for name in ("comem_prefill_fp8_attn", "comem_prefill_fp8_attn_paged", "comem_prefill_attn",
                 "comem_prefill_attn_paged"):
        monkeypatch.setattr(B, name, lambda *a, name=name: called.append(name))
    o = object.__new__(B.DecodeAttention)
    o.plan, o.dtype = None, dtype
    o.num_q_heads, o.num_kv_heads, o.head_dim = 8, 2, 64
    o._torch_device = torch.device("cpu")
    o._q_dtypes, o._kv_dtypes = B._torch_dtypes(dtype)
    o._stream = lambda s: 0
    cache = torch.uint8 if dtype == "fp8" else torch.bfloat16
    i32, i64 = torch.int32, torch.int64
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    lens = (torch.zeros(1, dtype=i64), torch.ones(1, dtype=i32), 3)
    o.prefill(q, *lens, torch.zeros(9, 2, 64, dtype=cache), torch.zeros(9, 2, 64, dtype=cache), torch.zeros(1, dtype=i64),
              torch.ones(1, dtype=i32), 9)
    o.prefill_paged(q, *lens, torch.zeros(2, 16, 2, 64, dtype=cache), torch.zeros(2, 16, 2, 64, dtype=cache),
                    torch.zeros(1, 1, dtype=i32), torch.ones(1, dtype=i32), 9)
    assert tuple(called) == names
    with pytest.raises(ValueError):
        o.prefill(q.float(), *lens, torch.zeros(9, 2, 64, dtype=cache), torch.zeros(9, 2, 64, dtype=cache),
                  torch.zeros(1, dtype=i64), torch.ones(1, dtype=i32), 9)


@pytest.mark.parametrize("current", [0, 1])
def test_the_plans_device_is_current_during_a_call(monkeypatch, current):
    """A call on a plan of another device switches to it (its current stream is asked for there) and back."""
    now, seen = [current], []

    class On:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *a):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    o = object.__new__(B.DecodeAttention)
    o.device, o._torch_device = 1, torch.device("cuda:1")
    B._call_on(o, None, lambda *a: seen.append((now[0], *a)), "x", 7)
    assert seen == [(1, "x", 7, 101)] and now == [current]
