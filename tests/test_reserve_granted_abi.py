"""comem_kv_reserve_granted without a GPU: validation, and what the wrapper passes on and refuses."""

import ctypes

import pytest
import torch

from paper_2605_30842_amd import binding as B

A = 1 << 20


def _plan():
    return B.comem_decode_attn_init(B.Config(num_q_heads=8, num_kv_heads=2, head_dim=64, dtype=B.BF16, scale=0.1,
                                             max_batch=4, max_ctx_len=64), B.NO_DEVICE)[0]


def test_validation():
    plan, lib = _plan(), B.load_library()
    state = B.PagesState(A, A, 0, 16 * 128, 128, 64, 1, 16, 10, A, A, A, 3, 4, 64)
    nbytes = B.comem_kv_pages_workspace(plan, state)

    def call(plan=plan, add=A, granted=2 * A, missing=A, workspace=A, nbytes=nbytes):
        return lib.comem_kv_reserve_granted(plan, ctypes.byref(state), add, granted, missing, workspace, nbytes, None)

    assert call() == B.ERR_NO_DEVICE
    assert call(plan=None) == B.ERR_BAD_HANDLE
    assert call(granted=None) == call(add=None) == call(missing=None) == call(workspace=None) == B.ERR_NULL_POINTER
    assert call(granted=A + 2) == call(add=A + 2) == call(missing=A + 1) == B.ERR_MISALIGNED
    assert call(nbytes=nbytes - 1) == B.ERR_WORKSPACE_TOO_SMALL
    state.num_rows = 0
    assert call() == B.ERR_INVALID_SHAPE
    B.comem_decode_attn_destroy(plan)


def test_wrapper(monkeypatch):
    seen = []
    for name in ("comem_kv_reserve", "comem_kv_reserve_granted"):
        monkeypatch.setattr(B, name, lambda *a, name=name: seen.append((name, a)))
    op = object.__new__(B.DecodeAttention)
    op.plan, op.dtype, op.device = _plan(), "bf16", 0
    op.num_q_heads, op.num_kv_heads, op.head_dim = 8, 2, 64
    op._torch_device = torch.device("cpu")
    op._q_dtypes, op._kv_dtypes = B._torch_dtypes("bf16")
    op._stream = lambda s: 0
    i32 = torch.int32
    pool = torch.zeros(10, 16, 2, 64, dtype=torch.bfloat16)
    p = B.KVPages(op, pool, pool.clone(), torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32),
                  torch.zeros(10, dtype=i32), 64)
    add, granted = torch.zeros(3, dtype=i32), torch.zeros(3, dtype=i32)
    p.reserve(add)
    p.reserve(add, granted=granted)
    assert [name for name, _ in seen] == ["comem_kv_reserve", "comem_kv_reserve_granted"]
    assert seen[1][1][2:4] == (add.data_ptr(), granted.data_ptr())
    both = torch.zeros(5, dtype=i32)
    for bad in (torch.zeros(2, dtype=i32), torch.zeros(3), torch.zeros(6, dtype=i32)[::2], [0, 0, 0]):
        with pytest.raises(ValueError):
            p.reserve(add, granted=bad)
    for first, second in ((both[:3], both[:3]), (both[:3], both[2:]), (both[2:], both[:3])):
        with pytest.raises(ValueError):
            p.reserve(first, granted=second)
    assert len(seen) == 2
