"""Prefill calls of more workgroups than a launch takes, or than the kernel can number, are refused on the host."""

import ctypes

import pytest

from paper_2605_30842_amd import binding as B

A = 1 << 20


def _call(plan, fp8, batch, most):
    lib = B.load_library()
    fn = lib.comem_prefill_fp8_attn if fp8 else lib.comem_prefill_attn_split
    ctx = 1 << 30
    status = fn(plan, A, A, A, most, A, A, 1024, 128, A, A, batch, ctx, A, None, None, 0, None)
    if not fp8:
        assert status == lib.comem_prefill_attn(plan, A, A, A, most, A, A, 1024, 128, A, A, batch, ctx, A, None, None)
    n = ctypes.c_size_t()
    size = (lib.comem_prefill_fp8_workspace if fp8 else lib.comem_prefill_attn_workspace)(plan, batch, most, ctx,
                                                                                          ctypes.byref(n))
    assert size == (B.OK if status == B.ERR_NO_DEVICE else status)
    return status


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_workgroups_of_a_call(fp8, group):
    plan, _ = B.comem_decode_attn_init(B.Config(num_q_heads=8 * group, num_kv_heads=8, head_dim=128,
                                                dtype=B.FP8_E4M3 if fp8 else B.BF16, scale=0.1, max_batch=65535,
                                                max_ctx_len=1 << 30, k_scale=1.0, v_scale=1.0), B.NO_DEVICE)
    tokens = 128 // group
    for batch in (1, 31, 4096, 65535):
        # 512 threads a workgroup, less than 2^32 along a dimension; 8 KV heads a sequence, numbers up to 2^31 - 1.
        blocks = min((1 << 23) - 1, ((1 << 31) - 1) // (8 * batch))
        most = min(blocks * tokens, 1 << 30)
        assert _call(plan, fp8, batch, most) == B.ERR_NO_DEVICE
        if most < 1 << 30:
            assert _call(plan, fp8, batch, most + 1) == B.ERR_INVALID_SHAPE
    B.comem_decode_attn_destroy(plan)
