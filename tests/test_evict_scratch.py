"""When the wrapper asks for a keep call's workspace, and when the library would use one (no device)."""

import pytest

from paper_2605_30842_amd import binding as B


@pytest.mark.parametrize("dtype,d", [(B.F32, 64), (B.BF16, 128)])
def test_the_wrapper_asks_wherever_the_library_would_use_one(dtype, d):
    p, _ = B.comem_decode_attn_init(B.Config(num_q_heads=8, num_kv_heads=8, head_dim=d, dtype=dtype, scale=0.1, max_batch=4,
                                             max_ctx_len=1 << 30), B.NO_DEVICE)
    bound = B.KEEP_CHUNKS_MIN_CTX
    for n in range(1, 40):
        assert all(B.comem_keep_tokens_workspace(p, n, length) == 0 for length in (0, 1, bound // 2, bound - 1, bound))
    assert B.comem_keep_tokens_workspace(p, 1, bound + 1) > 0
    B.comem_decode_attn_destroy(p)
