"""Attention of prompts over a paged cache and of shared prefixes: what the library refuses or asks for, without a GPU."""
import pytest

from test_oracle_paged import SHAPE, WORKSPACE, _Cache, _paged, _shared, lib  # noqa: F401


@pytest.mark.parametrize("call", [_paged, _shared])
@pytest.mark.parametrize("kv", [1, 16])
def test_more_query_heads_than_the_kernels_divide_by(lib, call, kv):  # noqa: F811
    """A row's token and head come from a multiplication that is exact up to 2^16 heads of a KV head.  With 1048575 of them, heads from 1048561 on
    came out as heads -14 .. -1 of the next token: Q, O and LSE outside their rows."""
    cache = _Cache(0x1000, 0x2000, 0x2000, 1, 64, 10, kv, 128)
    for group in (65536, 1048575) if kv == 1 else (65536,):
        assert call(lib, cache=cache, H=kv * group, T=1) == SHAPE
        assert lib.fp4attn_paged_attention_workspace_bytes(1, kv * group, kv, 1, 128) == 0
        assert lib.fp4attn_shared_prefix_attention_workspace_bytes(1, kv * group, kv, 1, 128, 1) == 0
    # the most that there may be get as far as the next check
    assert call(lib, cache=cache, H=kv * 65535, T=1, bytes=0) == WORKSPACE


def test_token_and_head_by_a_multiplication():
    """The division as the kernels make it, at every number that it gets, for heads of every size class up to the most."""
    import numpy as np
    for d in [1, 2, 3, 5, 7, 8, 12, 40, 64, 127, 255, 256, 257, 4095, 4097, 32767, 65521, 65534, 65535]:
        n = np.arange(d + 256, dtype=np.uint64)
        assert np.array_equal(n * np.uint64(-(-2 ** 36 // d)) >> np.uint64(36), n // np.uint64(d))
    for d in range(1, 65):                                          # tokens of a call; of a group
        n = np.arange(65535 * d + 256, dtype=np.uint64)[:: 1 if d < 4 else 61]
        assert np.array_equal(n * np.uint64(-(-2 ** 36 // d)) >> np.uint64(36), n // np.uint64(d))


@pytest.mark.parametrize("B,kv", [(1, 1), (32, 8), (5, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_workspace_of_a_step_is_that_of_the_kernel_that_runs(lib, d, B, kv):  # noqa: F811
    """Rows of a KV head that go to the kernel of warps whatever the format and the masks: two partial results (O, maximum, sum) of its row tile per block."""
    for group, T in ((1, 1), (4, 1), (8, 1), (4, 2), (1, 7)) + (((16, 1), (9, 1), (4, 3)) if d == 64 else ()):
        R = 8 if group * T <= 8 else 16
        n = lib.fp4attn_paged_attention_workspace_bytes(B, group * kv, kv, T, d)
        assert 0 < n <= 2 * 640 * R * (4 * d + 8) + 8 * B * kv + 32
    # with more of them no call may ask for less than 128 rows in lanes leave
    for rows in (17, 33, 64, 200):
        assert lib.fp4attn_paged_attention_workspace_bytes(B, kv, kv, rows, d) >= 2 * 148 * 128 * (4 * d + 8)
    assert lib.fp4attn_paged_attention_workspace_bytes(B, 9 * kv, kv, 1, 128) >= 2 * 148 * 128 * (4 * 128 + 8)          # NVFP4 with a mask
