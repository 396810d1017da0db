"""What the binding's serving calls refuse, beside tests/test_serving_gpu.py, and in which words."""
import pytest
import torch

from test_serving_gpu import _bd, _filled, _gen, _i32, _randn

pytestmark = pytest.mark.gpu


def test_empty_batches_are_named():
    """No sequence, or no token: refused, and not with words about types and layouts."""
    Bd, g = _bd(), _gen(1)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    start, f = _i32([3, 4]), Bd.fp4attn_rotary_frequencies(64)
    for B, N in ((0, 3), (2, 0)):
        q, k, pos = _randn(g, B, 4, N, 64), _randn(g, B, 2, N, 64), torch.zeros(B, N, dtype=torch.int32, device="cuda")
        for call in (lambda: Bd.fp4attn_rotary(q, pos, f), lambda: Bd.fp4attn_rotary_backward(q, pos, f, k=k),
                     lambda: Bd.fp4attn_cache_write(cache, k, k, table[:B], start[:B]), lambda: Bd.fp4attn_cache_read(cache, table[:B], start[:B], N),
                     lambda: Bd.fp4attn_tree_attention(q, cache, table[:B], start[:B])):
            with pytest.raises(AssertionError, match="at least one sequence"):
                call()
