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


def test_whole_numbers_beyond_32_bits():
    """2^32 + n is not n."""
    Bd, g = _bd(), _gen(2)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    start = _i32([3, 4])
    with pytest.raises(OverflowError):
        Bd.fp4attn_cache_read(cache, table, start, (1 << 32) + 3)
    q = _randn(g, 2, 4, 3, 64)
    for fmt, page in ((cache.fmt + (1 << 32), 16), (cache.fmt, 16 - (1 << 32))):
        wrong = Bd.QuantizedCache(cache.pages, cache.k_G, cache.v_G, fmt, page, 64)
        with pytest.raises(OverflowError):
            Bd.fp4attn_tree_attention(q, wrong, table, start)
    x = _randn(g, 1, 1, 128, 64)
    with pytest.raises(OverflowError):
        Bd.fp4attn_quantize(x, Bd.FMT_NVFP4 + (1 << 32), 0)


def test_outputs_over_one_another():
    """The same memory for both outputs, an output over the other input, or over its own in another order: rows would be overwritten while
    others are still read, or twice."""
    Bd, g = _bd(), _gen(3)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    f = Bd.fp4attn_rotary_frequencies(64)
    q, k, pos = _randn(g, 2, 2, 2, 64), _randn(g, 2, 2, 2, 64), _i32([[0, 1]] * 2)
    out, kept = torch.zeros_like(q), (q.clone(), k.clone())
    for call in (lambda: Bd.fp4attn_rotary(q, pos, f, k=k, q_out=out, k_out=out), lambda: Bd.fp4attn_rotary(q, pos, f, k=k, q_out=k),
                 lambda: Bd.fp4attn_rotary(q, pos, f, k=k, k_out=q), lambda: Bd.fp4attn_rotary(q, pos, f, k=k, q_out=k, k_out=q),
                 lambda: Bd.fp4attn_rotary(q, pos, f, q_out=q.transpose(1, 2)), lambda: Bd.fp4attn_rotary(q, pos, f, k=k, q_out=q, k_out=q),
                 lambda: Bd.fp4attn_cache_read(cache, table, _i32([3, 4]), 2, k_out=out, v_out=out)):
        with pytest.raises(AssertionError, match="overlap"):
            call()
    assert not out.any() and torch.equal(q, kept[0]) and torch.equal(k, kept[1])
    want = [x.clone() for x in Bd.fp4attn_rotary(q, pos, f, k=k)]
    Bd.fp4attn_rotary(q, pos, f, k=k, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
