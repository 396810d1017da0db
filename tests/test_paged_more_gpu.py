"""Attention of prompts and of shared prefixes over a paged cache: calls that padded and partly empty batches make, tensors that lie over one another."""
import pytest
import torch

from test_paged_gpu import _check_shared, _shared
from test_serving_gpu import _bd, _gen, _i32, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("members", [2, 40])
def test_a_prefix_of_sequences_without_tokens_is_nobodys_loss(members):
    """A batch padded to its size: sequences of no tokens behind a prefix whose pages have gone, or whose length its table has no room for.  No row would
    see them, so they are not reported; with one token behind the prefix they are.  40 members are two row tiles of a KV head."""
    Bd, g = _bd(), _gen(members)
    H, kv, T, d, P = 8, 2, 1, 64, 16
    prefixes, starts, context = [50, 70], [0, 3, 3 + members], [20, 0, 5] + [9] * members
    cache, prefix_table, table = _shared(Bd, g, "nvfp4", kv, P, d, prefixes, context, T)
    q = _randn(g, 3 + members, H, T, d)
    gone = prefix_table.clone()
    gone[1] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for lengths in (prefixes, [50, 1000]):
        counts = [1, 0, 1] + [0] * members
        got = Bd.fp4attn_shared_prefix_attention(q, cache, gone, _i32(lengths), _i32(starts), table, _i32(context), count=_i32(counts), status=status)
        assert status.item() == 0
        _check_shared(got, q, cache, gone, [50, 70], starts, table, context, counts=counts)
        for last in (3, 2 + members):
            counts = [1, 0, 1] + [0] * members
            counts[last] = 1
            Bd.fp4attn_shared_prefix_attention(q, cache, gone, _i32(lengths), _i32(starts), table, _i32(context), count=_i32(counts), status=status)
            assert status.item() == Bd.ERR_PAGE
            status.zero_()
