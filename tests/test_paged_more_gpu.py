"""Attention of prompts and of shared prefixes over a paged cache: calls that padded and partly empty batches make, tensors that lie over one another."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from test_paged_gpu import _check_shared, _shared
from test_serving_gpu import _bd, _filled, _gen, _i32, _randn, _tree_bits

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


def _both(Bd, g, H, kv, T, d=64, P=16):
    """Calls of either operator that take q and the tensors of the caller's, of 2 sequences whose items fall to several blocks."""
    context = [700, 90]
    cache, table = _filled(Bd, g, "e4m3", 2, kv, P, d, max(context) + T)
    paged = lambda q, **kw: Bd.fp4attn_paged_attention(q, cache, table, _i32(context), **kw)
    capped = lambda q, **kw: Bd.fp4attn_paged_attention(q, cache, table, _i32(context), soft_cap=20.0, **kw)
    shared = lambda q, **kw: Bd.fp4attn_shared_prefix_attention(q, cache, table[:1], _i32([300]), _i32([0, 2]), table, _i32(context), **kw)
    return (paged, capped) + ((shared,) if T <= 64 else ())


def test_outputs_over_one_another():
    """Both outputs in one place, LSE over q, O over q in another order or shifted: rows would be overwritten that others have still to read, or twice."""
    Bd, g = _bd(), _gen(91)
    H, kv, T, d = 4, 2, 3, 64
    room = _randn(g, 4 * 2 * H * T * d)
    n = 2 * H * T * d
    q = room[:n].view(2, H, T, d)
    kept = room.clone()
    for call in _both(Bd, g, H, kv, T):
        lse = lambda at: room[at:at + 4 * H * T].view(torch.float32).view(2, H, T)
        for kw in (dict(out=room[8:n + 8].view(2, H, T, d)), dict(out=room[n - 8:2 * n - 8].view(2, H, T, d)), dict(lse=lse(0)), dict(lse=lse(n - 8)),
                   dict(out=room[n:2 * n].view(2, H, T, d), lse=lse(n)), dict(out=room[n:2 * n].view(2, H, T, d), lse=lse(2 * n - 8))):
            with pytest.raises(AssertionError, match="overlap"):
                call(q, **kw)
        with pytest.raises(AssertionError, match="overlap"):
            call(room[:n].view(2, T, H, d).transpose(1, 2), out=q)
        with pytest.raises(AssertionError, match="overlap"):
            call(q[:1].expand(2, H, T, d), out=q)
        assert torch.equal(room, kept)
        # side by side, and in the gaps of one another, nothing overlaps
        want = call(q)
        got = call(q, out=room[n:2 * n].view(2, H, T, d), lse=lse(2 * n))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        wide = torch.zeros(2, 3 * H * T * d, dtype=q.dtype, device="cuda")
        apart = wide[:, :H * T * d].unflatten(1, (H, T, d))
        apart.copy_(q)
        inside = wide[0, H * T * d:].view(2, H, T, d)
        assert torch.equal(call(apart, out=inside)[0], want[0])
        room.copy_(kept)


@pytest.mark.parametrize("T", [1, 7, 40, 200])
def test_outputs_over_the_queries_themselves(T):
    Bd, g = _bd(), _gen(T)
    for call in _both(Bd, g, 8, 2, T):
        q = _randn(g, 2, 8, T, 64)
        want = call(q)
        got = call(q, out=q)
        assert got[0] is q and torch.equal(q, want[0]) and torch.equal(got[1], want[1])


def test_a_page_released_twice_is_free_twice():
    """As documented: while other pages are held nobody notices, and two sequences get the page.  Of a page that two tables share, one lets go: the other
    keeps its first 16 tokens' pages."""
    Bd, P = _bd(), 16
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def shared():
        pool, table = Bd.fp4attn_pages_create(12, P), torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
        Bd.fp4attn_pages_assign(pool, table, _i32([0, 16, 0]), _i32([48, 16, 64]))
        table[1, 0] = table[0, 0]
        return pool, table

    for keep, left in (([0, 0, 64], 9), ([0, 16, 64], 8)):
        pool, table = shared()
        free, want = pool.free.tolist(), table.tolist()
        assert pool.count.item() == 4 and want == [[0, 1, 2, -1], [0, 3, -1, -1], [4, 5, 6, 7]]
        Bd.fp4attn_pages_release(pool, table, _i32([48, 32, 64]), keep=_i32(keep), status=status)
        assert S.pages_release(free, 4, want, [48, 32, 64], keep, P) == (left, True)
        assert status.item() == 0 and pool.count.item() == left and pool.free.tolist() == free and table.tolist() == want
        assert free[:left].count(0) == (2 if left == 9 else 1)
    # twice in two calls, with too little room on the stack for all of them: the ones that have none are reported
    Bd.fp4attn_pages_release(pool, table, _i32([0, 16, 64]), status=status)
    assert status.item() == Bd.ERR_PAGE and pool.count.item() == 12


@pytest.mark.parametrize("kw", [dict(), dict(soft_cap=9.0), dict(slopes=True), dict(soft_cap=9.0, slopes=True)], ids=["scaled", "capped", "biased", "both"])
@pytest.mark.parametrize("fmt", ["nvfp4", "e4m3"])
@pytest.mark.parametrize("T,P", [(1, 64), (6, 16), (33, 128)])
def test_shared_prefixes_what_nobody_sees(T, P, fmt, kw):
    """Bytes of every token that no row sees are 0xFF, NaN as an E4M3 code or scale: behind a prefix's and a sequence's last token, drafted tokens that no mask
    names, sequences without tokens, pages of nobody.  The same bits as with a cache that was written whole."""
    Bd, g, rng = _bd(), _gen(T + P), np.random.default_rng(T)
    H, kv, d = 4, 2, 64
    prefixes, starts, context = [333, 61, 0], [0, 3, 5, 6], [130, 0, 7, 64, 31, 5, 200]
    B, counts = len(context), [T, T, max(1, T - 2), T, 0, T, T]
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, P, d, prefixes, context, T)
    q = _randn(g, B, H, T, d)
    if kw.get("slopes"):
        kw = dict(kw, slopes=torch.tensor([0.5, 0.0, -0.01, 0.1], device="cuda"))
    for bits in (None, _tree_bits(rng, B, T) & torch.as_tensor(rng.integers(0, 2 ** 62, (B, 1)) | 1, device="cuda")):
        call = lambda c: Bd.fp4attn_shared_prefix_attention(q, c, prefix_table, _i32(prefixes), _i32(starts), table, _i32(context), tree_mask=bits, count=_i32(counts), **kw)
        want = call(cache)
        held = np.zeros((len(cache.pages), P), bool)                # tokens that some row sees
        for g_, n in enumerate(prefixes):
            for pos in range(n):
                held[int(prefix_table[g_, pos // P]), pos % P] = True
        for b in range(B):
            seen = set(range(context[b])) if counts[b] else set()
            for t in range(counts[b]):
                seen |= {context[b] + j for j in range(T) if (j <= t if bits is None else int(bits[b, t]) >> j & 1)}
            for pos in seen:
                held[int(table[b, pos // P]), pos % P] = True
        kc, ks, vc, vs, _ = S.places(fmt, P, d)
        raw = cache.pages.cpu().numpy().copy()
        for page, t in zip(*np.nonzero(~held)):
            for a in ([kc[t], vc[t]] if ks is None else [kc[t], ks[t], vs[t]]):
                raw[page][:, a] = 255
        got = call(Bd.QuantizedCache(torch.as_tensor(raw, device="cuda"), cache.k_G, cache.v_G, cache.fmt, P, d))
        assert torch.isfinite(want[0]).all()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
