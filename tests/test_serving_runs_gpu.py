"""The serving kernels where a block walks a long run: several tiles of one item, several items, tokens of several batch entries, several heads.
(tests/test_serving_gpu.py has the small calls, in which every block has one of each.)  Sizes follow from the SM count, and each test asserts
that its call does give the blocks such runs."""
import math

import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import serving as S
from test_serving_gpu import FMTS, HALF, U, _bd, _cache, _check_rotary, _gen, _i32, _randn, _tree_bits

pytestmark = pytest.mark.gpu
TILE = 128


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _tiles_and_ctas(fmt, d, rows, kv, lengths):
    """128-key tiles of a call of tree attention, and how many blocks share them: by warps up to 16 rows per KV head (as many blocks an SM as
    their stages and registers allow, four at most), one block an SM beyond."""
    R = 16 if rows <= 16 else 32 if rows <= 32 else 64
    tiles = sum(max(1, -(-n // TILE)) for n in lengths) * kv * -(-rows // R)
    return tiles, _sms() * (4 if rows <= 16 else 1)


def _pool_values(cache):
    """K and V of every token of every page, fp64 on the device [pages, kv, P, d], from the places that the layout gives each element."""
    P, d, fmt = cache.page_size, cache.d, "nvfp4" if cache.fmt == 1 else "e4m3"
    kc, ks, vc, vs, shift = S.places(fmt, P, d)
    pages = cache.pages.cpu().numpy()
    out = []
    for codes, scales, G in ((kc, ks, cache.k_G), (vc, vs, cache.v_G)):
        if fmt == "e4m3":
            x = F.e4m3_decode(pages[..., codes])
        else:
            x = F.e2m1_decode(pages[..., codes] >> shift & 15) * np.repeat(F.e4m3_decode(pages[..., scales]), 16, axis=-1)
        out.append(torch.from_numpy(np.ascontiguousarray(x)).cuda() / G.double()[None, :, None, None])
    return out


def _check(got, q, cache, table, context, bits, pool, missing=None):
    """As _check_attention of tests/test_serving_gpu.py, by its bounds: out by 2 (ds + 2^-20 + n u) + 2^-11 of sum p |v|, 2^-32 a key of the
    largest |v| and its type's rounding; LSE by ds + 2^-20 + n u and fp32's rounding.  A reference that moves multiplies sum and O by one more
    factor of hardware exp2, 2^-21 and u, at most once per 128 keys: less than the 128 u that those keys add to n u."""
    B, H, T, d = q.shape
    kv = cache.k_G.numel()
    scale, dev = 1 / math.sqrt(d), q.device
    j = torch.arange(T, device=dev)
    for b in range(B):
        n = context[b] + T
        at = table[b, :-(-n // cache.page_size)].long()
        k, v = (x[at.clamp(min=0)].transpose(0, 1).flatten(1, 2)[:, :n] for x in pool)               # [kv, n, d]
        held = (at >= 0).repeat_interleave(cache.page_size)[:n]
        x = q[b].double().unflatten(0, (kv, -1))                                                    # [kv, group, T, d]
        z = torch.einsum("hgtd,hkd->hgtk", x, k) * scale
        mask = torch.ones(T, n, dtype=torch.bool, device=dev)
        mask[:, context[b]:] = (bits[b][:, None] >> j & 1) > 0 if bits is not None else j[None] <= j[:, None]
        mask &= held
        any_seen = mask.any(1)
        z = z.masked_fill(~mask, -math.inf)
        lse = torch.logsumexp(z, -1)
        p = torch.exp(z - lse[..., None]).masked_fill(~mask, 0.0)
        o, pv = torch.einsum("hgtk,hkd->hgtd", p, v), torch.einsum("hgtk,hkd->hgtd", p, v.abs())
        size = (torch.einsum("hgtd,hkd->hgtk", x.abs(), k.abs()) * scale).masked_fill(~mask, 0.0).amax(-1)
        ds = (d + 10) * U * size
        bound = HALF[q.dtype] * o.abs() + (2 * (ds + 2.0 ** -20 + n * U) + 2.0 ** -11)[..., None] * pv + n * 2.0 ** -32 * v.abs().max() + 2.0 ** -40
        out, l = got[0][b].double().unflatten(0, (kv, -1)), got[1][b].double().unflatten(0, (kv, -1))
        err = (out - o).abs()
        assert (err <= bound * (1 + 2.0 ** -8))[:, :, any_seen].all(), (b, (err - bound)[:, :, any_seen].max().item())
        lbound = ds + 2.0 ** -20 + n * U + 2 * U * (lse.abs() + 1 + size)
        assert ((l - lse).abs() <= lbound)[:, :, any_seen].all(), (b, ((l - lse).abs() - lbound)[:, :, any_seen].max().item())
        assert not out[:, :, ~any_seen].any() and torch.isneginf(l[:, :, ~any_seen]).all()


ROWS = [  # heads per KV head, drafted tokens: one and two groups of eight rows by warps, then tiles of 32, 64, and several of 64
    (1, 1), (4, 2), (8, 1), (3, 5), (16, 1), (2, 12), (32, 1), (1, 33), (4, 16), (5, 26), (4, 64)]


@pytest.mark.parametrize("runs", [3, 11, 40])
@pytest.mark.parametrize("group,T", ROWS)
@pytest.mark.parametrize("fmt,d,P", [("nvfp4", 128, 64), ("nvfp4", 64, 16), ("e4m3", 128, 128), ("e4m3", 64, 32)])
def test_tree_attention_long_runs(fmt, d, P, group, T, runs):
    """`runs` tiles a block and more, items of unlike lengths that begin and end inside the runs, some shorter than a tile; pages shared between
    sequences.  The longer the runs, the longer the items."""
    Bd, g, rng = _bd(), _gen(1000 * runs + 10 * group + T), np.random.default_rng(100 * runs + group + T)
    kv, rows, longest = 3, group * T, {3: 900, 11: 2500, 40: 6000}[runs]
    tiles, ctas, context = 0, 1, []
    while tiles < runs * ctas:
        context.append(int(rng.integers(0, longest)) if len(context) % 5 else int(rng.integers(0, 100)))
        tiles, ctas = _tiles_and_ctas(fmt, d, rows, kv, [c + T for c in context])
    B = len(context)
    assert tiles >= runs * ctas and runs > 2
    pool = 2 * (-(-(longest + T) // P))
    cache = _cache(Bd, fmt, pool, kv, P, d)
    everything = torch.arange(pool, device="cuda", dtype=torch.int32)[None]
    Bd.fp4attn_cache_write(cache, _randn(g, 1, kv, pool * P, d), _randn(g, 1, kv, pool * P, d), everything, _i32([0]))
    table = torch.stack([torch.randperm(pool, generator=g, device="cuda")[:pool // 2] for _ in range(B)]).to(torch.int32)
    dtype = torch.float16 if (group + T) % 2 else torch.bfloat16
    q = _randn(g, B, T, group * kv, d, dtype=dtype).transpose(1, 2)
    bits = _tree_bits(rng, B, T) if T % 3 else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits, status=status)
    assert status.item() == 0
    again = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    _check(got, q, cache, table, context, bits, _pool_values(cache))


@pytest.mark.parametrize("group,T", [(2, 3), (5, 3), (8, 3), (8, 6), (16, 8)])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64), ("nvfp4", 64), ("e4m3", 128)])
def test_tree_attention_references_that_move(fmt, d, group, T):
    """Logits that rise along the keys by some 14 octaves a tile (a row's reference is left behind by more than it may in every tile), fall
    (the maximum comes first), or do neither, rows of the three kinds side by side; every block walks several tiles of an item."""
    Bd, g = _bd(), _gen(70 + group + T)
    kv, P, rows = 2, 64, group * T
    length = 9 * TILE + 50
    need = 4 * _sms() * (4 if rows <= 16 else 1)
    B = -(-need // (10 * kv))
    context = [length - 3 * (b % 7) for b in range(B)]
    tiles, ctas = _tiles_and_ctas(fmt, d, rows, kv, [c + T for c in context])
    assert tiles >= 3 * ctas
    pool = -(-(length + T) // P)
    cache = _cache(Bd, fmt, pool, kv, P, d)
    u = torch.where(torch.rand(kv, 1, d, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    k = (u * torch.linspace(0.02, 4.4, length + T, device="cuda")[:, None]).to(torch.bfloat16)[None]
    everything = torch.arange(pool, device="cuda", dtype=torch.int32)[None]
    Bd.fp4attn_cache_write(cache, k.contiguous(), _randn(g, 1, kv, length + T, d), everything, _i32([0]))
    # a logit is c sqrt(d) times the key's size: 4.4 c sqrt(d) log2(e) octaves over ten tiles
    c = 140 / (4.4 * math.sqrt(d) * math.log2(math.e))
    kinds = torch.tensor([c, -c, 0.02 * c, 0.3 * c, 1e-3 * c], device="cuda")
    q = (u[:, None] * kinds[torch.arange(rows, device="cuda") % 5].view(1, group, T, 1)).flatten(0, 1)[None].expand(B, -1, -1, -1)
    q = (q + 0.01 * c * torch.randn(q.shape, generator=g, device="cuda")).to(torch.bfloat16)
    table = everything.expand(B, -1).contiguous()
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context))
    _check(got, q, cache, table, context, None, _pool_values(cache))


@pytest.mark.parametrize("group,T", [(1, 6), (2, 7), (1, 20), (3, 20), (4, 40)])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
def test_tree_attention_first_key_in_a_later_tile(fmt, d, group, T):
    """Contexts without pages for their first tiles, so that no row sees a key there; of the drafted tokens, which two tiles share, some rows see
    those of the first tile only, some those of the second, some none.  Several tiles of an item in a block."""
    Bd, g, rng = _bd(), _gen(90 + T), np.random.default_rng(T)
    kv, P, rows = 2, 16, group * T
    B = -(-4 * _sms() * (4 if rows <= 16 else 1) // (5 * kv))
    first = [5 * TILE - 2 - int(x) for x in rng.integers(0, T - 2, B)]                  # the drafted tokens cross into the sixth tile
    tiles, ctas = _tiles_and_ctas(fmt, d, rows, kv, [c + T for c in first])
    assert tiles >= 2 * ctas
    pool = -(-(5 * TILE + T) // P)
    cache = _cache(Bd, fmt, pool, kv, P, d)
    everything = torch.arange(pool, device="cuda", dtype=torch.int32)[None]
    Bd.fp4attn_cache_write(cache, _randn(g, 1, kv, pool * P, d), _randn(g, 1, kv, pool * P, d), everything, _i32([0]))
    table = everything.expand(B, -1).contiguous()
    kept = 4 * TILE // P
    for b in range(B):
        if b % 3 == 0:
            table[b, :first[b] // P] = -1                   # of the context, at most the last page's tokens (there where drafted tokens are)
        elif b % 3 == 1:
            table[b, :kept] = -1                            # the fifth tile is there
        else:
            table[b, ::2] = -1
    bits = torch.from_numpy(rng.integers(0, 2 ** min(T, 62), (B, T))).cuda()
    for t in range(T):
        if t % 4 == 1:
            bits[:, t] = 0
        if t % 4 == 2:
            bits[:, t] = 1 << (T - 1)
        if t % 4 == 3:
            bits[:, t] = 1
    q = _randn(g, B, group * kv, T, d)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32(first), tree_mask=bits, status=status)
    assert status.item() == Bd.ERR_PAGE
    _check(got, q, cache, table, first, bits, _pool_values(cache))


# ---------------------------------------------------------------- rotary and the rotated write
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("B,H,kv,N,d,pairs,interleaved", [(7, 2, 1, 343, 64, 32, False), (3, 3, 2, 1601, 128, 32, True), (9, 1, 1, 1001, 64, 30, False),
                                                          (9001, 1, 0, 1, 64, 8, True), (2, 5, 1, 4501, 64, 16, False), (1, 2, 1, 9001, 250, 125, True)])
def test_rotary_blocks_of_many_tokens(B, H, kv, N, d, pairs, interleaved, offset, dtype):
    """Up to four tokens a block, across the borders of batch entries, the last block partly filled."""
    Bd, g = _bd(), _gen(N)
    per = min(4, B * N // (8 * _sms()))
    assert per >= 2 and B * N % per
    flat = _randn(g, B * N * (H + kv) * d + 8, dtype=dtype)
    x = flat[offset:offset + B * N * (H + kv) * d].view(B, N, H + kv, d).transpose(1, 2)
    q, k = x[:, :H], x[:, H:] if kv else None
    pos, f = torch.randint(0, 1 << 17, (B, N), generator=g, device="cuda").to(torch.int32), Bd.fp4attn_rotary_frequencies(2 * pairs)
    for call, transposed in ((Bd.fp4attn_rotary, False), (Bd.fp4attn_rotary_backward, True)):
        got = call(q, pos, f, k=k, interleaved=interleaved)
        for y, z in zip(got if kv else [got], [q, k]):
            _check_rotary(y, z, pos, f, dtype, interleaved=interleaved, transposed=transposed)
    want = [y.clone() for y in (got if kv else [got])]
    Bd.fp4attn_rotary_backward(q, pos, f, k=k, interleaved=interleaved, q_out=q, k_out=k)
    assert all(torch.equal(a, b) for a, b in zip((q, k), want))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,kv,N,d,pairs,interleaved,positions", [(2, 5, 4001, 128, 64, False, False), (3, 7, 4005, 64, 28, True, True), (16, 11, 333, 128, 32, True, False),
                                                                  (1, 13, 9003, 64, 32, False, True)])
def test_rotated_write_of_several_heads_a_block(B, kv, N, d, pairs, interleaved, positions, fmt):
    """Heads that share the cosines and sines of their tokens, the last range of heads a part of one: the bytes of rotary followed by a plain
    write."""
    Bd, g = _bd(), _gen(N + kv)
    P = 32
    blocks = (N + 4096 // d - 2) // (4096 // d) + 1
    per = min(kv, blocks * B * kv // (4 * _sms()))
    assert per >= 2 and kv % per
    starts = [(37 * b) % 91 for b in range(B)]
    per_seq = -(-(N + 91) // P)
    table = torch.randperm(B * per_seq, generator=g, device="cuda").reshape(B, per_seq).to(torch.int32)
    k, v = _randn(g, B, N, kv, d).transpose(1, 2), _randn(g, B, kv, N, d)
    f = Bd.fp4attn_rotary_frequencies(2 * pairs)
    at = _i32(starts)[:, None] + torch.arange(N, device="cuda", dtype=torch.int32)
    if positions:
        at = torch.randint(0, 1 << 20, (B, N), generator=g, device="cuda").to(torch.int32)
    one, two = _cache(Bd, fmt, B * per_seq, kv, P, d), _cache(Bd, fmt, B * per_seq, kv, P, d)
    Bd.fp4attn_cache_write(one, k, v, table, _i32(starts), inv_freq=f, positions=at if positions else None, interleaved=interleaved)
    Bd.fp4attn_cache_write(two, Bd.fp4attn_rotary(k, at, f, interleaved=interleaved), v, table, _i32(starts))
    assert one.pages.any() and torch.equal(one.pages, two.pages)


@pytest.mark.parametrize("group,T", [(1, 5), (2, 8), (4, 8), (4, 16), (4, 40)])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
def test_tree_attention_rows_that_are_not_finite(fmt, d, group, T):
    """Queries with NaN and infinities: their own rows are NaN, the rows beside them right."""
    Bd, g, rng = _bd(), _gen(5 * T + group), np.random.default_rng(T)
    kv, P, rows = 2, 32, group * T
    need = 3 * _sms() * (4 if rows <= 16 else 1)
    B = -(-need // (5 * kv * -(-rows // 64)))
    context = [5 * TILE - int(x) for x in rng.integers(0, 100, B)]
    pool = -(-(5 * TILE + T) // P)
    cache = _cache(Bd, fmt, pool, kv, P, d)
    everything = torch.arange(pool, device="cuda", dtype=torch.int32)[None]
    Bd.fp4attn_cache_write(cache, _randn(g, 1, kv, pool * P, d), _randn(g, 1, kv, pool * P, d), everything, _i32([0]))
    table = everything.expand(B, -1).contiguous()
    q = _randn(g, B, group * kv, T, d)
    bad = q.clone()
    bad[:, 0, 1, 3], bad[:, 0, 3, 5], bad[:, -1, 0, 7], bad[:, -1, 4] = math.nan, math.inf, -math.inf, math.nan
    got = Bd.fp4attn_tree_attention(bad, cache, table, _i32(context))
    clean = Bd.fp4attn_tree_attention(q, cache, table, _i32(context))
    for h, t in ((0, 1), (0, 3), (group * kv - 1, 0), (group * kv - 1, 4)):
        assert torch.isnan(got[0][:, h, t]).all() and torch.isnan(got[1][:, h, t]).all(), (h, t)
        for x, y in zip(got, clean):
            x[:, h, t] = y[:, h, t]
    _check(got, q, cache, table, context, None, _pool_values(cache))
