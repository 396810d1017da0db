"""Every byte of a cache through the kernels' conversions, wherever in a word it stands and whatever stands beside it: rows that see one key
each, so that O is that key's V exactly and LSE its score alone."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as S
from test_serving_gpu import U, _bd, _gen, _i32, _randn
from test_serving_runs_gpu import _pool_values

pytestmark = pytest.mark.gpu
FORMATS = [("nvfp4", 128, 64), ("nvfp4", 64, 16), ("e4m3", 128, 16), ("e4m3", 64, 128)]
SHAPES = [(1, 7), (2, 8), (1, 32), (1, 61), (4, 64)]                  # heads per KV head, tokens: an instance of the kernels each


def _random_cache(Bd, gen, fmt, pages, kv, P, d):
    """All 256 bytes of codes, all finite bytes of E4M3; factors of 1."""
    G = torch.ones(kv, device="cuda")
    cache = Bd.fp4attn_cache_create(pages, P, d, Bd.FMT_NVFP4 if fmt == "nvfp4" else Bd.FMT_E4M3, G, G)
    finite = torch.tensor([b for b in range(256) if b & 127 != 127], dtype=torch.uint8, device="cuda")
    kc, ks, vc, vs, _ = (None if x is None else torch.from_numpy(np.unique(x)).cuda() for x in S.places(fmt, P, d))
    for at, among in ((kc, None if fmt == "nvfp4" else finite), (vc, None if fmt == "nvfp4" else finite), (ks, finite[:127]), (vs, finite[:127])):
        if at is not None:
            x = torch.randint(0, 256 if among is None else len(among), (pages, kv, len(at)), generator=gen, device="cuda")
            cache.pages[:, :, at] = x.to(torch.uint8) if among is None else among[x]
    return cache


def _assert_covered(cache, tokens, k=True):
    """The bytes of these tokens (numbers in the pool) have all values in all four places of a word, in K and in V."""
    P, fmt = cache.page_size, "nvfp4" if cache.fmt == 1 else "e4m3"
    kc, _, vc, _, _ = S.places(fmt, P, cache.d)
    pages = cache.pages.cpu().numpy()
    for at in (kc, vc) if k else (vc,):
        seen = set()
        for t in tokens:
            where = at[t % P]
            seen.update(zip((where % 4).tolist() * pages.shape[1], pages[t // P][:, where].reshape(-1).tolist()))
        assert len(seen) == 4 * (256 if fmt == "nvfp4" else 254)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group,T", SHAPES)
@pytest.mark.parametrize("fmt,d,P", FORMATS)
def test_every_byte_of_drafted_tokens(fmt, d, P, group, T, dtype):
    """A row sees one drafted token, some tokens are seen by no row (their bytes are NaN), no context.  O: the value itself, which has six bits at most:
    its one probability is off by the rounding of the reference, 2^-24 of a score of less than 2^11 octaves, and 16 bits round that away (half
    a step is 2^-12 of the value or more).  LSE: one score, d products summed in fp32, (d + 10) u of their magnitudes as in _check_attention,
    and its own few roundings."""
    Bd, g, rng = _bd(), _gen(T + group), np.random.default_rng(T + d)
    kv, per_seq = 2, -(-T // P)
    B = -(-(600 if fmt == "e4m3" else 900) // (T * (d // 64)))
    cache = _random_cache(Bd, g, fmt, B * per_seq, kv, P, d)
    table = torch.randperm(B * per_seq, generator=g, device="cuda").reshape(B, per_seq).to(torch.int32)
    sees = np.stack([np.resize(rng.permutation(T)[:max(1, T - T // 3)], T) for _ in range(B)])       # two thirds of the tokens
    bits = torch.tensor([[(1 << int(j)) - (1 << 64 if j == 63 else 0) for j in row] for row in sees], dtype=torch.int64, device="cuda")
    pool = _pool_values(cache)
    tokens = [int(table[b, j // P]) * P + j % P for b in range(B) for j in np.unique(sees[b]).tolist()]
    _assert_covered(cache, tokens)
    pages = cache.pages.cpu().numpy()
    for at in S.places(fmt, P, d)[:4]:
        for t in set(range(B * per_seq * P)) - set(tokens):
            if at is not None:
                pages[t // P, :, at[t % P]] = 0xFF if t % 2 else 0x7F
    cache.pages.copy_(torch.from_numpy(pages))
    q = _randn(g, B, group * kv, T, d, dtype=dtype, scale=2.0 ** -4)
    out, lse = Bd.fp4attn_tree_attention(q, cache, table, _i32([0] * B), tree_mask=bits)
    at = table.long().gather(1, torch.from_numpy(sees // P).cuda()) * P + torch.from_numpy(sees % P).cuda()       # [B, T]
    k, v = (x.transpose(0, 1).flatten(1, 2)[:, at].transpose(0, 1) for x in pool)                               # [B, kv, T, d]
    x = q.double().unflatten(1, (kv, group))
    assert torch.equal(out.double().unflatten(1, (kv, group)), v[:, :, None].expand_as(x))
    assert (x.abs() * k[:, :, None].abs()).sum(-1).max() / math.sqrt(d) * math.log2(math.e) < 2 ** 11
    z, size = (x * k[:, :, None]).sum(-1) / math.sqrt(d), (x.abs() * k[:, :, None].abs()).sum(-1) / math.sqrt(d)
    assert ((lse.double().unflatten(1, (kv, group)) - z).abs() <= (d + 10) * U * size + 2.0 ** -20 + 2 * U * (z.abs() + 1 + size)).all()


@pytest.mark.parametrize("group,T", SHAPES)
@pytest.mark.parametrize("fmt,d,P", FORMATS)
def test_every_byte_of_whole_tiles_of_a_context(fmt, d, P, group, T):
    """Keys of signs, queries that are one key's signs: its score is above any other's by more than 64 octaves, which no probability or sum holds beside
    it, so that O is that key's V (as above, scores below 2^11 octaves).  The keys stand in whole tiles of the context."""
    Bd, g, rng = _bd(), _gen(3 * T + group), np.random.default_rng(T)
    kv, context = 1, 256
    per_seq = -(-(context + T) // P)
    B = -(-(800 if fmt == "e4m3" else 1100) // (T * group * (d // 64)))
    cache = _random_cache(Bd, g, fmt, B * per_seq, kv, P, d)
    kc, ks, _, _, _ = S.places(fmt, P, d)
    signs = torch.randint(0, 2, (B * per_seq, kv, P, d), generator=g, device="cuda").to(torch.uint8)
    if fmt == "nvfp4":                                                   # +-6 times 448
        cache.pages[:, :, torch.from_numpy(kc[:, ::2]).cuda()] = (0x77 + 8 * signs[..., ::2] + 128 * signs[..., 1::2]).to(torch.uint8)
        cache.pages[:, :, torch.from_numpy(ks).cuda()] = 0x7E
    else:
        cache.pages[:, :, torch.from_numpy(kc).cuda()] = (0x7E + 128 * signs).to(torch.uint8)
    table = torch.randperm(B * per_seq, generator=g, device="cuda").reshape(B, per_seq).to(torch.int32)
    k, v = (x.transpose(0, 1).flatten(1, 2)[0] for x in _pool_values(cache))                                     # [tokens, d]
    target = torch.from_numpy(rng.integers(0, context, (B, group * T))).cuda()
    at = table.long().gather(1, target // P) * P + target % P
    _assert_covered(cache, at.flatten().tolist(), k=False)
    q = (torch.sign(k[at]) * 2.0 ** (-6 if fmt == "nvfp4" else -3)).to(torch.bfloat16).view(B, group, T, d)
    # a key's score against another's: they differ in many of d signs
    z = torch.einsum("brd,bnd->brn", q.double().view(B, -1, d), k[(table.long()[:, :, None] * P + torch.arange(P, device="cuda")).flatten(1)[:, :context + T]]) / math.sqrt(d)
    top = z.topk(2, -1).values
    assert ((top[..., 0] - top[..., 1]) * math.log2(math.e) > 64).all() and (top[..., 0] * math.log2(math.e) < 2 ** 11).all()
    out, lse = Bd.fp4attn_tree_attention(q, cache, table, _i32([context] * B))
    assert torch.equal(out.double().view(B, -1, d), v[at])
    assert ((lse.double().view(B, -1) - top[..., 0]).abs() <= (d + 14) * U * top[..., 0] + 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fmt,d,P", FORMATS)
def test_every_byte_read_back(fmt, d, P, dtype):
    Bd, g = _bd(), _gen(8)
    pages = -(-2048 // P)
    cache = _random_cache(Bd, g, fmt, pages, 2, P, d)
    _assert_covered(cache, range(pages * P))
    table = torch.randperm(pages, generator=g, device="cuda")[None].to(torch.int32)
    for start, n in ((0, pages * P), (3, 1001)):
        got = Bd.fp4attn_cache_read(cache, table, _i32([start]), n, dtype=dtype)
        for y, x in zip(got, _pool_values(cache)):
            assert torch.equal(y[0].double(), x[table[0].long()].transpose(0, 1).flatten(1, 2)[:, start:start + n])
