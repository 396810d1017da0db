"""Rotary positions, the quantized paged cache and tree attention against the fp64 oracle.

Tolerances.  A type's rounding is off by at most half a step, eps / 2 of the value.  u = 2^-24 is fp32's.
"""
import math

import numpy as np
import pytest
import torch

from oracle import serving as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: U}
FMTS = ["nvfp4", "e4m3"]


def _bd():
    from paper_2609_04105_b200 import binding as Bd
    return Bd


def _np(t):
    return t.detach().double().cpu().numpy()


def _randn(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (scale * torch.randn(shape, generator=gen, device="cuda")).to(dtype)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- rotary
def _check_rotary(got, x, positions, freq, dtype, **kw):
    """cos and sin are within 2^-50 of theirs before they are rounded; two products and a sum, each rounded: at most (u + u + u)
    (|x1| + |x2|) factor to first order, then the type's rounding of the result."""
    want = S.rotary(_np(x), _np(positions), freq.cpu().numpy(), **kw)
    rot = 2 * freq.numel()
    pairs = S.rotary(np.abs(_np(x)), 0 * _np(positions), freq.cpu().numpy(), factor=abs(kw.get("factor", 1.0)), interleaved=kw.get("interleaved", False))
    size = np.zeros_like(want)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if kw.get("interleaved") else (i, i + rot // 2)
    size[..., a] = size[..., b] = pairs[..., a] + pairs[..., b]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0                               # half a step of a subnormal
    bound = HALF[dtype] * np.abs(want) + (3 * U + 2.0 ** -45) * (1 + 2 * HALF[dtype]) * size + tiny
    bound[..., rot:] = 0.0
    assert (np.abs(_np(got) - want) <= bound).all(), np.max(np.abs(_np(got) - want) - bound)


ROTARY = [  # B, H, kv, N, d, pairs, interleaved
    (2, 4, 2, 5, 128, 64, False), (1, 3, 1, 1, 64, 16, True), (3, 2, 2, 77, 64, 28, False), (2, 5, 1, 33, 128, 30, True),
    (1, 1, 0, 300, 64, 32, False), (1, 2, 1, 3, 250, 125, False), (1, 2, 1, 9, 6, 1, False), (2, 8, 8, 129, 256, 128, True),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("B,H,kv,N,d,pairs,interleaved", ROTARY)
def test_rotary(B, H, kv, N, d, pairs, interleaved, dtype):
    Bd, g = _bd(), _gen(B * 1000 + N)
    q = _randn(g, B, H, N, d, dtype=dtype)
    k = _randn(g, B, kv, N, d, dtype=dtype) if kv else None
    pos = torch.randint(0, 1 << 20, (B, N), generator=g, device="cuda").to(torch.int32)
    pos[0, 0] = 0
    f = Bd.fp4attn_rotary_frequencies(2 * pairs)
    for transposed in (False, True):
        call = Bd.fp4attn_rotary_backward if transposed else Bd.fp4attn_rotary
        got = call(q, pos, f, k=k, interleaved=interleaved, attention_factor=1.25)
        for y, x in zip(got if kv else [got], [q, k] if kv else [q]):
            assert y.dtype == dtype and y.shape == x.shape
            _check_rotary(y, x, pos, f, dtype, interleaved=interleaved, transposed=transposed, factor=1.25)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_rotary_strides_alignment_in_place(interleaved, offset):
    """Q and K as slices of one projection, at addresses that 16-byte accesses can and cannot use; then in place; then broadcast."""
    Bd, g = _bd(), _gen(5)
    B, H, kv, N, d = 2, 3, 1, 19, 64
    flat = _randn(g, B * N * (H + kv) * d + 8)
    x = flat[offset:offset + B * N * (H + kv) * d].view(B, N, (H + kv), d).transpose(1, 2)
    q, k = x[:, :H], x[:, H:]
    pos, f = _i32([list(range(N)), list(range(100, 100 + N))]), Bd.fp4attn_rotary_frequencies(48)
    want = [t.clone() for t in Bd.fp4attn_rotary(q.contiguous(), pos, f, k=k.contiguous(), interleaved=interleaved)]
    got = Bd.fp4attn_rotary(q, pos, f, k=k, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    before = flat.clone()
    again = Bd.fp4attn_rotary(q, pos, f, k=k, interleaved=interleaved, q_out=q, k_out=k)
    assert again[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(flat[:offset], before[:offset]) and torch.equal(flat[offset + B * N * (H + kv) * d:], before[offset + B * N * (H + kv) * d:])
    one = _randn(g, 1, 1, N, d).expand(B, H, N, d)
    assert torch.equal(Bd.fp4attn_rotary(one, pos, f, interleaved=interleaved), Bd.fp4attn_rotary(one.contiguous(), pos, f, interleaved=interleaved))
    with pytest.raises(AssertionError, match="output"):
        Bd.fp4attn_rotary(one, pos, f, q_out=one)                                      # would write one element many times


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient(interleaved):
    """Against the formula's through autograd in 64 bits, and against differences (the map is linear: any step is exact but for
    rounding, 2^-24 of the values on each side of a difference over 1)."""
    Bd, g = _bd(), _gen(6)
    B, H, N, d, pairs = 1, 2, 7, 64, 24
    x, dy = _randn(g, B, H, N, d, dtype=torch.float32), _randn(g, B, H, N, d, dtype=torch.float32)
    pos, f = _i32([[3, 1, 4, 100000, 5, 9, 2]]), Bd.fp4attn_rotary_frequencies(2 * pairs)
    dx = Bd.fp4attn_rotary_backward(dy, pos, f, interleaved=interleaved, attention_factor=0.7)
    z = x.double().requires_grad_()
    th = pos.double()[:, None, :, None] * f.double()
    a, b = (z[..., :2 * pairs:2], z[..., 1:2 * pairs:2]) if interleaved else (z[..., :pairs], z[..., pairs:2 * pairs])
    c, s = 0.7 * th.cos(), 0.7 * th.sin()
    p, r = a * c - b * s, b * c + a * s
    y = torch.cat((torch.stack((p, r), -1).flatten(-2) if interleaved else torch.cat((p, r), -1), z[..., 2 * pairs:]), -1)
    y.backward(dy.double())
    assert (dx.double() - z.grad).abs().max() <= 4 * U * 2 * dy.abs().max()
    for e in (0, 1, 23, 24, 40, 47, 63):
        up, down = x.clone(), x.clone()
        up[0, 1, 3, e] += 0.5
        down[0, 1, 3, e] -= 0.5
        diff = (Bd.fp4attn_rotary(up, pos, f, interleaved=interleaved, attention_factor=0.7).double() -
                Bd.fp4attn_rotary(down, pos, f, interleaved=interleaved, attention_factor=0.7).double())
        step = float(up[0, 1, 3, e].double() - down[0, 1, 3, e].double())
        assert abs((diff * dy.double()).sum().item() / step - dx[0, 1, 3, e].item()) <= 64 * U * 5 * dy.abs().max().item()


# ---------------------------------------------------------------- the cache
def _cache(Bd, fmt, pages, kv, P, d, k_max=4.5, v_max=4.5, fill=None):
    full = 2688.0 if fmt == "nvfp4" else 448.0
    scale = torch.linspace(1.0, 1.5, kv, device="cuda")
    cache = Bd.fp4attn_cache_create(pages, P, d, Bd.FMT_NVFP4 if fmt == "nvfp4" else Bd.FMT_E4M3, full / (k_max * scale), full / (v_max / scale))
    if fill is not None:
        cache.pages.fill_(fill)
    return cache


def _table(gen, B, per_seq, pages):
    return torch.randperm(pages, generator=gen, device="cuda")[:B * per_seq].reshape(B, per_seq).to(torch.int32)


def _same_bytes(got, want, fmt, P, d):
    """Equal but for the sign of a zero code."""
    kc, ks, vc, vs, _ = S.places(fmt, P, d)
    got, want = got.copy(), want.copy()
    for at in (kc, vc):
        i = np.unique(at)
        for x in (got, want):
            b = x[..., i]
            if fmt == "nvfp4":
                b = np.where(b & 0x0F == 0x08, b & 0xF0, b)
                b = np.where(b & 0xF0 == 0x80, b & 0x0F, b)
            else:
                b = np.where(b == 0x80, 0, b)
            x[..., i] = b
    return np.array_equal(got, want)


CACHE = [  # B, kv, N, d, P, starts, counts
    (1, 1, 1, 128, 64, [0], None),
    (2, 2, 1, 64, 16, [15, 16], None),
    (3, 2, 37, 128, 32, [0, 5, 31], None),
    (2, 3, 50, 64, 128, [100, 127], [50, 7]),
    (4, 1, 20, 128, 16, [3, 0, 16, 9], [0, 20, 1, 19]),
    (1, 4, 129, 64, 64, [63], None),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,kv,N,d,P,starts,counts", CACHE)
def test_cache_write_bytes_and_read(B, kv, N, d, P, starts, counts, fmt, dtype):
    """Every byte of the pages, those of other tokens among them; then the values: exact but for the product by fl(1 / G) (two
    roundings of fp32) and the type's rounding."""
    Bd, g = _bd(), _gen(N + d)
    per_seq = -(-(max(starts) + N) // P)
    cache = _cache(Bd, fmt, B * per_seq + 2, kv, P, d, fill=0x35)
    table = _table(g, B, per_seq, B * per_seq + 2)
    k = _randn(g, B, N, kv, d, dtype=dtype).transpose(1, 2)                            # token by token, as a projection leaves it
    v = _randn(g, B, kv, N, d, dtype=dtype)
    k[0, 0, 0, :16] = 0.0
    k[0, 0, 0, 16] = 1000.0                                                            # beyond the calibrated range: saturates
    count = None if counts is None else _i32(counts)
    want = cache.pages.cpu().numpy().copy()
    kG, vG = cache.k_G.cpu().numpy(), cache.v_G.cpu().numpy()
    assert S.write(want, _np(k), _np(v), table.tolist(), starts, counts, kG, vG, fmt, P)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Bd.fp4attn_cache_write(cache, k, v, table, _i32(starts), count=count, status=status)
    assert _same_bytes(cache.pages.cpu().numpy(), want, fmt, P, d)
    got = Bd.fp4attn_cache_read(cache, table, _i32(starts), N, count=count, dtype=dtype, status=status)
    assert status.item() == 0
    for b in range(B):
        n = N if counts is None else counts[b]
        for h in range(kv):
            vals = S.values(want, table[b].tolist(), h, starts[b] + n, kG, vG, fmt, P, d)
            for y, x in zip(got, vals):
                x = x[starts[b]:]
                err = np.abs(_np(y[b, h, :n]) - x)
                assert (err <= (HALF[dtype] + 3 * U) * np.abs(x) + (2.0 ** -25 if dtype == torch.float16 else 0.0)).all()
                assert not y[b, h, n:].any()                                           # a tensor of the call's own: zero behind the count
    out = [torch.full((B, N, kv, d), 7.0, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    Bd.fp4attn_cache_read(cache, table, _i32(starts), N, count=count, dtype=dtype, k_out=out[0], v_out=out[1])
    for y, x in zip(out, got):
        for b in range(B):
            n = N if counts is None else counts[b]
            assert torch.equal(y[b, :, :n], x[b, :, :n]) and (y[b, :, n:] == 7.0).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("pairs,interleaved,d", [(64, False, 128), (32, True, 64), (16, False, 64), (28, False, 64), (30, True, 128), (16, True, 128)])
def test_cache_write_rotates_as_rotary_does(pairs, interleaved, d, fmt):
    Bd, g = _bd(), _gen(pairs)
    B, kv, N, P = 2, 3, 21, 16
    starts = [30, 100000 % 41]
    table = _table(g, B, 4, 9)
    k, v = _randn(g, B, N, kv, d).transpose(1, 2), _randn(g, B, kv, N, d)
    f = Bd.fp4attn_rotary_frequencies(2 * pairs)
    for positions in (None, torch.randint(0, 1 << 20, (B, N), generator=g, device="cuda").to(torch.int32)):
        at = positions if positions is not None else _i32(starts)[:, None] + torch.arange(N, device="cuda", dtype=torch.int32)
        one, two = _cache(Bd, fmt, 9, kv, P, d), _cache(Bd, fmt, 9, kv, P, d)
        Bd.fp4attn_cache_write(one, k, v, table, _i32(starts), inv_freq=f, positions=positions, interleaved=interleaved, attention_factor=0.9)
        Bd.fp4attn_cache_write(two, Bd.fp4attn_rotary(k, at, f, interleaved=interleaved, attention_factor=0.9), v, table, _i32(starts))
        assert one.pages.any() and torch.equal(one.pages, two.pages)


@pytest.mark.parametrize("fmt", FMTS)
def test_cache_token_by_token_equals_at_once(fmt):
    """Also: odd addresses (no 16-byte accesses), and NaN, infinities, subnormals, ties."""
    Bd, g = _bd(), _gen(9)
    B, kv, N, d, P = 2, 2, 35, 128, 32
    table, starts = _table(g, B, 3, 7), [13, 29]
    flat = _randn(g, 2 * B * kv * N * d + 1)
    k, v = flat[1:].view(2, B, kv, N, d)
    k[0, 0, 3, :8] = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-40, 1e38, -1.0], device="cuda")
    v[1, 1, 4, 20] = math.nan
    one, two = _cache(Bd, fmt, 7, kv, P, d), _cache(Bd, fmt, 7, kv, P, d)
    Bd.fp4attn_cache_write(one, k, v, table, _i32(starts))
    for n in range(N):
        Bd.fp4attn_cache_write(two, k[:, :, n:n + 1], v[:, :, n:n + 1], table, _i32([s + n for s in starts]))
    assert torch.equal(one.pages, two.pages)
    want = np.zeros_like(one.pages.cpu().numpy())
    S.write(want, _np(k), _np(v), table.tolist(), starts, None, one.k_G.cpu().numpy(), one.v_G.cpu().numpy(), fmt, P)
    assert _same_bytes(one.pages.cpu().numpy(), want, fmt, P, d)
    for y in Bd.fp4attn_cache_read(one, table, _i32(starts), N):
        assert torch.isfinite(y).all()


def test_cache_tokens_without_a_page():
    """Entries that name no page, positions outside the table, starts below 0: skipped, reported, nothing else touched; read as zero."""
    Bd, g = _bd(), _gen(10)
    B, kv, N, d, P = 5, 1, 40, 64, 16
    table = _i32([[0, 1, 2], [3, -1, 4], [5, 99, 6], [7, 8, 9], [10, 11, 12]])
    starts = [0, 0, 0, 20, -20]
    k, v = _randn(g, B, kv, N, d), _randn(g, B, kv, N, d)
    cache = _cache(Bd, "nvfp4", 13, kv, P, d, fill=0x21)
    want = cache.pages.cpu().numpy().copy()
    assert not S.write(want, _np(k), _np(v), table.tolist(), starts, None, cache.k_G.cpu().numpy(), cache.v_G.cpu().numpy(), "nvfp4", P)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Bd.fp4attn_cache_write(cache, k, v, table, _i32(starts), status=status)
    assert status.item() == Bd.ERR_PAGE and _same_bytes(cache.pages.cpu().numpy(), want, "nvfp4", P, d)
    status.zero_()
    got = Bd.fp4attn_cache_read(cache, table, _i32(starts), N, status=status)[0]
    assert status.item() == Bd.ERR_PAGE
    assert not got[1, 0, 16:32].any() and got[1, 0, 32:].any() and not got[3, 0, 28:].any() and not got[4, 0, :20].any() and got[4, 0, 20:].any()
    for extreme in ([2 ** 31 - 1] * B, [-2 ** 31] * B):
        before = cache.pages.clone()
        Bd.fp4attn_cache_write(cache, k, v, table, _i32(extreme))
        assert torch.equal(cache.pages, before)
        assert not Bd.fp4attn_cache_read(cache, table, _i32(extreme), N)[0].any()


# ---------------------------------------------------------------- attention
def _check_attention(got, q, cache, table, context, bits, counts=None, scale=None, unseen=()):
    """With size = the largest sum of |q k| scale over a row's keys: a score is off by d sums in fp32 and a few roundings of its
    constant, ds = (d + 8) u size; exp2 by 2^-21 and the rounding of its argument, 2 u |z| <= 2 u size; a probability by the f16
    rounding, 2^-11, or half a step of f16's subnormals, 2^-25 of at least 2^-7 of the largest; a sum of n terms in fp32, in any order, by (n - 1) u of the sum of their
    magnitudes.  These enter numerator and sum, so O is off by 2 (ds + 2^-20 + n u) + 2^-11 of sum p |v| and 2^-32 a key of max |v|, then
    by its type's rounding; LSE by ds + 2^-20 + n u and fp32's rounding."""
    out, lse = (_np(x) for x in got)
    B, H, T, d = q.shape
    kv = cache.k_G.numel()
    P, fmt = cache.page_size, "nvfp4" if cache.fmt == 1 else "e4m3"
    pages, kG, vG = cache.pages.cpu().numpy(), cache.k_G.cpu().numpy(), cache.v_G.cpu().numpy()
    scale = scale or 1 / math.sqrt(d)
    for b in range(B):
        n = T if counts is None else counts[b]
        ctx = max(0, context[b])
        for h in range(kv):
            k, v, held = S.values(pages, table[b].tolist(), h, ctx + T, kG, vG, fmt, P, d)
            mask = S.seen(ctx, T, None if bits is None else [int(x) & (2 ** 64 - 1) for x in bits[b]], held)
            for j in unseen:
                mask[:, j] = False
            for hq in range(h * (H // kv), (h + 1) * (H // kv)):
                o, l, pv, size = S.attend(_np(q[b, hq]), k, v, mask, scale)
                ds = (d + 10) * U * size[:, None]
                bound = HALF[q.dtype] * np.abs(o) + (2 * (ds + 2.0 ** -20 + len(held) * U) + 2.0 ** -11) * pv + len(held) * 2.0 ** -32 * np.abs(v).max(initial=0.0) + 2.0 ** -40
                err = np.abs(out[b, hq] - o)
                assert (err[:n] <= bound[:n] * (1 + 2.0 ** -8)).all(), (b, hq, np.max(err[:n] - bound[:n]))
                a = l[:n]
                fine = np.isfinite(a)
                assert np.array_equal(np.isneginf(lse[b, hq, :n]), ~fine) and not out[b, hq, :n][~fine].any()
                assert (np.abs(lse[b, hq, :n][fine] - a[fine]) <= (ds[:n, 0] + 2.0 ** -20 + len(held) * U + 2 * U * (np.abs(a) + 1 + size[:n]))[fine]).all()


def _filled(Bd, gen, fmt, B, kv, P, d, length, extra_pages=2):
    per_seq = -(-length // P)
    cache = _cache(Bd, fmt, B * per_seq + extra_pages, kv, P, d)
    table = _table(gen, B, per_seq, B * per_seq + extra_pages)
    k, v = _randn(gen, B, kv, length, d), _randn(gen, B, kv, length, d)
    Bd.fp4attn_cache_write(cache, k, v, table, _i32([0] * B))
    return cache, table


def _tree_bits(rng, B, T):
    rows = []
    for _ in range(B):
        bits = []
        for t in range(T):
            p = int(rng.integers(-1, t)) if t else -1
            bits.append((bits[p] if p >= 0 else 0) | 1 << t)
        rows.append([x - (1 << 64) if x >> 63 else x for x in bits])
    return torch.tensor(rows, dtype=torch.int64, device="cuda")


TREE = [  # B, H, kv, T, d, P, contexts
    (1, 1, 1, 1, 128, 64, [0]),
    (1, 4, 1, 1, 64, 16, [1]),
    (2, 8, 2, 1, 128, 64, [127, 128]),
    (3, 6, 2, 3, 64, 32, [0, 61, 300]),
    (2, 5, 1, 7, 128, 128, [250, 121]),
    (2, 4, 4, 16, 64, 16, [17, 1000]),
    (1, 16, 2, 64, 128, 64, [513]),
    (2, 40, 1, 13, 128, 32, [90, 0]),
    (1, 3, 3, 64, 64, 16, [0]),
    (5, 2, 1, 2, 128, 16, [5, 2000, 0, 64, 700]),
    (1, 2, 1, 1, 128, 64, [20011]),
    (2, 9, 1, 1, 128, 16, [333, 129]),
    (1, 3, 1, 5, 64, 128, [1025]),
    (2, 8, 1, 64, 64, 128, [200, 66]),
    (1, 24, 2, 33, 128, 16, [127]),
    (40, 2, 2, 1, 64, 16, [(37 * i) % 300 for i in range(40)]),
    (35, 5, 1, 5, 128, 32, [(91 * i) % 200 for i in range(35)]),
    (1030, 1, 1, 1, 64, 16, [i % 19 for i in range(1030)]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,H,kv,T,d,P,context", TREE)
def test_tree_attention(B, H, kv, T, d, P, context, fmt, dtype):
    Bd, g = _bd(), _gen(H * T + d)
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, max(context) + T)
    q = _randn(g, B, T, H, d, dtype=dtype, scale=2.0).transpose(1, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bits in (None, _tree_bits(np.random.default_rng(T), B, T)):
        got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits, status=status)
        assert got[0].dtype == dtype and got[0].shape == q.shape and got[1].shape == q.shape[:3]
        _check_attention(got, q, cache, table, context, None if bits is None else bits.tolist())
    assert status.item() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_tree_attention_empty_rows_counts_and_what_nobody_sees(fmt):
    """Rows whose mask leaves nothing; rows behind a count; unseen bytes of every kind, NaN codes and scales among them, inside the last
    page, in the tokens that no row sees and in pages that belong to nobody."""
    Bd, g = _bd(), _gen(21)
    B, H, kv, T, d, P = 4, 4, 2, 5, 128, 32
    context = [0, 30, 0, 200]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 210)
    bits = torch.tensor([[0, 1, 0, 5, 16], [0, 0, 4, 0, 1], [0, 0, 0, 0, 0], [31, 16, 0, 1, 2]], dtype=torch.int64, device="cuda")
    q = _randn(g, B, H, T, d)
    want = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits)
    _check_attention(want, q, cache, table, context, bits.tolist())
    assert not want[0][2].any() and torch.isneginf(want[1][2]).all() and not want[0][0, :, 0].any()
    # everything from context + T on, and everything that the table does not name
    used = torch.zeros(cache.pages.shape[0], dtype=torch.bool, device="cuda")
    for b in range(B):
        last = -(-(context[b] + T) // P)
        used[table[b, :last].long()] = True
    cache.pages[~used] = 0xFF
    kc, ks, vc, vs, _ = S.places(fmt, P, d)
    for b in range(B):
        end = context[b] + T
        page = int(table[b, (end - 1) // P])
        for t in range((end - 1) % P + 1, P):
            for at in (kc, ks, vc, vs):
                if at is not None:
                    cache.pages[page, :, torch.from_numpy(np.unique(at[t])).cuda()] = 0xFF
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    counts = [5, 0, 3, 2]
    out, lse = torch.full_like(want[0], 9.0), torch.full_like(want[1], 9.0)
    Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits, count=_i32(counts), out=out, lse=lse)
    own = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=bits, count=_i32(counts))
    for b, n in enumerate(counts):
        assert torch.equal(out[b, :, :n], want[0][b, :, :n]) and torch.equal(lse[b, :, :n], want[1][b, :, :n])
        assert (out[b, :, n:] == 9.0).all() and (lse[b, :, n:] == 9.0).all()
        assert not own[0][b, :, n:].any() and torch.isneginf(own[1][b, :, n:]).all()


@pytest.mark.parametrize("H", [4, 40])
@pytest.mark.parametrize("fmt", FMTS)
def test_tree_attention_drafted_tokens_that_were_not_written(fmt, H):
    """Behind a count, and where no row's bit is set, the drafted tokens' bytes may be anything too: other rows are as without them."""
    Bd, g = _bd(), _gen(26)
    B, kv, T, d, P = 3, 2, 6, 64, 16
    context, counts = [40, 0, 125], [3, 6, 1]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 140)
    q = _randn(g, B, H, T, d)
    bits = torch.tensor([[1, 3, 7, 15, 31, 63], [1, 3, 1, 1, 3, 1], [1, 3, 5, 9, 17, 33]], dtype=torch.int64, device="cuda")
    for mask in (None, bits):
        want = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=mask, count=_i32(counts))
        kept = cache.pages.clone()
        kc, ks, vc, vs, _ = S.places(fmt, P, d)
        for b in range(B):
            unseen = [j for j in range(T) if j >= counts[b] or (mask is not None and not any(int(x) >> j & 1 for x in bits[b, :counts[b]]))]
            for j in unseen:
                pos = context[b] + j
                for at in (kc, ks, vc, vs):
                    if at is not None:
                        cache.pages[int(table[b, pos // P]), :, torch.from_numpy(np.unique(at[pos % P])).cuda()] = 0xFF
        got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), tree_mask=mask, count=_i32(counts))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        cache.pages.copy_(kept)


@pytest.mark.parametrize("H", [4, 40])
@pytest.mark.parametrize("fmt", FMTS)
def test_tree_attention_padded_batch(fmt, H):
    """Entries without rows need no pages and no context of sense; pages behind a count need not exist.  Nothing of that is an error, and
    the other entries are as without them; a page missing below a count is reported."""
    Bd, g = _bd(), _gen(27)
    B, kv, T, d, P = 4, 2, 6, 128, 16
    context, counts = [46, 2 ** 31 - 1, 128, 31], [2, 0, 6, 1]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 144)
    q = _randn(g, B, H, T, d)
    bits = torch.tensor([[1, 3, 7, 15, 31, 63]] * B, dtype=torch.int64, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    few = table.clone()
    few[0, 3:] = -1                                             # position 48: the third drafted token
    few[1] = -1
    few[3, 2:] = 1 << 30
    for mask in (None, bits):
        got = Bd.fp4attn_tree_attention(q, cache, few, _i32(context), tree_mask=mask, count=_i32(counts), status=status)
        assert status.item() == 0
        for b in (0, 2, 3):
            alone = Bd.fp4attn_tree_attention(q[b:b + 1], cache, table[b:b + 1], _i32(context[b:b + 1]), tree_mask=None if mask is None else mask[b:b + 1],
                                              count=_i32(counts[b:b + 1]))
            for x, y in zip(got, alone):
                # Other splits of the keys: other references, so other roundings of each probability, by 2^-11 of it on either side,
                # 2^-10 of sum p |v| and of the sum together 2^-9 max |v| <= 2^-6 (|v| < 6 here); then bf16's on either side, 2^-7 of the value
                assert torch.allclose(x[b].float(), y[0].float(), rtol=2.0 ** -7, atol=2.0 ** -6)
        assert not got[0][1].any() and torch.isneginf(got[1][1]).all()
        few[3, 1] = -1
        Bd.fp4attn_tree_attention(q, cache, few, _i32(context), tree_mask=mask, count=_i32(counts), status=status)
        assert status.item() == Bd.ERR_PAGE
        status.zero_()
        few[3, 1] = table[3, 1]
    # nobody there at all
    out, lse = Bd.fp4attn_tree_attention(q, cache, torch.full_like(table, -1), _i32([7] * B), count=_i32([0, -3, 0, 0]), status=status)
    assert status.item() == 0 and not out.any() and torch.isneginf(lse).all()


def test_tree_attention_extreme_logits_and_queries():
    """Logits of thousands (one key takes all), rows of unlike sizes side by side, tiny and zero queries, a scale of the caller's."""
    Bd, g = _bd(), _gen(22)
    B, H, kv, T, d, P = 1, 8, 1, 4, 128, 64
    cache, table = _filled(Bd, g, "nvfp4", B, kv, P, d, 700)
    q = _randn(g, B, H, T, d)
    q[0, 1] *= 1000.0
    q[0, 2] *= 1e-6
    q[0, 3] = 0.0
    q[0, 4] *= 1e-30
    q[0, 5, :, 1:] = 0.0
    q[0, 6, 2] *= 300.0
    for context in ([0], [640], [696]):
        for scale in (0.0, 0.3):
            got = Bd.fp4attn_tree_attention(q, cache, table, _i32(context), softmax_scale=scale)
            _check_attention(got, q, cache, table, context, None, scale=scale)


def test_tree_attention_growing_logits():
    """Keys whose logits rise along the sequence: the running maximum moves in every tile."""
    Bd, g = _bd(), _gen(23)
    kv, P, d, length = 1, 64, 64, 1500
    cache = _cache(Bd, "e4m3", 24, kv, P, d)
    table = torch.arange(24, device="cuda", dtype=torch.int32)[None]
    u = torch.randn(d, generator=g, device="cuda")
    k = (u * torch.linspace(0.01, 1.0, length, device="cuda")[:, None]).to(torch.bfloat16)[None, None]
    v = _randn(g, 1, 1, length, d)
    Bd.fp4attn_cache_write(cache, k, v, table, _i32([0]))
    q = (u * torch.tensor([[-30.0], [5.0], [30.0]], device="cuda")).to(torch.bfloat16)[None, None].expand(1, 2, 3, d)
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32([1490]))
    _check_attention(got, q, cache, table, [1490], None)


def test_tree_attention_tokens_without_a_page():
    Bd, g = _bd(), _gen(24)
    B, H, kv, T, d, P = 2, 2, 1, 3, 64, 16
    cache, table = _filled(Bd, g, "nvfp4", B, kv, P, d, 300)
    q = _randn(g, B, H, T, d)
    broken = table.clone()
    broken[0, 3], broken[0, 8], broken[1, 0] = -1, cache.pages.shape[0], 1 << 30
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_tree_attention(q, cache, broken, _i32([200, 20]), status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_attention(got, q, cache, broken, [200, 20], None)
    status.zero_()
    # a context that reaches behind the table, and one below 0
    got = Bd.fp4attn_tree_attention(q, cache, table, _i32([302, -7]), status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_attention(got, q, cache, table, [302, -7], None)
    for extreme in ([2 ** 31 - 1, 5], [5, -2 ** 31]):
        status.zero_()
        got = Bd.fp4attn_tree_attention(q, cache, table, _i32(extreme), status=status)
        one = 1 if extreme[1] < 0 else 0
        want = Bd.fp4attn_tree_attention(q, cache, table, _i32([5, 0] if one else [5, 5]))
        keep = slice(0, 2) if one else slice(1, 2)
        assert torch.equal(got[0][keep], want[0][keep])
        assert status.item() == (0 if one else Bd.ERR_PAGE)


def test_cache_beyond_four_gigabytes():
    """Pages whose offsets pass 32 bits."""
    Bd, g = _bd(), _gen(25)
    kv, P, d = 8, 128, 128
    record = S.record_bytes("e4m3", P, d)
    pages = (1 << 32) // (record * kv) + 40
    G = torch.full((kv,), 100.0, device="cuda")
    cache = Bd.QuantizedCache(torch.empty((pages, kv, record), dtype=torch.uint8, device="cuda"), G, G, Bd.FMT_E4M3, P, d)
    small = Bd.fp4attn_cache_create(4, P, d, Bd.FMT_E4M3, G, G)
    k, v = _randn(g, 1, kv, 400, d), _randn(g, 1, kv, 400, d)
    q = _randn(g, 1, 16, 2, d)
    results = []
    for c, table in ((cache, _i32([[pages - 1, pages - 3, 2, pages - 30]])), (small, _i32([[0, 1, 2, 3]]))):
        Bd.fp4attn_cache_write(c, k, v, table, _i32([0]))
        results.append([*Bd.fp4attn_cache_read(c, table, _i32([0]), 400), *Bd.fp4attn_tree_attention(q, c, table, _i32([398]))])
    assert all(torch.equal(a, b) for a, b in zip(*results))


# ---------------------------------------------------------------- together, as a program uses them
def _step(Bd, s):
    """Positions on Q, K rotated into the cache, attention over it."""
    q = Bd.fp4attn_rotary(s["q"], s["positions"], s["f"])
    Bd.fp4attn_cache_write(s["cache"], s["k"], s["v"], s["table"], s["start"], inv_freq=s["f"], positions=s["positions"])
    return Bd.fp4attn_tree_attention(q, s["cache"], s["table"], s["start"], tree_mask=s["bits"])


def _step_state(Bd, seed, fmt="nvfp4", T=6):
    g = _gen(seed)
    B, H, kv, d, P = 3, 8, 2, 128, 16
    starts = [37, 250, 0]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 260)
    rng = np.random.default_rng(seed)
    bits = _tree_bits(rng, B, T)
    depth = torch.tensor([[bin(x & (2 ** 64 - 1)).count("1") - 1 for x in row] for row in bits.tolist()], device="cuda")
    return {"q": _randn(g, B, H, T, d), "k": _randn(g, B, kv, T, d), "v": _randn(g, B, kv, T, d), "cache": cache, "table": table,
            "start": _i32(starts), "starts": starts, "bits": bits, "positions": (_i32(starts)[:, None] + depth).to(torch.int32),
            "f": Bd.fp4attn_rotary_frequencies(d)}


@pytest.mark.parametrize("fmt", FMTS)
def test_step_of_a_drafted_tree(fmt):
    """Rotary, write and attention in a row against the oracle in a row; then the accepted branch alone, token by token, gives what the
    tree gave its last token."""
    Bd = _bd()
    s = _step_state(Bd, 31, fmt)
    want = s["cache"].pages.cpu().numpy().copy()
    f, pos = s["f"].cpu().numpy(), _np(s["positions"])
    rotated = [torch.from_numpy(S.rotary(_np(s[x]), pos, f)).to(torch.bfloat16).cuda() for x in ("q", "k")]
    got = _step(Bd, s)
    qk = Bd.fp4attn_rotary(s["q"], s["positions"], s["f"], k=s["k"])
    assert all((a.float() - b.float()).abs().max() <= 2.0 ** -8 * b.float().abs().max() for a, b in zip(qk, rotated))
    S.write(want, _np(qk[1]), _np(s["v"]), s["table"].tolist(), s["starts"], None, s["cache"].k_G.cpu().numpy(), s["cache"].v_G.cpu().numpy(), fmt, 16)
    assert _same_bytes(s["cache"].pages.cpu().numpy(), want, fmt, 16, 128)
    _check_attention(got, qk[0], s["cache"], s["table"], s["starts"], s["bits"].tolist())
    b, last = 1, 5
    branch = [j for j in range(6) if int(s["bits"][b, last]) >> j & 1]
    start, table = s["start"][b:b + 1], s["table"][b:b + 1]
    for i, j in enumerate(branch):
        at = start + i
        Bd.fp4attn_cache_write(s["cache"], s["k"][b:b + 1, :, j:j + 1], s["v"][b:b + 1, :, j:j + 1], table, at, inv_freq=s["f"])
        q = Bd.fp4attn_rotary(s["q"][b:b + 1, :, j:j + 1], at[:, None].contiguous(), s["f"])
        one = Bd.fp4attn_tree_attention(q, s["cache"], table, at)
    # the same keys in another order: twice what one result may be off by
    assert (one[0].float() - got[0][b:b + 1, :, last:].float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -10) * got[0].float().abs().max()
    assert torch.allclose(one[1], got[1][b:b + 1, :, last:], rtol=0, atol=1e-4)


def test_step_repeats_captures_and_runs_beside_another():
    """The same bits every time: again, captured into graphs and replayed (two graphs whose workspaces are one pool's, in turn and at
    once), on a stream of its own beside another's."""
    Bd = _bd()
    states = [_step_state(Bd, 41), _step_state(Bd, 42, "e4m3", T=3)]
    want = [[x.clone() for x in _step(Bd, s)] for s in states]
    for s, w in zip(states, want):
        assert all(torch.equal(a, b) for a, b in zip(_step(Bd, s), w))
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(_step(Bd, s))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(x, want[i % 2]))
    graphs, outs = [], []
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(_step(Bd, s))
        graphs.append(graph)
    for _ in range(3):
        for o in outs:
            for x in o:
                x.zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
    # new contents in the captured inputs
    states[0]["q"].copy_(_randn(_gen(77), *states[0]["q"].shape))
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], _step(Bd, states[0])))


def test_binding_refuses_tensors_of_another_shape():
    """As many elements in another order of the axes are another tensor."""
    Bd, g = _bd(), _gen(52)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    start, f = _i32([3, 4]), Bd.fp4attn_rotary_frequencies(64)
    q, k, pos = _randn(g, 2, 4, 3, 64), _randn(g, 2, 2, 3, 64), _i32([[0, 1, 2]] * 2)
    bits = torch.ones(2, 3, dtype=torch.int64, device="cuda")
    for call in (lambda: Bd.fp4attn_tree_attention(q, cache, table, start, out=torch.empty_like(q.transpose(1, 2).contiguous())),
                 lambda: Bd.fp4attn_tree_attention(q, cache, table, start, lse=torch.empty(2, 3, 4, device="cuda")),
                 lambda: Bd.fp4attn_tree_attention(q, cache, table, start, tree_mask=bits.t().contiguous()),
                 lambda: Bd.fp4attn_rotary(q, pos.t().contiguous(), f), lambda: Bd.fp4attn_rotary(q, pos.flatten(), f),
                 lambda: Bd.fp4attn_cache_write(cache, k, k, table, start, inv_freq=f, positions=pos.t().contiguous())):
        with pytest.raises(AssertionError):
            call()


def test_binding_refusals_on_the_device():
    Bd, g = _bd(), _gen(51)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    start = _i32([3, 4])
    k = _randn(g, 2, 2, 3, 64)
    q = _randn(g, 2, 4, 3, 64)
    pos = _i32([[0, 1, 2]] * 2)
    f = Bd.fp4attn_rotary_frequencies(64)
    bad = [lambda: Bd.fp4attn_cache_write(cache, k.float(), k, table, start), lambda: Bd.fp4attn_cache_write(cache, k, k.half(), table, start),
           lambda: Bd.fp4attn_cache_write(cache, k, k, table.long(), start), lambda: Bd.fp4attn_cache_write(cache, k, k, table, start.long()),
           lambda: Bd.fp4attn_cache_write(cache, k, k, table[:1], start), lambda: Bd.fp4attn_cache_write(cache, k, k, table, start[:1]),
           lambda: Bd.fp4attn_cache_write(cache, k[:, :1], k[:, :1], table, start), lambda: Bd.fp4attn_cache_write(cache, k.transpose(2, 3), k, table, start),
           lambda: Bd.fp4attn_cache_write(cache, k, k, table, start, positions=pos), lambda: Bd.fp4attn_cache_write(cache, k, k, table, start, inv_freq=f.double()),
           lambda: Bd.fp4attn_cache_write(cache, k, k, table.cpu(), start), lambda: Bd.fp4attn_cache_write(cache, k, k, table, start, status=start),
           lambda: Bd.fp4attn_cache_read(cache, table, start, 0), lambda: Bd.fp4attn_cache_read(cache, table, start, 3, k_out=k[:1]),
           lambda: Bd.fp4attn_cache_read(cache, table, start, 3, k_out=k[:, :, :1].expand(2, 2, 3, 64)),
           lambda: Bd.fp4attn_cache_read(cache, table, start, 3, dtype=torch.float16, k_out=k),
           lambda: Bd.fp4attn_tree_attention(q[:, :3], cache, table, start), lambda: Bd.fp4attn_tree_attention(q.float(), cache, table, start),
           lambda: Bd.fp4attn_tree_attention(q, cache, table, start, tree_mask=pos), lambda: Bd.fp4attn_tree_attention(q, cache, table, start, out=q.half()),
           lambda: Bd.fp4attn_tree_attention(q, cache, table, start, out=q.transpose(1, 2)), lambda: Bd.fp4attn_tree_attention(q, cache, table, start, lse=q),
           lambda: Bd.fp4attn_tree_attention(q[..., :32], cache, table, start),
           lambda: Bd.fp4attn_rotary(q, pos.long(), f), lambda: Bd.fp4attn_rotary(q, pos[:1], f), lambda: Bd.fp4attn_rotary(q, pos, f, k=k[:1]),
           lambda: Bd.fp4attn_rotary(q, pos, f, k_out=k), lambda: Bd.fp4attn_rotary(q, pos, f, q_out=q[:, :2]), lambda: Bd.fp4attn_rotary(q[0], pos, f)]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: Bd.fp4attn_rotary(q, pos, torch.ones(33, device="cuda")),
                 lambda: Bd.fp4attn_cache_write(cache, k, k, table, start, inv_freq=torch.ones(33, device="cuda")),
                 lambda: Bd.fp4attn_tree_attention(_randn(g, 2, 4, 65, 64), cache, table, start)):
        with pytest.raises(Bd.Fp4AttnError, match="unsupported shape"):
            call()
    with pytest.raises(Bd.Fp4AttnError):
        Bd.fp4attn_tree_attention(q, cache, table, start, softmax_scale=-1.0)
    wrong = Bd.QuantizedCache(cache.pages, cache.k_G, cache.v_G, Bd.FMT_E4M3, 16, 64)
    with pytest.raises(AssertionError, match="record"):
        Bd.fp4attn_cache_read(wrong, table, start, 3)
