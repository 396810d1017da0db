"""Attention of prompts over the paged cache and of batches that share prefixes, and pages from a pool, against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import serving as S
from test_serving_gpu import FMTS, HALF, U, _bd, _cache, _filled, _gen, _i32, _randn, _tree_bits

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- the oracle's side: oracle/serving.py's attend_scores, in fp64 on the device
def _table(decode, n):
    return torch.tensor(np.asarray(decode(np.arange(n, dtype=np.uint8)), dtype=np.float64), device="cuda")


def _values(cache, row, length):
    """S.values of all heads: K, V float64 [kv, length, d], and which positions have a page."""
    P, d, fmt = cache.page_size, cache.d, "nvfp4" if cache.fmt == 1 else "e4m3"
    at = [None if x is None else torch.as_tensor(np.ascontiguousarray(x), device="cuda").long() for x in S.places(fmt, P, d)]
    kc, ks, vc, vs, shift = at
    row = row[:max(1, -(-length // P))].long()
    there = (row >= 0) & (row < len(cache.pages))
    rec = cache.pages[torch.where(there, row, 0)].transpose(0, 1)                            # [kv, pages, bytes]
    byte = _table(F.e4m3_decode, 256)
    if fmt == "e4m3":
        k, v = byte[rec[:, :, kc].long()], byte[rec[:, :, vc].long()]
    else:
        code = _table(F.e2m1_decode, 16)
        k = code[rec[:, :, kc].long() >> shift & 15] * byte[rec[:, :, ks].long()].repeat_interleave(16, -1)
        v = code[rec[:, :, vc].long() >> shift & 15] * byte[rec[:, :, vs].long()].repeat_interleave(16, -1)
    held = there.repeat_interleave(P)
    n = min(length, len(held))
    pad = lambda x, shape: torch.cat((x, torch.zeros(shape, dtype=x.dtype, device="cuda")), x.dim() - 2 if x.dim() > 1 else 0)
    kv = cache.k_G.numel()
    out = [pad(x.flatten(1, 2)[:, :n] / G.double()[:, None, None], (kv, length - n, d)) for x, G in ((k, cache.k_G), (v, cache.v_G))]
    return *out, pad(held[:n], (length - n,))


def _check(got, q, kv, keys_of, n_of, scale=0.0, cap=0.0, slopes=None):
    """keys_of(b) -> K, V [kv, keys, d], mask [T, keys], distances [T, keys].

    With size = the largest sum of |q k| scale over a row's keys, far = the largest slope * distance: a score is off by d sums in fp32 and a few
    roundings of its constant, (d + 8) u size; by 2^-20 of the cap where there is one (whose slope is at most 1); by the roundings of the bias and
    of its sum, 8 u far.  All that is ds.  exp2 is off by 2^-21 and the rounding of its argument, 2 u (size + far); a probability by the f16 rounding,
    2^-11, or half a step of f16's subnormals, 2^-25 of at least 2^-7 of the largest; a sum of n terms in fp32, in any order, by (n - 1) u of the
    sum of their magnitudes.  These enter numerator and sum, so O is off by 2 (ds + 2^-20 + n u) + 2^-11 of sum p |v| and 2^-32 a key of max |v|,
    then by its type's rounding; LSE by ds + 2^-20 + n u and fp32's rounding."""
    B, H, T, d = q.shape
    scale, bad = scale or 1 / math.sqrt(d), []
    for b in range(B):
        n = n_of(b)
        k, v, mask, far = keys_of(b)
        used = mask.any(0)[None, :, None]
        k, v = torch.where(used, k, 0.0), torch.where(used, v, 0.0)
        x = q[b].double().unflatten(0, (kv, H // kv))                                        # [kv, group, T, d]
        z = torch.einsum("hgtd,hkd->hgtk", x, k) * scale
        size = torch.where(mask, torch.einsum("hgtd,hkd->hgtk", x.abs(), k.abs()) * scale, 0.0)
        size = size.amax(-1) if size.shape[-1] else size.sum(-1)
        if cap:
            z = cap * torch.tanh(z / cap)
        reach = torch.zeros_like(size)
        if slopes is not None:
            slope = slopes.double().view(kv, -1, 1, 1)
            z = z - slope * far
            reach = (slope.abs() * torch.where(mask, far, 0.0)).amax(-1) if z.shape[-1] else reach
        z = torch.where(mask, z, -math.inf)
        seen = mask.any(-1).expand(size.shape)
        top = z.amax(-1) if z.shape[-1] else torch.full_like(size, -math.inf)
        p = torch.exp(z - torch.where(seen, top, 0.0)[..., None])
        total = p.sum(-1)
        p = p / torch.where(seen, total, 1.0)[..., None]
        o, pv = torch.einsum("hgtk,hkd->hgtd", p, v), torch.einsum("hgtk,hkd->hgtd", p, v.abs())
        lse = top + torch.log(total)
        ds = (d + 10) * U * size + 2.0 ** -20 * cap + 8 * U * reach
        keys = k.shape[1]
        most = v.abs().amax() if v.numel() else 0.0
        bound = HALF[q.dtype] * o.abs() + (2 * (ds[..., None] + 2.0 ** -20 + keys * U) + 2.0 ** -11) * pv + keys * 2.0 ** -32 * most + 2.0 ** -40
        out, l = got[0][b].double().unflatten(0, (kv, -1)), got[1][b].double().unflatten(0, (kv, -1))
        fine = (out - o).abs() <= bound * (1 + 2.0 ** -8)
        fine &= torch.where(seen, (l - lse).abs() <= ds + 2.0 ** -20 + keys * U + 2 * U * (lse.abs() + 1 + size + reach), torch.isneginf(l))[..., None]
        fine &= seen[..., None] | (out == 0)
        bad.append((~fine[:, :, :n]).sum())
    bad = torch.stack(bad).tolist()
    assert not any(bad), [(b, x) for b, x in enumerate(bad) if x][:8]


def _check_paged(got, q, cache, table, context, counts=None, first=None, last=None, unseen=(), **kw):
    T = q.shape[2]
    n_of = lambda b: T if counts is None else min(max(counts[b], 0), T)

    def keys_of(b):
        ctx, n = max(0, context[b]), n_of(b)
        mask = S.between(ctx, T, n, None if first is None else first[b], None if last is None else last[b])
        k, v, held = _values(cache, table[b], ctx + n)
        at = torch.arange(ctx + n, device="cuda")
        return k, v, torch.as_tensor(mask, device="cuda") & held, (ctx + torch.arange(T, device="cuda")[:, None] - at).abs().double()

    _check(got, q, cache.k_G.numel(), keys_of, n_of, **kw)


def _check_shared(got, q, cache, prefix_table, prefix_length, group_start, table, context, bits=None, counts=None, **kw):
    T = q.shape[2]
    n_of = lambda b: T if counts is None else min(max(counts[b], 0), T)

    def keys_of(b):
        group = [g for g in range(len(prefix_length)) if group_start[g] <= b < group_start[g + 1]]
        before = max(0, prefix_length[group[0]]) if group else 0
        ctx, n = max(0, context[b]), n_of(b)
        k, v, held = _values(cache, table[b], ctx + T)
        seen = S.seen(ctx, T, None if bits is None else [int(x) & (2 ** 64 - 1) for x in bits[b]], held.cpu().numpy())
        if bits is None:
            seen[:, ctx + n:] = False
        mask = torch.as_tensor(seen, device="cuda")
        if before:
            kp, vp, hp = _values(cache, prefix_table[group[0]], before)
            k, v, mask = torch.cat((kp, k), 1), torch.cat((vp, v), 1), torch.cat((hp.expand(T, -1), mask), 1)
        far = before + ctx + torch.arange(T, device="cuda")[:, None] - torch.arange(before + ctx + T, device="cuda")
        return k, v, mask, far.abs().double()

    _check(got, q, cache.k_G.numel(), keys_of, n_of, **kw)


# ---------------------------------------------------------------- prompts
PAGED = [  # B, H, kv, T, d, P, contexts, counts
    (1, 1, 1, 1, 128, 64, [0], None),
    (1, 4, 1, 1, 64, 16, [1], None),
    (2, 8, 2, 1, 128, 64, [127, 128], None),
    (3, 6, 2, 3, 64, 32, [0, 61, 300], [3, 0, 2]),
    (2, 5, 1, 7, 128, 128, [250, 121], None),
    (1, 16, 2, 64, 128, 64, [513], None),
    (1, 8, 2, 65, 64, 16, [0], None),
    (2, 4, 2, 127, 128, 32, [3, 200], [127, 5]),
    (1, 4, 1, 128, 128, 128, [0], None),
    (1, 1, 1, 129, 64, 64, [1], None),
    (2, 6, 2, 257, 128, 16, [40, 0], [200, 257]),
    (1, 3, 3, 300, 64, 32, [77], None),
    (1, 40, 1, 33, 128, 64, [90], None),
    (5, 2, 1, 2, 128, 16, [5, 2000, 0, 64, 700], None),
    (1, 2, 1, 1, 128, 64, [20011], None),
    (1, 8, 1, 700, 128, 64, [1500], None),
    (1, 4, 4, 1100, 64, 128, [0], None),
    (3, 16, 2, 200, 64, 64, [1000, 30, 0], [200, 77, 1]),
    (40, 2, 2, 3, 64, 16, [(37 * i) % 300 for i in range(40)], [i % 4 for i in range(40)]),
    (1030, 1, 1, 1, 64, 16, [i % 19 for i in range(1030)], None),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,H,kv,T,d,P,context,counts", PAGED)
def test_paged_attention(B, H, kv, T, d, P, context, counts, fmt, dtype):
    Bd, g = _bd(), _gen(H * T + d)
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, max(context) + T)
    q = _randn(g, B, T, H, d, dtype=dtype, scale=2.0).transpose(1, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), count=None if counts is None else _i32(counts), status=status)
    assert got[0].dtype == dtype and got[0].shape == q.shape and got[1].shape == q.shape[:3] and status.item() == 0
    _check_paged(got, q, cache, table, context, counts)
    if counts is not None:
        for b, n in enumerate(counts):
            assert not got[0][b, :, n:].any() and torch.isneginf(got[1][b, :, n:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,kv,T,context,counts", [(4, 2, 8, [300, 0, 1], None), (9, 1, 3, [127, 4000, 128], [3, 0, 2]), (8, 2, 8, [1001, 5, 77], [1, 8, 7]),
                                                   (16, 2, 4, [0, 640, 2500], None), (1, 1, 32, [95, 96, 97], [32, 31, 0]), (11, 1, 3, [500, 31, 0], None)])
def test_some_rows_of_a_kv_head(H, kv, T, context, counts, d, fmt, dtype):
    """16 to 33 of them, on either side of where another kernel takes over: none of it shows, nor does a mask that hides nothing."""
    Bd, g = _bd(), _gen(H * T + d)
    cache, table = _filled(Bd, g, fmt, 3, kv, 32, d, max(context) + T)
    q = _randn(g, 3, T, H, d, dtype=dtype, scale=2.0).transpose(1, 2)
    count = None if counts is None else _i32(counts)
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), count=count)
    _check_paged(got, q, cache, table, context, counts)
    first = torch.zeros(3, T, dtype=torch.int32, device="cuda")
    masked = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), count=count, first=first)
    _check_paged(masked, q, cache, table, context, counts)
    again = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), count=count)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def _masks(rng, B, T, context, kind):
    """first, last of some kinds; None where a kind leaves one out."""
    p = np.array(context)[:, None] + np.arange(T)[None]
    if kind == "window":
        return np.maximum(0, p + 1 - 37), None
    if kind == "documents":
        starts = np.sort(np.concatenate([np.zeros((B, 1), int), rng.integers(0, max(context) + T, (B, 6))], 1), 1)
        return np.stack([s[np.searchsorted(s, x, side="right") - 1] for s, x in zip(starts, p)]), None
    if kind == "prefix":
        return None, np.maximum(p + 1, rng.integers(0, max(context) + T, (B, 1)))
    if kind == "whole":
        return None, np.full((B, T), 2 ** 31 - 1)
    first = rng.integers(-5, max(context) + T + 5, (B, T))                                   # anything, nothing among it
    return first, first + rng.integers(-3, 200, (B, T))


@pytest.mark.parametrize("fmt,dtype", [("nvfp4", torch.bfloat16), ("e4m3", torch.float16)])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.5, False), (0.0, True), (30.0, True)])
@pytest.mark.parametrize("kind", ["window", "documents", "prefix", "whole", "any"])
@pytest.mark.parametrize("B,H,kv,T,d,P,context", [(2, 4, 2, 3, 64, 16, [200, 0]), (2, 6, 1, 150, 128, 32, [70, 301]), (1, 4, 1, 290, 64, 64, [130])])
def test_paged_attention_masks_caps_and_biases(B, H, kv, T, d, P, context, kind, cap, bias, fmt, dtype):
    Bd, g, rng = _bd(), _gen(T + d), np.random.default_rng(T)
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, max(context) + T)
    q = _randn(g, B, H, T, d, dtype=dtype, scale=2.0)
    first, last = _masks(rng, B, T, context, kind)
    slopes = torch.tensor([0.0, 2.0 ** -7, -0.25, 0.5, 1e-3, 3.0][:H], device="cuda") if bias else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), first=None if first is None else _i32(first.tolist()),
                                     last=None if last is None else _i32(last.tolist()), soft_cap=cap, slopes=slopes, status=status)
    assert status.item() == 0
    _check_paged(got, q, cache, table, context, first=first, last=last, cap=cap, slopes=slopes)


@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64), ("e4m3", 128)])
@pytest.mark.parametrize("T", [1, 2, 9])
def test_paged_attention_steps_far_into_contexts(T, fmt, d):
    """Few rows, with windows and documents that begin anywhere in contexts of up to 20000 tokens, capped, with a bias, and both."""
    Bd, g, rng = _bd(), _gen(d + T), np.random.default_rng(T)
    B, H, kv, P = 3, 4, 2, 32
    context = [20000, 127, 4096]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 20000 + T)
    q = _randn(g, B, H, T, d, scale=2.0)
    slopes = torch.tensor([0.01, 0.0, 2.0, -0.001], device="cuda")
    p = np.array(context)[:, None] + np.arange(T)[None]
    for first in (None, np.maximum(0, p + 1 - 100), np.maximum(0, p - 5000), rng.integers(0, np.array(context)[:, None] + 1, (B, T))):
        for kw in (dict(), dict(cap=20.0), dict(slopes=slopes), dict(cap=1.5, slopes=slopes)):
            got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), first=None if first is None else _i32(first.tolist()), soft_cap=kw.get("cap", 0.0),
                                             slopes=kw.get("slopes"))
            _check_paged(got, q, cache, table, context, first=first, **kw)


def test_paged_attention_many_items():
    """More items than a block remembers, of one tile each."""
    Bd, g = _bd(), _gen(81)
    B, H, kv, T, d, P = 620, 16, 8, 66, 64, 16
    context = [(i * 7) % 40 for i in range(B)]
    cache, table = _filled(Bd, g, "e4m3", B, kv, P, d, 40 + T)
    q = _randn(g, B, H, T, d)
    _check_paged(Bd.fp4attn_paged_attention(q, cache, table, _i32(context)), q, cache, table, context)


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("fmt", FMTS)
def test_paged_attention_what_nobody_sees(fmt, T):
    """Unseen bytes of every kind, NaN codes and scales among them: behind the last token, between the intervals of rows, in pages of nobody.  Rows that
    see nothing; rows behind a count, left as they were; pages that a window has left behind, which need not exist."""
    Bd, g = _bd(), _gen(21 + T)
    B, H, kv, d, P = 2, 4, 2, 128, 32
    context, counts = [300, 40], [T, T - 3]
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 300 + T)
    first = np.zeros((B, T), int)
    first[0] = 150
    first[1, 1] = 2 ** 31 - 1
    last = np.stack([np.where(np.arange(T) % 2, 180, 300 + T), np.arange(T) + 41])
    last[0, 2] = 100
    last[1, 3] = -2 ** 31
    first[0, T // 2:] = np.where(np.arange(T // 2, T) % 2, 150, 310)                         # nobody sees 180 .. 309 there
    q = _randn(g, B, H, T, d)
    kw = dict(count=_i32(counts), first=_i32(first.tolist()), last=_i32(last.tolist()))
    want = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), **kw)
    _check_paged(want, q, cache, table, context, counts, first, last)
    assert not want[0][0, :, 2].any() and torch.isneginf(want[1][0, :, 2]).all()
    written = Bd.QuantizedCache(cache.pages.clone(), cache.k_G, cache.v_G, cache.fmt, P, d)
    seen = np.zeros((B, table.shape[1] * P), bool)
    for b in range(B):
        for t in range(counts[b]):
            seen[b, max(0, first[b, t]):max(0, min(last[b, t], context[b] + counts[b]))] = True
    # every byte of an unseen token is 0xFF: NaN as an E4M3 code or scale
    kc, ks, vc, vs, shift = S.places(fmt, P, d)
    broken, gone = table.clone(), []
    bytes_of = written.pages.cpu().numpy()
    for b in range(B):
        for pos in np.flatnonzero(~seen[b]):
            t = pos % P
            for a in ([kc[t], vc[t]] if ks is None else [kc[t], ks[t], vs[t]]):
                bytes_of[int(table[b, pos // P])][:, a] = 255
        gone += [(b, i) for i in range(table.shape[1]) if not seen[b, i * P:(i + 1) * P].any()]
    written.pages.copy_(torch.as_tensor(bytes_of))
    free = [i for i in range(len(cache.pages)) if i not in table.flatten().tolist()]
    written.pages[free] = 255
    got = Bd.fp4attn_paged_attention(q, written, table, _i32(context), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for b, i in gone:
        broken[b, i] = -1 if i % 2 else 1 << 30
    mine = torch.full_like(want[0], 7.0), torch.full_like(want[1], 5.0)
    assert gone
    got = Bd.fp4attn_paged_attention(q, written, broken, _i32(context), out=mine[0], lse=mine[1], **kw)
    assert got[0] is mine[0] and got[1] is mine[1]
    for b, n in enumerate(counts):
        assert torch.equal(got[0][b, :, :n], want[0][b, :, :n]) and torch.equal(got[1][b, :, :n], want[1][b, :, :n])
        assert (got[0][b, :, n:] == 7.0).all() and (got[1][b, :, n:] == 5.0).all()


@pytest.mark.parametrize("T", [3, 140])
def test_paged_attention_tokens_without_a_page(T):
    Bd, g = _bd(), _gen(24)
    B, H, kv, d, P = 2, 2, 1, 64, 16
    cache, table = _filled(Bd, g, "nvfp4", B, kv, P, d, 300 + T)
    q = _randn(g, B, H, T, d)
    broken = table.clone()
    broken[0, 3], broken[0, 8], broken[1, 0] = -1, cache.pages.shape[0], 1 << 30
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_paged_attention(q, cache, broken, _i32([200, 20]), status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_paged(got, q, cache, broken, [200, 20])
    status.zero_()
    # a context that reaches behind the table, and one below 0
    room = table.shape[1] * P
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32([room - 1, -7]), status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_paged(got, q, cache, table, [room - 1, -7])
    status.zero_()
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32([5, -2 ** 31]), status=status)
    want = Bd.fp4attn_paged_attention(q, cache, table, _i32([5, 0]))
    assert torch.equal(got[0], want[0]) and status.item() == 0
    status.zero_()
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32([2 ** 31 - 1, 5]), status=status)
    assert status.item() == Bd.ERR_PAGE and torch.equal(got[0][1], Bd.fp4attn_paged_attention(q, cache, table, _i32([5, 5]))[0][1])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T", [4, 260])
def test_paged_attention_extreme_queries(T, fmt):
    """Logits of thousands, rows of unlike sizes side by side, tiny and zero queries; NaN and infinities stay in their rows."""
    Bd, g = _bd(), _gen(22)
    B, H, kv, d, P = 1, 8, 1, 128, 64
    cache, table = _filled(Bd, g, fmt, B, kv, P, d, 700 + T)
    q = _randn(g, B, H, T, d)
    q[0, 1] *= 1000.0
    q[0, 2] *= 1e-6
    q[0, 3] = 0.0
    q[0, 4] *= 1e-30
    q[0, 5, :, 1:] = 0.0
    q[0, 6, 2] *= 300.0
    for context in ([0], [640], [696]):
        for scale in (0.0, 0.3):
            for cap in (0.0, 20.0):
                got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), softmax_scale=scale, soft_cap=cap)
                _check_paged(got, q, cache, table, context, scale=scale, cap=cap)
    want = Bd.fp4attn_paged_attention(q, cache, table, _i32([640]))
    bad = q.clone()
    bad[0, 0, 1, 3], bad[0, 7, T - 1, 0], bad[0, 2, 2, 5] = math.nan, math.inf, -math.inf
    got = Bd.fp4attn_paged_attention(bad, cache, table, _i32([640]))
    hit = torch.zeros(H, T, dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[7, T - 1] = hit[2, 2] = True
    assert torch.equal(got[0][0][~hit], want[0][0][~hit]) and torch.equal(got[1][0][~hit], want[1][0][~hit])


def test_paged_attention_growing_logits():
    """Keys whose logits rise along the sequence: the running maximum moves in every tile."""
    Bd, g = _bd(), _gen(23)
    kv, P, d, length = 1, 64, 64, 1500
    cache = _cache(Bd, "e4m3", 24, kv, P, d)
    table = torch.arange(24, device="cuda", dtype=torch.int32)[None]
    u = torch.randn(d, generator=g, device="cuda")
    k = (u * torch.linspace(0.01, 1.0, length, device="cuda")[:, None]).to(torch.bfloat16)[None, None]
    v = _randn(g, 1, 1, length, d)
    Bd.fp4attn_cache_write(cache, k, v, table, _i32([0]))
    for T in (3, 300):
        q = (u * torch.linspace(-30.0, 30.0, T, device="cuda")[:, None]).to(torch.bfloat16)[None, None].expand(1, 2, T, d)
        got = Bd.fp4attn_paged_attention(q, cache, table, _i32([1500 - T]))
        _check_paged(got, q, cache, table, [1500 - T])


@pytest.mark.parametrize("T", [2, 131])
def test_paged_attention_strides(T):
    """Heads side by side, one sequence's queries for all, rows that begin anywhere; outputs of the caller's; no LSE wanted by nobody."""
    Bd, g = _bd(), _gen(31)
    B, H, kv, d, P = 2, 4, 2, 64, 16
    cache, table = _filled(Bd, g, "nvfp4", B, kv, P, d, 100 + T)
    x = _randn(g, B * T * (H * d + 3) + 1)
    q = x[1:].reshape(B, T, H * d + 3)[..., 3:].unflatten(2, (H, d)).transpose(1, 2)
    assert q.data_ptr() % 16 and q.stride(3) == 1
    want = Bd.fp4attn_paged_attention(q.contiguous(), cache, table, _i32([100, 3]))
    got = Bd.fp4attn_paged_attention(q, cache, table, _i32([100, 3]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = _randn(g, 1, H, T, d)
    want = Bd.fp4attn_paged_attention(one.repeat(B, 1, 1, 1), cache, table, _i32([100, 3]))
    got = Bd.fp4attn_paged_attention(one.expand(B, H, T, d), cache, table, _i32([100, 3]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_paged_attention_beyond_four_gigabytes():
    """Pages whose offsets pass 32 bits."""
    Bd, g = _bd(), _gen(25)
    kv, P, d = 8, 128, 128
    pages = (1 << 32) // (kv * Bd.fp4attn_cache_record_bytes(Bd.FMT_E4M3, P, d)) + 40
    cache = _cache(Bd, "e4m3", pages, kv, P, d)
    table = _i32([[pages - 1, 3, pages - 7], [pages - 30, pages - 2, 5]])
    k, v = _randn(g, 2, kv, 380, d), _randn(g, 2, kv, 380, d)
    Bd.fp4attn_cache_write(cache, k, v, table, _i32([0, 0]))
    q = _randn(g, 2, kv, 150, d)
    _check_paged(Bd.fp4attn_paged_attention(q, cache, table, _i32([200, 220])), q, cache, table, [200, 220])
    got = Bd.fp4attn_shared_prefix_attention(q[:, :, :5], cache, table[:1], _i32([370]), _i32([0, 2]), table, _i32([200, 220]))
    _check_shared(got, q[:, :, :5], cache, table[:1], [370], [0, 2], table, [200, 220])


# ---------------------------------------------------------------- shared prefixes
SHARED = [  # H, kv, T, d, P, prefixes, group_start, contexts, counts
    (1, 1, 1, 128, 64, [1], [0, 1], [0], None),
    (8, 2, 1, 128, 64, [500], [0, 5], [0, 3, 64, 130, 1], None),
    (6, 2, 4, 64, 16, [129, 0, 300], [0, 2, 3, 6], [50, 0, 7, 128, 300, 16], [4, 2, 0, 4, 1, 3]),
    (4, 1, 1, 64, 32, [700, 40], [1, 1, 4], [9, 9, 200, 31, 64], None),                     # an empty group; entries in no group
    (16, 2, 9, 128, 128, [1000], [0, 6], [256, 0, 5, 90, 255, 128], None),
    (5, 5, 64, 64, 64, [333], [0, 3], [1, 100, 64], [64, 10, 33]),
    (40, 1, 2, 128, 16, [2000, 77], [0, 9, 11], [i * 13 for i in range(11)], None),
    (2, 1, 1, 64, 16, [260], [0, 300], [i % 23 for i in range(300)], None),
    (4, 4, 1, 128, 64, [9000], [0, 4], [5, 2, 0, 600], None),
    (8, 8, 1, 64, 16, [3, 200], [0, 500, 700], [i % 37 for i in range(700)], None),         # more items than a block remembers
]


def _shared(Bd, g, fmt, kv, P, d, prefixes, context, T):
    """A cache, its prefixes' and its sequences' tables."""
    groups, B = len(prefixes), len(context)
    per_group, per_seq = max(1, -(-max(prefixes) // P)), -(-(max(context) + T) // P)
    total = groups * per_group + B * per_seq + 2
    cache = _cache(Bd, fmt, total, kv, P, d)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    prefix_table, table = order[:groups * per_group].reshape(groups, per_group), order[groups * per_group:-2].reshape(B, per_seq)
    for t, n in ((prefix_table, per_group * P), (table, per_seq * P)):
        x = _randn(g, len(t), kv, n, d), _randn(g, len(t), kv, n, d)
        Bd.fp4attn_cache_write(cache, *x, t, _i32([0] * len(t)))
    return cache, prefix_table, table


@pytest.mark.parametrize("fmt,dtype", [("nvfp4", torch.bfloat16), ("e4m3", torch.float16), ("e4m3", torch.bfloat16)])
@pytest.mark.parametrize("H,kv,T,d,P,prefixes,starts,context,counts", SHARED)
def test_shared_prefix_attention(H, kv, T, d, P, prefixes, starts, context, counts, fmt, dtype):
    Bd, g, B = _bd(), _gen(H * T + d), len(context)
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, P, d, prefixes, context, T)
    q = _randn(g, B, T, H, d, dtype=dtype, scale=2.0).transpose(1, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    slopes = 2.0 ** -(torch.arange(H, device="cuda") % 9 + 1.0)
    for bits, kw in ((None, {}), (_tree_bits(np.random.default_rng(T), B, T), {}), (None, dict(cap=15.0, slopes=slopes))):
        got = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32(prefixes), _i32(starts), table, _i32(context), tree_mask=bits,
                                                 count=None if counts is None else _i32(counts), soft_cap=kw.get("cap", 0.0), slopes=kw.get("slopes"),
                                                 status=status)
        assert got[0].dtype == dtype and got[0].shape == q.shape and status.item() == 0
        _check_shared(got, q, cache, prefix_table, prefixes, starts, table, context, None if bits is None else bits.tolist(), counts, **kw)
        if counts is not None:
            for b, n in enumerate(counts):
                assert not got[0][b, :, n:].any() and torch.isneginf(got[1][b, :, n:]).all()


def test_shared_prefix_attention_rows_of_nothing_and_lost_pages():
    """A row without a prefix whose mask is empty; masks that see only the prefix, or nothing of it; pages of a prefix and of a sequence that are not there."""
    Bd, g = _bd(), _gen(61)
    kv, P, d, T, H = 2, 16, 64, 3, 4
    prefixes, starts, context = [0, 90], [0, 2, 4], [0, 20, 0, 33]
    cache, prefix_table, table = _shared(Bd, g, "e4m3", kv, P, d, prefixes, context, T)
    q = _randn(g, 4, H, T, d)
    bits = torch.tensor([[0, 1, 4], [0, 0, 7], [0, 2, 0], [0, 1, 3]], dtype=torch.int64, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (q, cache, prefix_table, _i32(prefixes), _i32(starts), table, _i32(context))
    got = Bd.fp4attn_shared_prefix_attention(*args, tree_mask=bits, status=status)
    assert status.item() == 0 and not got[0][0, :, 0].any() and torch.isneginf(got[1][0, :, 0]).all()
    _check_shared(got, q, cache, prefix_table, prefixes, starts, table, context, bits.tolist())
    broken, other = prefix_table.clone(), table.clone()
    broken[1, 2] = -1
    got = Bd.fp4attn_shared_prefix_attention(q, cache, broken, *args[3:], tree_mask=bits, status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_shared(got, q, cache, broken, prefixes, starts, table, context, bits.tolist())
    status.zero_()
    other[3, 1] = 1 << 30
    got = Bd.fp4attn_shared_prefix_attention(*args[:5], other, args[6], tree_mask=bits, status=status)
    assert status.item() == Bd.ERR_PAGE
    _check_shared(got, q, cache, prefix_table, prefixes, starts, other, context, bits.tolist())
    # lengths beyond the table, below 0; starts beyond the batch
    status.zero_()
    got = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32([-5, 2 ** 31 - 1]), _i32([-3, 2, 99]), table, _i32(context), tree_mask=bits, status=status)
    assert status.item() == Bd.ERR_PAGE
    room = prefix_table.shape[1] * P
    want = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32([0, room]), _i32([0, 2, 4]), table, _i32(context), tree_mask=bits)
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("fmt", FMTS)
def test_shared_prefix_attention_is_attention_over_both(fmt):
    """The same numbers, within the roundings of two calls, as fp4attn_tree_attention over tables that begin with the prefix's pages."""
    Bd, g = _bd(), _gen(62)
    kv, P, d, T, H, B = 2, 32, 128, 5, 8, 6
    prefixes, context = [320], [64, 0, 3, 100, 31, 32]
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, P, d, prefixes, context, T)
    q = _randn(g, B, H, T, d)
    got = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32(prefixes), _i32([0, B]), table, _i32(context))
    both = torch.cat((prefix_table.expand(B, -1), table), 1).contiguous()
    want = Bd.fp4attn_tree_attention(q, cache, both, _i32([x + 320 for x in context]))
    assert torch.allclose(got[1], want[1], rtol=0, atol=1e-5)
    # each is off by its rounding to bf16, half a step of 2^-7, and by what f16 probabilities give, 2^-10 of sum p |v| (values up to 4.5)
    assert (got[0].float() - want[0].float()).abs().max() <= 2.0 ** -7 * want[0].float().abs().max() + 2.0 ** -9 * 4.5


# ---------------------------------------------------------------- pages
def _pool(Bd, free, left, P):
    return Bd.PagePool(_i32(free), _i32([left]), P)


@pytest.mark.parametrize("B,N,P,most", [(1, 1, 64, 0), (1, 1, 16, 1), (7, 5, 16, 100), (300, 1, 16, 50), (1000, 3, 32, 400), (33, 700, 128, 900),
                                        (3, 5000, 16, 40), (2100, 1, 64, 129), (9, 2048, 64, 1), (4, 2049, 16, 33), (64, 64, 16, 64)])
def test_pages_assign_and_release(B, N, P, most):
    """Random starts and counts, twice in a row, then everything back: tables, stack, slots, positions as the oracle has them."""
    Bd, rng = _bd(), np.random.default_rng(B * N + P)
    start = rng.integers(0, most + 1, B)
    room = -(-(most + 2 * N) // P) + 1
    pages = int(sum(-(-s // P) for s in start)) + B * (-(-2 * N // P) + 2)
    free = rng.permutation(pages).tolist()
    left = pages
    table = [[-1] * room for _ in range(B)]
    for b in range(B):
        for i in range(-(-int(start[b]) // P)):
            left -= 1
            table[b][i] = free[left]
    pool, dev = _pool(Bd, free, left, P), _i32(table)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = pool.free.clone(), pool.count.clone(), dev.clone()
    first = start.copy()
    for counts in (rng.integers(-1, N + 1, B), None):
        got = Bd.fp4attn_pages_assign(pool, dev, _i32(start.tolist()), None if counts is None else _i32(counts.tolist()), N=N, status=status)
        left, slots, positions, fine = S.pages_assign(free, left, table, start, counts, N, P)
        assert fine and status.item() == 0 and pool.count.item() == left and pool.turn.item() == 0
        assert dev.tolist() == table and got[0].tolist() == slots and got[1].tolist() == positions
        assert got[0].dtype == torch.int64 and got[1].dtype == torch.int32
        start = start + (N if counts is None else np.maximum(counts, 0))
    Bd.fp4attn_pages_release(pool, dev, _i32(start.tolist()), keep=_i32(((first + start) // 2).tolist()), status=status)
    left, fine = S.pages_release(free, left, table, start, (first + start) // 2, P)
    assert fine and status.item() == 0 and pool.count.item() == left and dev.tolist() == table and pool.free.tolist() == free
    Bd.fp4attn_pages_release(pool, dev, _i32(start.tolist()), status=status)
    left, fine = S.pages_release(free, left, table, start, None, P)
    assert left == pages and pool.count.item() == pages and pool.free.tolist() == free and (dev == -1).all() and status.item() == 0
    # an assign undone leaves the stack as it was
    pool, dev = _pool(Bd, kept[0].tolist(), kept[1].item(), P), kept[2].clone()
    n = _i32(rng.integers(0, N + 1, B).tolist())
    Bd.fp4attn_pages_assign(pool, dev, _i32(first.tolist()), n, N=N)
    Bd.fp4attn_pages_release(pool, dev, _i32(first.tolist()) + n, keep=_i32(first.tolist()))
    assert torch.equal(pool.free, kept[0]) and torch.equal(pool.count, kept[1]) and torch.equal(dev, kept[2])


def test_pages_run_out():
    """A stack that ends inside an entry, a table without room, an empty stack, entries that are not to get any; pages released twice, holes, numbers
    of no page."""
    Bd, P = _bd(), 16
    free, table = list(range(10)), [[-1] * 6 for _ in range(5)]
    pool, dev = _pool(Bd, free, 10, P), _i32(table)
    start, count = [0, 0, -4, 0, 0], [64, 200, 50, 0, 17]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = Bd.fp4attn_pages_assign(pool, dev, _i32(start), _i32(count), N=40, status=status)
    left, slots, positions, fine = S.pages_assign(free, 10, table, start, count, 40, P)
    assert not fine and left == 0 and status.item() == Bd.ERR_PAGE
    assert dev.tolist() == table and got[0].tolist() == slots and got[1].tolist() == positions and pool.count.item() == 0 and pool.turn.item() == 0
    status.zero_()
    table[0][1] = 99                                                # of no pool
    dev[0, 1] = 99
    length = [64, 96, 7, 2 ** 31 - 1, -3]
    Bd.fp4attn_pages_release(pool, dev, _i32(length), status=status)
    left, fine = S.pages_release(free, 0, table, length, None, P)
    assert fine and status.item() == 0 and pool.count.item() == left == 9 and pool.free.tolist() == free and dev.tolist() == table
    table[1][:4], table[2][0] = [5, 6, 7, 8], 3
    dev.copy_(_i32(table))
    Bd.fp4attn_pages_release(pool, dev, _i32([0, 64, 16, 0, 0]), status=status)
    left, fine = S.pages_release(free, left, table, [0, 64, 16, 0, 0], None, P)
    assert not fine and status.item() == Bd.ERR_PAGE and pool.count.item() == left == 10 and pool.free.tolist() == free and dev.tolist() == table
    # only pages, no slots
    pool, dev = Bd.fp4attn_pages_create(9, P), torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    assert Bd.fp4attn_pages_assign(pool, dev, _i32([0, 0]), _i32([33, 1])) == (None, None)
    assert dev.tolist() == [[0, 1, 2, -1], [3, -1, -1, -1]] and pool.count.item() == 5


def test_pages_in_a_captured_loop():
    """A step that takes pages by itself: captured once, replayed; every token gets the page and place that the oracle gives it."""
    Bd, P, B = _bd(), 16, 5
    pool, table = Bd.fp4attn_pages_create(40, P), torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
    length, one = _i32([0, 3, 15, 16, 31]), _i32([1, 1, 1, 0, 1])
    Bd.fp4attn_pages_assign(pool, table, torch.zeros_like(length), length)
    free, left, want = list(range(39, -1, -1)), 40, [[-1] * 8 for _ in range(B)]
    left = S.pages_assign(free, left, want, [0] * B, length.tolist(), 0, P)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    now = length.tolist()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            slots, positions = Bd.fp4attn_pages_assign(pool, table, length, one, N=1)
            length.add_(one)
        for _ in range(40):
            graph.replay()
            side.synchronize()
            left, s, p, fine = S.pages_assign(free, left, want, now, one.tolist(), 1, P)
            now = [x + y for x, y in zip(now, one.tolist())]
            assert slots.tolist() == s and positions.tolist() == p and table.tolist() == want and pool.count.item() == left


# ---------------------------------------------------------------- a run of them, as a server makes it
def _serve(Bd, s):
    """Pages for a prompt, its keys rotated and written, attention over it; then a drafted step behind the shared prefix, turned down again."""
    slots, positions = Bd.fp4attn_pages_assign(s["pool"], s["table"], s["zero"], s["count"], N=s["N"])
    q = Bd.fp4attn_rotary(s["q"], positions, s["freq"])
    Bd.fp4attn_cache_write(s["cache"], s["k"], s["v"], s["table"], s["zero"], count=s["count"], inv_freq=s["freq"], positions=positions)
    prompt = Bd.fp4attn_paged_attention(q, s["cache"], s["table"], s["zero"], count=s["count"], soft_cap=40.0)
    Bd.fp4attn_pages_assign(s["pool"], s["table"], s["count"], s["T"])
    Bd.fp4attn_cache_write(s["cache"], s["k2"], s["v2"], s["table"], s["count"], inv_freq=s["freq"])
    step = Bd.fp4attn_shared_prefix_attention(s["q2"], s["cache"], s["prefix_table"], s["prefix_length"], s["group_start"], s["table"], s["count"],
                                              tree_mask=s["bits"])
    Bd.fp4attn_pages_release(s["pool"], s["table"], s["count"] + s["T"])
    return slots, positions, *prompt, *step, s["pool"].free, s["pool"].count


def _server(Bd, seed, fmt, T=4):
    g = _gen(seed)
    B, H, kv, d, P, N = 3, 8, 2, 64, 16, 150
    s = {"N": N, "zero": _i32([0] * B), "count": _i32([150, 37, 128]), "T": _i32([T] * B), "freq": Bd.fp4attn_rotary_frequencies(d)}
    s["pool"] = Bd.fp4attn_pages_create(60, P)
    s["cache"] = _cache(Bd, fmt, 60, kv, P, d)
    s["table"] = torch.full((B, 11), -1, dtype=torch.int32, device="cuda")
    s["q"], s["k"], s["v"] = _randn(g, B, H, N, d), _randn(g, B, kv, N, d), _randn(g, B, kv, N, d)
    s["q2"], s["k2"], s["v2"] = _randn(g, B, H, T, d), _randn(g, B, kv, T, d), _randn(g, B, kv, T, d)
    s["bits"] = _tree_bits(np.random.default_rng(seed), B, T)
    s["prefix_table"] = torch.full((1, 9), -1, dtype=torch.int32, device="cuda")
    s["prefix_length"], s["group_start"] = _i32([140]), _i32([0, B])
    Bd.fp4attn_pages_assign(s["pool"], s["prefix_table"], s["zero"][:1], s["prefix_length"])
    Bd.fp4attn_cache_write(s["cache"], _randn(g, 1, kv, 140, d), _randn(g, 1, kv, 140, d), s["prefix_table"], s["zero"][:1])
    return s


@pytest.mark.parametrize("fmt", FMTS)
def test_a_server(fmt):
    Bd = _bd()
    s = _server(Bd, 71, fmt)
    table = s["table"]
    before = s["pool"].free.clone(), s["pool"].count.clone()
    slots, positions, out, lse, out2, lse2, *_ = _serve(Bd, s)
    assert torch.equal(s["pool"].free, before[0]) and torch.equal(s["pool"].count, before[1]) and (table == -1).all()
    # the same pages again, to look at what was written
    Bd.fp4attn_pages_assign(s["pool"], table, s["zero"], s["count"])
    Bd.fp4attn_pages_assign(s["pool"], table, s["count"], s["T"])
    counts = s["count"].tolist()
    for b, n in enumerate(counts):
        for t in (0, 15, 16, n - 1):
            assert slots[b, t].item() == table[b, t // 16].item() * 16 + t % 16
        assert (slots[b, n:] == -1).all()
    q = Bd.fp4attn_rotary(s["q"], positions, s["freq"])
    _check_paged((out, lse), q, s["cache"], table, [0] * 3, counts, cap=40.0)
    _check_shared((out2, lse2), s["q2"], s["cache"], s["prefix_table"], [140], [0, 3], table, counts, s["bits"].tolist())


def test_a_server_repeats_captures_and_runs_beside_another():
    """The same bits every time: again, captured and replayed (two graphs whose workspaces are one pool's, in turn and at once), beside another's."""
    Bd = _bd()
    states = [_server(Bd, 72, "nvfp4"), _server(Bd, 73, "e4m3", T=7)]
    want = [[x.clone() for x in _serve(Bd, s)] for s in states]
    for s, w in zip(states, want):
        assert all(torch.equal(a, b) for a, b in zip(_serve(Bd, s), w))
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append([x.clone() for x in _serve(Bd, s)])
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(x, want[i % 2]))
    graphs, outs = [], []
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(_serve(Bd, s))
        graphs.append(graph)
    for _ in range(3):
        for o in outs:
            for x in o[:-2]:
                x.zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
    states[0]["q"].copy_(_randn(_gen(77), *states[0]["q"].shape))
    graphs[0].replay()
    torch.cuda.synchronize()
    kept = [x.clone() for x in outs[0]]
    assert all(torch.equal(a, b) for a, b in zip(kept, _serve(Bd, states[0])))


# ---------------------------------------------------------------- refusals
def test_refusals():
    Bd, g = _bd(), _gen(51)
    cache, table = _filled(Bd, g, "nvfp4", 2, 2, 16, 64, 20)
    start, q = _i32([3, 4]), _randn(g, 2, 4, 3, 64)
    prefix = (table[:1], _i32([20]), _i32([0, 2]))
    both = _i32([[0, 1, 2]] * 2)
    paged = lambda q=q, cache=cache, table=table, start=start, **kw: Bd.fp4attn_paged_attention(q, cache, table, start, **kw)
    shared = lambda q=q, cache=cache, prefix=prefix, table=table, start=start, **kw: Bd.fp4attn_shared_prefix_attention(q, cache, *prefix, table, start, **kw)
    bad = []
    for call in (paged, shared):
        bad += [lambda c=call: c(q=q.float()), lambda c=call: c(q=q[:, :3]), lambda c=call: c(q=q[..., :32]), lambda c=call: c(q=q.cpu()), lambda c=call: c(q=q[0]),
                lambda c=call: c(table=table.long()), lambda c=call: c(table=table[:1]), lambda c=call: c(table=table.t()), lambda c=call: c(start=start.long()),
                lambda c=call: c(start=start[:1]), lambda c=call: c(count=start.long()), lambda c=call: c(count=start[:1]), lambda c=call: c(slopes=torch.ones(3, device="cuda")),
                lambda c=call: c(slopes=torch.ones(4)), lambda c=call: c(slopes=torch.ones(4, device="cuda", dtype=torch.float64)), lambda c=call: c(out=q.half()),
                lambda c=call: c(out=torch.empty_like(q.transpose(1, 2).contiguous())), lambda c=call: c(lse=torch.empty(2, 3, 4, device="cuda")),
                lambda c=call: c(lse=q), lambda c=call: c(status=start), lambda c=call: c(q=q.clone().requires_grad_()),
                lambda c=call: c(slopes=torch.ones(4, device="cuda", requires_grad=True))]
    bad += [lambda: paged(first=both.long()), lambda: paged(last=both[:1]), lambda: paged(first=both.t().contiguous()), lambda: paged(last=both.flatten()), lambda: paged(first=both.cpu()),
            lambda: shared(tree_mask=both), lambda: shared(tree_mask=both.long()[:1]), lambda: shared(prefix=(table[0], *prefix[1:])), lambda: shared(prefix=(table[:1].long(), *prefix[1:])),
            lambda: shared(prefix=(table[:1], _i32([20, 3]), prefix[2])), lambda: shared(prefix=(table[:1], prefix[1], _i32([0, 1, 2]))), lambda: shared(prefix=(table[:1], prefix[1].cpu(), prefix[2]))]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    for call in (paged, shared):
        for kw in (dict(softmax_scale=-1.0), dict(soft_cap=-1.0), dict(soft_cap=math.nan), dict(softmax_scale=math.inf), dict(soft_cap=math.inf)):
            with pytest.raises(Bd.Fp4AttnError, match="invalid argument"):
                call(**kw)
        for B, T in ((0, 3), (2, 0)):
            with pytest.raises(AssertionError, match="at least one sequence"):
                call(q=_randn(g, B, 4, T, 64))
    with pytest.raises(Bd.Fp4AttnError, match="unsupported shape"):
        shared(q=_randn(g, 2, 4, 65, 64))
    with torch.no_grad():
        paged(q=q.clone().requires_grad_())
    pool, dev = Bd.fp4attn_pages_create(8, 16), torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    one = _i32([1, 1])
    wrong = lambda **kw: Bd.PagePool(**{**dict(free=pool.free, count=pool.count, page_size=16, turn=pool.turn), **kw})
    for call in (lambda: Bd.fp4attn_pages_assign(pool, dev.long(), one, one), lambda: Bd.fp4attn_pages_assign(pool, dev.t(), one, one), lambda: Bd.fp4attn_pages_assign(pool, dev[0], one, one),
                 lambda: Bd.fp4attn_pages_assign(pool, dev, one.long(), one), lambda: Bd.fp4attn_pages_assign(pool, dev, one, one[:1]), lambda: Bd.fp4attn_pages_assign(pool, dev, one),
                 lambda: Bd.fp4attn_pages_assign(pool, dev, one, one, N=-1), lambda: Bd.fp4attn_pages_assign(pool, dev, one, one, status=one), lambda: Bd.fp4attn_pages_assign(pool, dev[:0], one[:0], one[:0]),
                 lambda: Bd.fp4attn_pages_release(pool, dev, one.cpu()), lambda: Bd.fp4attn_pages_release(pool, dev, one, keep=one[:1]), lambda: Bd.fp4attn_pages_release(pool, dev.cpu(), one),
                 lambda: Bd.fp4attn_pages_assign(wrong(free=pool.free.long()), dev, one, one), lambda: Bd.fp4attn_pages_assign(wrong(count=one), dev, one, one),
                 lambda: Bd.fp4attn_pages_release(wrong(turn=pool.turn.cpu()), dev, one), lambda: Bd.fp4attn_pages_release(wrong(free=pool.free[:0]), dev, one)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(Bd.Fp4AttnError, match="unsupported shape"):
        Bd.fp4attn_pages_assign(wrong(page_size=48), dev, one, one)
    with pytest.raises(OverflowError):
        Bd.fp4attn_pages_assign(pool, dev, one, one, N=1 << 32)
    assert (dev == -1).all() and pool.count.item() == 8
