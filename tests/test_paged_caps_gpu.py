"""Caps of every size: a capped score is right to its own size, not to the cap's, in every kernel and in every part of a row alike."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as S
from test_paged_gpu import _shared, _values
from test_serving_gpu import HALF, U, _bd, _filled, _gen, _i32, _randn

pytestmark = pytest.mark.gpu


def _check(got, q, kv, keys_of, cap, slopes=None):
    """keys_of(b) -> K, V [kv, keys, d], mask [T, keys], distances [T, keys].

    As test_paged_gpu's, but for the cap: with size = the largest sum of |q k| scale over a row's keys, far = the largest slope * distance, a score is
    off by d sums in fp32 and ten roundings (its constant, the product with it, u, the last products of the cap), (d + 10) u size, and by the
    2^-20 of itself of the polynomial, or of the exponential form, together no more than 2^-19 of min(size, cap); by 8 u far.  All that is ds; the
    slope of the cap is at most 1.  exp2 is off by 2^-21, its argument by 2 u of what it is subtracted from; a probability by f16, 2^-11, or 2^-32 of
    the largest; sums of n terms by n u.  O is off by 2 (ds + 2^-20 + n u) + 2^-11 of sum p |v|, 2^-32 a key of max |v| and its type's rounding."""
    B, H, T, d = q.shape
    for b in range(B):
        k, v, mask, far = keys_of(b)
        x = q[b].double().unflatten(0, (kv, H // kv))
        z = torch.einsum("hgtd,hkd->hgtk", x, k) / math.sqrt(d)
        size = torch.where(mask, torch.einsum("hgtd,hkd->hgtk", x.abs(), k.abs()) / math.sqrt(d), 0.0).amax(-1)
        z = cap * torch.tanh(z / cap)
        reach = torch.zeros_like(size)
        if slopes is not None:
            slope = slopes.double().view(kv, -1, 1, 1)
            z = z - slope * far
            reach = (slope.abs() * torch.where(mask, far, 0.0)).amax(-1)
        z = torch.where(mask, z, -math.inf)
        assert mask.any(-1).all()
        lse, p = torch.logsumexp(z, -1), torch.softmax(z, -1)
        o, pv = torch.einsum("hgtk,hkd->hgtd", p, v), torch.einsum("hgtk,hkd->hgtd", p, v.abs())
        ds = (d + 10) * U * size + 2.0 ** -19 * size.clamp(max=cap) + 8 * U * reach
        n = k.shape[1]
        bound = HALF[q.dtype] * o.abs() + (2 * (ds[..., None] + 2.0 ** -20 + n * U) + 2.0 ** -11) * pv + n * 2.0 ** -32 * v.abs().amax() + 2.0 ** -40
        out, l = got[0][b].double().unflatten(0, (kv, -1)), got[1][b].double().unflatten(0, (kv, -1))
        assert ((out - o).abs() <= bound * (1 + 2.0 ** -8)).all(), (cap, (out - o).abs().max().item())
        assert ((l - lse).abs() <= ds + 2.0 ** -20 + n * U + 2 * U * (lse.abs() + 1 + size + reach)).all(), (cap, (l - lse).abs().max().item())


CAPS = [0.7, 5.0, 200.0, 1e4, 1e6, 1e8, 1e9, 2.0 ** 60]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("nvfp4", 64), ("e4m3", 64)])
@pytest.mark.parametrize("H,kv,T,context", [(8, 2, 1, 1500), (6, 1, 2, 900), (8, 2, 12, 500), (4, 2, 60, 700), (4, 1, 150, 600)])
def test_caps_of_every_size(H, kv, T, context, fmt, d, bias):
    """4 to 600 rows of a KV head; scores of up to some 60 and, in one row, of thousands; with a window, and without a mask."""
    Bd, g = _bd(), _gen(H * T + d)
    cache, table = _filled(Bd, g, fmt, 1, kv, 32, d, context + T)
    q = _randn(g, 1, H, T, d, scale=6.0)
    q[0, 1, 0] *= 100.0
    slopes = torch.tensor([0.05, 0.0, -0.01, 0.5, 1e-3, 2.0, 0.02, 0.1][:H], device="cuda") if bias else None
    k, v, held = _values(cache, table[0], context + T)
    assert held.all()
    at = torch.arange(context + T, device="cuda")
    far = (context + torch.arange(T, device="cuda")[:, None] - at).abs().double()
    for first in (None, np.maximum(0, context + np.arange(T)[None] - 300)):
        mask = torch.as_tensor(S.between(context, T, T, None if first is None else first[0]), device="cuda")
        for cap in CAPS:
            got = Bd.fp4attn_paged_attention(q, cache, table, _i32([context]), first=None if first is None else _i32(first.tolist()), soft_cap=cap, slopes=slopes)
            _check(got, q, kv, lambda b: (k, v, mask, far), cap, slopes)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
@pytest.mark.parametrize("T", [1, 9, 40])
def test_caps_of_every_size_over_shared_prefixes(T, fmt, d, bias):
    Bd, g = _bd(), _gen(T + d)
    H, kv, B = 4, 2, 3
    prefixes, starts, context = [400], [0, B], [40, 0, 130]
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, 16, d, prefixes, context, T)
    q = _randn(g, B, H, T, d, scale=6.0)
    slopes = torch.tensor([0.05, 0.0, -0.01, 0.5], device="cuda") if bias else None
    kp, vp, _ = _values(cache, prefix_table[0], 400)

    def keys_of(b):
        k, v, _ = _values(cache, table[b], context[b] + T)
        n = 400 + context[b]
        p, j = n + torch.arange(T, device="cuda")[:, None], torch.arange(n + T, device="cuda")
        return torch.cat((kp, k), 1), torch.cat((vp, v), 1), j <= p, (p - j).abs().double()

    for cap in CAPS:
        got = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32(prefixes), _i32(starts), table, _i32(context), soft_cap=cap, slopes=slopes)
        _check(got, q, kv, keys_of, cap, slopes)
