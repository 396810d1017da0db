"""Pins of the serving oracle, and what the serving entry points refuse (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import serving as S


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_rotation(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 5, 64))
    pos = rng.integers(0, 1 << 20, (2, 5))
    f = (10000.0 ** (-np.arange(0, 48, 2) / 48)).astype(np.float32)
    y = S.rotary(x, pos, f, interleaved)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)                 # lengths stay
    assert np.array_equal(y[..., 48:], x[..., 48:])                                    # behind the rotated part: as it was
    assert np.allclose(S.rotary(y, pos, f, interleaved, transposed=True), x, atol=1e-12)
    a, b = (0, 1) if interleaved else (0, 24)                                          # pair 0 turns by the position itself
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, None].astype(np.float64))
    assert np.allclose(y[..., a], z.real, atol=1e-9) and np.allclose(y[..., b], z.imag, atol=1e-9)
    # the product of a rotated query and key goes by the difference of their positions
    q, k = x[:1, :1, :1], x[1:, 1:2, 1:2]
    p = lambda i: np.array([[i]])
    dots = [(S.rotary(q, p(i + 7), f, interleaved) * S.rotary(k, p(i), f, interleaved)).sum() for i in (0, 5, 1000)]
    assert np.allclose(dots, dots[0], atol=1e-9)


@pytest.mark.parametrize("fmt", ["nvfp4", "e4m3"])
@pytest.mark.parametrize("P,d", [(16, 64), (128, 128)])
def test_every_byte_of_a_record_has_one_meaning(fmt, P, d):
    kc, ks, vc, vs, shift = S.places(fmt, P, d)
    size = S.record_bytes(fmt, P, d)
    used = np.zeros(size, dtype=int)
    for at in (kc, vc):
        np.add.at(used, at.reshape(-1), 1)
    if fmt == "nvfp4":
        for at in (ks, vs):
            np.add.at(used, at.reshape(-1), 2)
        assert set(used) == {2}                       # two codes, or one scale
    else:
        assert set(used) == {1}
    # the order of V scales, by hand
    if fmt == "nvfp4":
        assert [int(vs[t, 0] - vs[0, 0]) for t in range(9)] == [0, 2, 4, 6, 1, 3, 5, 7, 8]


@pytest.mark.parametrize("fmt", ["nvfp4", "e4m3"])
def test_cache_round_trip(fmt):
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 1, 2, 5, 64))
    full = 2688.0 if fmt == "nvfp4" else 448.0
    G = np.full(2, full / 5, dtype=np.float32)
    pages = np.zeros((3, 2, S.record_bytes(fmt, 16, 64)), dtype=np.uint8)
    assert S.write(pages, k, v, [[2, 0]], [14], None, G, G, fmt, 16)
    got_k, got_v, held = S.values(pages, [2, 0], 1, 19, G, G, fmt, 16, 64)
    assert held.all()
    for got, x in ((got_k, k), (got_v, v)):
        err = np.abs(got[14:] - x[0, 1])
        if fmt == "e4m3":
            assert (err <= np.maximum(np.abs(x[0, 1]) * 2.0 ** -4, 2.0 ** -10 * 5 / 448 * 1.01)).all()
        else:                                          # half the widest step of E2M1 (1 of 6) of the block's largest, with its scale's rounding
            assert (err <= np.abs(x[0, 1]).max() * (1 / 6 + 2.0 ** -4) * 1.01).all()
    assert not S.write(pages, k, v, [[2, 3]], [14], None, G, G, fmt, 16)               # page 3 does not exist


def test_encode_edges():
    x = np.zeros((1, 64))
    x[0, :4] = [np.nan, np.inf, -np.inf, 1.0]
    codes, sb = S.encode(x, 1.0, "nvfp4")
    assert list(F.e2m1_decode(codes[0, :4])) == [0.0, 6.0, -6.0, 0.0] and F.e4m3_decode(sb[0, 0]) == 448.0
    assert list(F.e4m3_decode(S.encode(x, 100.0, "e4m3")[0][0, :4])) == [0.0, 448.0, -448.0, 96.0]     # 100: a tie, to even


def test_attend_against_brute_force_and_empty_rows():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    mask = S.seen(4, 2, [0b11, 0b00], np.ones(6, dtype=bool))
    assert mask.tolist() == [[True] * 6, [True] * 4 + [False] * 2]
    mask = np.vstack([mask, np.zeros((1, 6), dtype=bool)])
    o, lse, _, _ = S.attend(q, k, v, mask, 0.5)
    for t in range(2):
        w = [math.exp(0.5 * float(q[t] @ k[j])) if mask[t, j] else 0.0 for j in range(6)]
        assert np.allclose(o[t], sum(w[j] * v[j] for j in range(6)) / sum(w)) and np.isclose(lse[t], math.log(sum(w)))
    assert not o[2].any() and lse[2] == -np.inf


# ---------------------------------------------------------------- the library's own checks
@pytest.fixture(scope="module")
def lib():
    from paper_2609_04105_b200 import build
    return ctypes.CDLL(build.build())


class _View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_longlong), ("sh", ctypes.c_longlong), ("sn", ctypes.c_longlong)]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("k_G", ctypes.c_void_p), ("v_G", ctypes.c_void_p), ("fmt", ctypes.c_int),
                ("page_size", ctypes.c_int), ("num_pages", ctypes.c_int), ("kv_heads", ctypes.c_int), ("d", ctypes.c_int)]


def _view(at=0x1000):
    return ctypes.byref(_View(at, 64, 64, 64))


def test_record_bytes(lib):
    lib.fp4attn_cache_record_bytes.restype = ctypes.c_size_t
    for fmt, name in ((1, "nvfp4"), (2, "e4m3")):
        for P in (16, 32, 64, 128):
            for d in (64, 128):
                assert lib.fp4attn_cache_record_bytes(fmt, P, d) == S.record_bytes(name, P, d) and S.record_bytes(name, P, d) % 16 == 0
    assert lib.fp4attn_cache_record_bytes(0, 64, 128) == 0                             # MXFP4 is no format of a cache
    assert lib.fp4attn_cache_record_bytes(1, 48, 128) == 0 and lib.fp4attn_cache_record_bytes(1, 8, 128) == 0
    assert lib.fp4attn_cache_record_bytes(1, 256, 128) == 0 and lib.fp4attn_cache_record_bytes(1, 64, 96) == 0


def test_rotary_refusals(lib):
    vp, fl = ctypes.c_void_p, ctypes.c_float

    def call(q=_view(), k=_view(), type=0, B=1, H=2, kv=1, N=4, d=64, positions=0x1000, f=0x1000, pairs=32, inter=0, trans=0):
        return lib.fp4attn_rotary(q, k, _view(), _view(), type, B, H, kv, N, d, vp(positions), vp(f), pairs, inter, trans, fl(1.0), None)
    assert call(q=None) == 1 and call(k=None) == 1 and call(positions=0) == 1 and call(f=0) == 1
    assert call(type=3) == 1 and call(inter=2) == 1 and call(trans=-1) == 1 and call(pairs=0) == 1 and call(N=0) == 1
    assert call(pairs=33) == 2 and call(d=258) == 2
    assert call(q=_view(0x1001)) == 4 and call(type=2, q=_view(0x1002)) == 4 and call(positions=0x1002) == 4


def test_cache_and_attention_refusals(lib):
    vp, sz, fl = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float

    def cache(pages=0x1000, k_G=0x1000, v_G=0x1000, fmt=1, P=64, n=4, kv=2, d=128):
        return ctypes.byref(_Cache(pages, k_G, v_G, fmt, P, n, kv, d))

    def write(c=cache(), k=_view(), type=0, B=1, N=4, table=0x1000, pages=4, start=0x1000, positions=0, f=0, pairs=0):
        return lib.fp4attn_cache_write(c, k, _view(), type, B, N, vp(table), pages, vp(start), None, vp(positions), vp(f), pairs, 0, fl(1.0),
                                       None, None)

    def read(c=cache(), k=_view(), type=0, B=1, N=4, table=0x1000, pages=4, start=0x1000):
        return lib.fp4attn_cache_read(c, k, _view(), type, B, N, vp(table), pages, vp(start), None, None, None)

    def tree(c=cache(), q=_view(), type=0, B=1, H=4, T=4, table=0x1000, pages=4, start=0x1000, mask=0, scale=0.0, O=0x1000, ws=0x1000, n=1 << 40):
        return lib.fp4attn_tree_attention(q, type, c, B, H, T, vp(table), pages, vp(start), None, vp(mask), fl(scale), vp(O), None, None,
                                          vp(ws), sz(n), None)
    for call in (write, read, tree):
        assert call(c=None) == 1 and call(c=cache(pages=0)) == 1 and call(c=cache(k_G=0)) == 1 and call(c=cache(v_G=0)) == 1
        assert call(c=cache(fmt=0)) == 1 and call(c=cache(n=0)) == 1 and call(table=0) == 1 and call(start=0) == 1 and call(B=0) == 1
        assert call(c=cache(P=48)) == 2 and call(c=cache(d=96)) == 2 and call(B=70000) == 2 and call(pages=1 << 27) == 2
        assert call(c=cache(pages=0x1008)) == 4 and call(start=0x1002) == 4
        assert call(type=2) == 1                                                       # fp32
    assert write(k=None) == 1 and write(N=0) == 1 and write(k=_view(0x1001)) == 4
    assert write(pairs=32) == 1 and write(f=0x1000) == 1 and write(positions=0x1000) == 1 and write(f=0x1000, pairs=65) == 2
    assert read(k=None) == 1 and read(N=0) == 1
    assert tree(q=None) == 1 and tree(O=0) == 1 and tree(T=0) == 1 and tree(H=3) == 1 and tree(scale=-1.0) == 1 and tree(scale=math.nan) == 1
    assert tree(T=65) == 2 and tree(mask=0x1004) == 4 and tree(O=0x1008) == 4
    lib.fp4attn_tree_attention_workspace_bytes.restype = sz
    if lib.fp4attn_tree_attention_workspace_bytes(1, 4, 2, 4, 128):
        assert tree(ws=0) == 5 and tree(n=0) == 5 and tree(ws=0x1008) == 4


def test_binding_refuses_what_is_not_on_a_gpu(lib):
    from paper_2609_04105_b200 import binding as Bd
    z = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    i, f = torch.zeros((1, 4), dtype=torch.int32), torch.zeros(32)
    cache = Bd.fp4attn_cache_create(2, 16, 64, Bd.FMT_NVFP4, torch.ones(2), torch.ones(2))
    assert cache.pages.shape == (2, 2, S.record_bytes("nvfp4", 16, 64)) and not cache.pages.any()
    for call in (lambda: Bd.fp4attn_rotary(z, i, f), lambda: Bd.fp4attn_cache_write(cache, z, z, i, i[0, :1]),
                 lambda: Bd.fp4attn_cache_read(cache, i, i[0, :1], 4), lambda: Bd.fp4attn_tree_attention(z, cache, i, i[0, :1])):
        with pytest.raises(AssertionError, match="CUDA"):
            call()
    with pytest.raises(AssertionError, match="dtype"):
        Bd.fp4attn_cache_read(cache, i, i[0, :1], 4, dtype=torch.float32)
    with pytest.raises(AttributeError):
        Bd.fp4attn_tree_attention(z, object(), i, i[0, :1])
    with pytest.raises(Bd.Fp4AttnError):
        Bd.fp4attn_cache_create(2, 16, 96, Bd.FMT_NVFP4, torch.ones(2), torch.ones(2))
    with pytest.raises(Bd.Fp4AttnError):
        Bd.fp4attn_cache_create(2, 16, 64, Bd.FMT_MXFP4, torch.ones(2), torch.ones(2))


def test_rotary_frequencies():
    from paper_2609_04105_b200 import binding as Bd
    f = lambda *a, **kw: Bd.fp4attn_rotary_frequencies(*a, device="cpu", **kw).double()
    plain = f(64)
    assert plain.shape == (32,) and plain[0] == 1.0
    assert torch.allclose(plain[1:] / plain[:-1], torch.full((31,), 10000.0 ** (-2 / 64), dtype=torch.float64), rtol=1e-6)
    assert torch.allclose(f(64, scaling="linear", factor=4.0), plain / 4, rtol=1e-6)
    base = f(64, scaling="base", factor=4.0)
    assert base[0] == 1.0 and torch.allclose(base[-1], plain[-1] / 4, rtol=1e-5)
    parts = f(64, scaling="by_parts", factor=4.0, trained_length=4096)
    turns = 4096 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.allclose(parts[turns <= 1], plain[turns <= 1] / 4, rtol=1e-6)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (parts[between] < plain[between]).all() and (parts[between] > plain[between] / 4).all()
    for bad in (dict(rot_dim=3), dict(rot_dim=64, scaling="other"), dict(rot_dim=64, scaling="by_parts"), dict(rot_dim=64, factor=0.0),
                dict(rot_dim=2, scaling="base")):
        with pytest.raises(ValueError):
            Bd.fp4attn_rotary_frequencies(device="cpu", **bad)
