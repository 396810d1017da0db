"""Pins of the oracle of prompts over a paged cache, shared prefixes and page pools, and what the library refuses without a GPU."""
import ctypes

import numpy as np
import pytest

from oracle import serving as S


def test_scores_against_the_formula():
    rng = np.random.default_rng(1)
    T, n, d = 5, 9, 4
    q, k, v = rng.normal(size=(T, d)), rng.normal(size=(n, d)), rng.normal(size=(n, d))
    mask = S.between(4, T, T, first=[0, 2, 5, 9, 1], last=[5, 6, 7, 9, 40])
    far = np.abs(4 + np.arange(T)[:, None] - np.arange(n)[None])
    o, lse, pv, size, raw = S.attend_scores(q, k, v, mask, 0.7, 1.5, 0.25, far)
    for t in range(T):
        seen = [j for j in range(n) if mask[t, j]]
        if not seen:
            assert t == 3 and not o[t].any() and np.isneginf(lse[t])
            continue
        x = [1.5 * np.tanh(0.7 * q[t] @ k[j] / 1.5) - 0.25 * abs(4 + t - j) for j in seen]
        w = np.exp(x)
        assert np.allclose(o[t], (w[:, None] * v[seen]).sum(0) / w.sum()) and np.isclose(lse[t], np.log(w.sum()))
        assert np.isclose(raw[t], max(abs(0.7 * q[t] @ k[j]) for j in seen))
    a, b = S.attend_scores(q, k, v, mask, 0.7), S.attend(q, k, v, mask, 0.7)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_what_rows_see():
    assert np.array_equal(S.between(2, 3, 3), np.tril(np.ones((3, 5)), 2))
    assert np.array_equal(S.between(2, 3, 1), np.tril(np.ones((3, 3)), 2))
    assert not S.between(0, 2, 0).size
    assert S.between(1, 2, 2, first=[-4, 2], last=[9, 2]).tolist() == [[True] * 3, [False] * 3]


def test_pages_by_hand():
    free, table = [4, 9, 2, 7, 5] + [0] * 7, [[8, -1, -1], [-1, -1, -1], [3, 6, -1]]
    left, slots, positions, fine = S.pages_assign(free, 5, table, [3, 0, 30], [20, 16, 5], 4, 16)
    assert fine and left == 2 and table == [[8, 5, -1], [7, -1, -1], [3, 6, 2]]
    assert slots == [[131, 132, 133, 134], [112, 113, 114, 115], [110, 111, 32, 33]] and positions[2] == [30, 31, 32, 33]
    left, fine = S.pages_release(free, left, table, [23, 16, 35], [3, 0, 30], 16)
    assert fine and left == 5 and free[:5] == [4, 9, 2, 7, 5] and table == [[8, -1, -1], [-1, -1, -1], [3, 6, -1]]


class _View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_longlong) for n in ("b", "h", "n")]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("k_G", ctypes.c_void_p), ("v_G", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("fmt", "P", "num_pages", "kv_heads", "d")]


class _Pool(ctypes.Structure):
    _fields_ = [("free", ctypes.c_void_p), ("count", ctypes.c_void_p), ("turn", ctypes.c_void_p), ("num_pages", ctypes.c_int), ("page_size", ctypes.c_int)]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_04105_b200 import build
    lib = ctypes.CDLL(build.build())
    for n in ("paged_attention", "shared_prefix_attention", "pages_release"):
        getattr(lib, f"fp4attn_{n}_workspace_bytes").restype = ctypes.c_size_t
    return lib


INVALID, SHAPE, ALIGNMENT, WORKSPACE = 1, 2, 4, 5
vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t


def _paged(lib, **kw):
    a = dict(q=_View(0x1000, 512, 128, 128), type=0, cache=_Cache(0x1000, 0x2000, 0x2000, 1, 64, 10, 2, 128), B=1, H=4, T=3, table=0x3000, max_pages=4, context=0x4000,
             count=None, first=None, last=None, scale=0.0, cap=0.0, slopes=None, O=0x5000, LSE=None, status=None, ws=0x6000, bytes=1 << 40)
    a.update(kw)
    return lib.fp4attn_paged_attention(ctypes.byref(a["q"]), i(a["type"]), ctypes.byref(a["cache"]), i(a["B"]), i(a["H"]), i(a["T"]), vp(a["table"]), i(a["max_pages"]),
                                       vp(a["context"]), vp(a["count"]), vp(a["first"]), vp(a["last"]), f(a["scale"]), f(a["cap"]), vp(a["slopes"]), vp(a["O"]),
                                       vp(a["LSE"]), vp(a["status"]), vp(a["ws"]), sz(a["bytes"]), None)


def _shared(lib, **kw):
    a = dict(q=_View(0x1000, 512, 128, 128), type=0, cache=_Cache(0x1000, 0x2000, 0x2000, 1, 64, 10, 2, 128), B=1, H=4, T=3, groups=1, ptable=0x7000, ppages=2,
             length=0x8000, starts=0x9000, table=0x3000, max_pages=4, context=0x4000, count=None, mask=None, scale=0.0, cap=0.0, slopes=None, O=0x5000, LSE=None,
             status=None, ws=0x6000, bytes=1 << 40)
    a.update(kw)
    return lib.fp4attn_shared_prefix_attention(ctypes.byref(a["q"]), i(a["type"]), ctypes.byref(a["cache"]), i(a["B"]), i(a["H"]), i(a["T"]), i(a["groups"]),
                                               vp(a["ptable"]), i(a["ppages"]), vp(a["length"]), vp(a["starts"]), vp(a["table"]), i(a["max_pages"]), vp(a["context"]),
                                               vp(a["count"]), vp(a["mask"]), f(a["scale"]), f(a["cap"]), vp(a["slopes"]), vp(a["O"]), vp(a["LSE"]), vp(a["status"]),
                                               vp(a["ws"]), sz(a["bytes"]), None)


@pytest.mark.parametrize("call", [_paged, _shared])
def test_attention_refusals(lib, call):
    cache = lambda **kw: _Cache(**{**dict(pages=0x1000, k_G=0x2000, v_G=0x2000, fmt=1, P=64, num_pages=10, kv_heads=2, d=128), **kw})
    for kw in (dict(B=0), dict(T=0), dict(H=0), dict(H=3), dict(type=2), dict(type=-1), dict(table=None), dict(context=None), dict(O=None), dict(scale=-1.0),
               dict(scale=float("nan")), dict(cap=-0.5), dict(cap=float("inf")), dict(max_pages=0), dict(cache=cache(fmt=0)), dict(cache=cache(pages=None)),
               dict(cache=cache(k_G=None)), dict(cache=cache(num_pages=0)), dict(q=_View(0, 1, 1, 1))):
        assert call(lib, **kw) == INVALID, kw
    for kw in (dict(cache=cache(d=96)), dict(cache=cache(P=48)), dict(B=65536), dict(max_pages=1 << 24), dict(H=1 << 20, T=2048) if call is _paged else dict(T=65)):
        assert call(lib, **kw) == SHAPE, kw
    for kw in (dict(O=0x5008), dict(LSE=0x5002), dict(status=0x5001), dict(slopes=0x5002), dict(q=_View(0x1001, 1, 1, 1)), dict(ws=0x6008), dict(count=0x4002),
               dict(table=0x3002), dict(first=0x4001) if call is _paged else dict(mask=0x4004)):
        assert call(lib, **kw) == ALIGNMENT, kw
    assert call(lib, ws=None) == WORKSPACE and call(lib, bytes=0) == WORKSPACE
    if call is _shared:
        for kw in (dict(groups=0), dict(ppages=0), dict(ptable=None), dict(length=None), dict(starts=None)):
            assert call(lib, **kw) == INVALID, kw
        assert call(lib, groups=65536) == SHAPE and call(lib, ppages=1 << 24) == SHAPE and call(lib, starts=0x9002) == ALIGNMENT


def test_workspace_sizes(lib):
    paged, shared = lib.fp4attn_paged_attention_workspace_bytes, lib.fp4attn_shared_prefix_attention_workspace_bytes
    assert paged(1, 4, 2, 3, 128) > 0 and shared(1, 4, 2, 3, 128, 1) > 0
    for bad in ((0, 4, 2, 3, 128), (1, 3, 2, 3, 128), (1, 4, 0, 3, 128), (1, 4, 2, 0, 128), (1, 4, 2, 3, 96), (1, 1 << 20, 2, 1 << 11, 128)):
        assert paged(*bad) == 0 and shared(*bad, 1) == 0
    assert shared(1, 4, 2, 3, 128, 0) == 0 and shared(1, 4, 2, 65, 128, 1) == 0
    assert lib.fp4attn_pages_release_workspace_bytes(0) == 0 and lib.fp4attn_pages_release_workspace_bytes(5) >= 24


def test_pool_refusals(lib):
    pool = lambda **kw: _Pool(**{**dict(free=0x1000, count=0x2000, turn=0x2004, num_pages=10, page_size=64), **kw})

    def assign(p=None, B=2, N=3, table=0x3000, max_pages=4, start=0x4000, count=None, slots=0x5000, positions=0x6000, status=None):
        return lib.fp4attn_pages_assign(ctypes.byref(p or pool()), i(B), i(N), vp(table), i(max_pages), vp(start), vp(count), vp(slots), vp(positions), vp(status), None)

    def release(p=None, B=2, table=0x3000, max_pages=4, length=0x4000, keep=None, status=None, ws=0x5000, bytes=1000):
        return lib.fp4attn_pages_release(ctypes.byref(p or pool()), i(B), vp(table), i(max_pages), vp(length), vp(keep), vp(status), vp(ws), sz(bytes), None)

    for call in (assign, release):
        for kw in (dict(B=0), dict(table=None), dict(max_pages=0), dict(p=pool(free=None)), dict(p=pool(count=None)), dict(p=pool(turn=None)), dict(p=pool(num_pages=0)),
                   dict(p=pool(page_size=0))):
            assert call(**kw) == INVALID, kw
        for kw in (dict(B=65536), dict(p=pool(page_size=48)), dict(max_pages=1 << 24)):
            assert call(**kw) == SHAPE, kw
        for kw in (dict(table=0x3002), dict(p=pool(free=0x1001)), dict(status=0x7001)):
            assert call(**kw) == ALIGNMENT, kw
    for kw in (dict(start=None), dict(N=-1), dict(N=0, slots=None, positions=None), dict(N=0, count=0x4000)):
        assert assign(**kw) == INVALID, kw
    assert assign(N=1 << 30) == SHAPE and assign(slots=0x5004) == ALIGNMENT and assign(start=0x4002) == ALIGNMENT
    assert release(length=None) == INVALID and release(keep=0x4001) == ALIGNMENT and release(ws=None) == WORKSPACE and release(bytes=8) == WORKSPACE
