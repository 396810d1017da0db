"""Instances of the kernels of attention over a paged cache that few calls reach: caps alone and biases alone at every number of rows of a KV head,
workspaces exactly as long as asked for, no LSE wanted, outputs of the caller's."""
import ctypes

import numpy as np
import pytest
import torch

from test_paged_gpu import _check_paged, _check_shared, _masks, _shared
from test_serving_gpu import FMTS, _bd, _filled, _gen, _i32, _randn, _tree_bits
from test_serving_workspace import _Cache, _View

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["causal", "documents"])
@pytest.mark.parametrize("fmt,d", [(f, d) for f in FMTS for d in (64, 128)])
@pytest.mark.parametrize("H,kv,T", [(8, 2, 5), (12, 3, 12), (8, 2, 16), (4, 2, 50), (4, 2, 64), (3, 3, 128)])
def test_a_cap_alone_and_a_bias_alone(H, kv, T, fmt, d, kind):
    """20 to 128 rows of a KV head: kept four times, twice and once among the lanes."""
    Bd, g = _bd(), _gen(H * T + d)
    context = [500, 0, 77]
    cache, table = _filled(Bd, g, fmt, 3, kv, 32, d, max(context) + T)
    q = _randn(g, 3, H, T, d, scale=2.0)
    counts = [T, T - 3, T]
    first = None if kind == "causal" else _masks(np.random.default_rng(T), 3, T, context, kind)[0]
    slopes = 2.0 ** -(torch.arange(H, device="cuda") % 9 + 1.0)
    for kw in (dict(cap=15.0), dict(cap=1.0), dict(slopes=slopes), dict(slopes=-0.01 * slopes)):
        got = Bd.fp4attn_paged_attention(q, cache, table, _i32(context), count=_i32(counts), first=None if first is None else _i32(first.tolist()),
                                         soft_cap=kw.get("cap", 0.0), slopes=kw.get("slopes"))
        _check_paged(got, q, cache, table, context, counts, first, **kw)


@pytest.mark.parametrize("fmt,d", [(f, d) for f in FMTS for d in (64, 128)])
@pytest.mark.parametrize("H,kv,T,starts", [(8, 2, 1, [0, 2, 6]), (6, 2, 5, [0, 6, 6]), (4, 2, 20, [1, 2, 6]), (2, 2, 64, [0, 3, 6])])
def test_a_cap_alone_and_a_bias_alone_over_shared_prefixes(H, kv, T, starts, fmt, d):
    """Prefixes of 8 to 192 rows of a KV head, sequences of 4 to 64, with and without a tree."""
    Bd, g = _bd(), _gen(H * T + d)
    prefixes, context = [333, 60], [0, 130, 7, 64, 31, 200]
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, 32, d, prefixes, context, T)
    q = _randn(g, 6, H, T, d, scale=2.0)
    slopes = 2.0 ** -(torch.arange(H, device="cuda") % 9 + 1.0)
    for bits in (None, _tree_bits(np.random.default_rng(T), 6, T)):
        for kw in (dict(cap=15.0), dict(cap=1.0), dict(slopes=slopes), dict(slopes=-0.01 * slopes)):
            got = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, _i32(prefixes), _i32(starts), table, _i32(context), tree_mask=bits,
                                                     soft_cap=kw.get("cap", 0.0), slopes=kw.get("slopes"))
            _check_shared(got, q, cache, prefix_table, prefixes, starts, table, context, None if bits is None else bits.tolist(), **kw)


GUARD = 1 << 16


def _guarded(n):
    return torch.full((n + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")


def _p(x):
    return ctypes.c_void_p(None if x is None else x.data_ptr())


def _cache_of(cache):
    return _Cache(cache.pages.data_ptr(), cache.k_G.data_ptr(), cache.v_G.data_ptr(), cache.fmt, cache.page_size, len(cache.pages), cache.k_G.numel(), cache.d)


def _held_to_the_end(Bd, ws, n, call, want):
    """call(workspace, bytes, O, LSE) -> status: refused for a byte less; with exactly n, LSE wanted and not, the bits of `want` and nothing written behind."""
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    assert call(ws, n - 1, out, lse) == Bd.ERR_WORKSPACE
    for l in (lse, None):
        out.fill_(7.0)
        ws.fill_(0xA5)
        assert call(ws, n, out, l) == Bd.OK
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert (ws[n:] == 0xA5).all() and (ws[:n] != 0xA5).any()


@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
@pytest.mark.parametrize("group,T,window,cap", [(1, 1, 0, 0.0), (3, 2, 500, 20.0), (4, 3, 0, 0.0), (4, 3, 700, 0.0), (8, 4, 0, 0.0), (8, 4, 900, 0.0), (4, 10, 0, 30.0),
                                                (4, 20, 5000, 0.0), (4, 32, 0, 0.0), (4, 100, 0, 0.0), (4, 300, 3000, 9.0)])
def test_nothing_behind_the_workspace_of_paged_attention(fmt, d, group, T, window, cap):
    """4 to 1200 rows of a KV head; every item falls to several blocks, so that each block leaves its two parts."""
    Bd, g = _bd(), _gen(d + T)
    B, kv, P, context = 5, 2, 32, 12000
    cache, table = _filled(Bd, g, fmt, 1, kv, P, d, context + T)
    table = table.expand(B, -1).contiguous()
    q, ctx, H = _randn(g, B, group * kv, T, d), _i32([context] * B), group * kv
    first = None
    if window:
        first = (context + 1 - window + torch.arange(T, device="cuda", dtype=torch.int32)).expand(B, T).contiguous()
    want = Bd.fp4attn_paged_attention(q, cache, table, ctx, first=first, soft_cap=cap)
    lib = Bd.lib()
    size = lib.fp4attn_paged_attention_workspace_bytes
    size.restype = ctypes.c_size_t
    n = size(B, H, kv, T, d)

    def call(ws, given, out, lse):
        return lib.fp4attn_paged_attention(ctypes.byref(_View(q.data_ptr(), *q.stride()[:3])), 0, ctypes.byref(_cache_of(cache)), B, H, T, _p(table), table.shape[1], _p(ctx),
                                           None, _p(first), None, ctypes.c_float(0.0), ctypes.c_float(cap), None, _p(out), _p(lse), None, _p(ws), ctypes.c_size_t(given),
                                           ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))

    _held_to_the_end(Bd, _guarded(n), n, call, want)


@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
@pytest.mark.parametrize("H,kv,T,starts", [(4, 2, 1, [0, 9]), (8, 2, 4, [0, 1, 40, 41]), (2, 2, 64, [3, 5, 5, 9]), (6, 1, 1, [0, 300])])
def test_nothing_behind_the_workspace_of_shared_prefixes(fmt, d, H, kv, T, starts):
    """Groups of unlike sizes, an empty one, entries in none; prefixes that fall to many blocks and sequences that one has whole."""
    Bd, g = _bd(), _gen(d + T)
    B, groups, P = max(starts) + (1 if starts[0] else 0), len(starts) - 1, 16
    prefixes, context = [5000, 300, 77][:groups], [(17 * i) % 90 for i in range(B)]
    cache, prefix_table, table = _shared(Bd, g, fmt, kv, P, d, prefixes, context, T)
    q, ctx, length, start = _randn(g, B, H, T, d), _i32(context), _i32(prefixes), _i32(starts)
    want = Bd.fp4attn_shared_prefix_attention(q, cache, prefix_table, length, start, table, ctx)
    lib = Bd.lib()
    size = lib.fp4attn_shared_prefix_attention_workspace_bytes
    size.restype = ctypes.c_size_t
    n = size(B, H, kv, T, d, groups)

    def call(ws, given, out, lse):
        return lib.fp4attn_shared_prefix_attention(ctypes.byref(_View(q.data_ptr(), *q.stride()[:3])), 0, ctypes.byref(_cache_of(cache)), B, H, T, groups, _p(prefix_table),
                                                   prefix_table.shape[1], _p(length), _p(start), _p(table), table.shape[1], _p(ctx), None, None, ctypes.c_float(0.0),
                                                   ctypes.c_float(0.0), None, _p(out), _p(lse), None, _p(ws), ctypes.c_size_t(given),
                                                   ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))

    _held_to_the_end(Bd, _guarded(n), n, call, want)


class _Pool(ctypes.Structure):
    _fields_ = [("free", ctypes.c_void_p), ("count", ctypes.c_void_p), ("turn", ctypes.c_void_p), ("num_pages", ctypes.c_int), ("page_size", ctypes.c_int)]


@pytest.mark.parametrize("B,per", [(1, 3), (257, 5), (3, 700)])
def test_nothing_behind_the_workspace_of_a_release_or_behind_the_stack(B, per):
    Bd, P = _bd(), 16
    pages = B * per
    stack, table = torch.full((pages + GUARD,), -7, dtype=torch.int32, device="cuda"), torch.full((B * per + GUARD,), -7, dtype=torch.int32, device="cuda")
    table[:pages] = torch.randperm(pages, device="cuda").to(torch.int32)
    want = table[:pages].flip(0)
    count, turn, length = _i32([0]), _i32([0]), _i32([per * P] * B)
    size = Bd.lib().fp4attn_pages_release_workspace_bytes
    size.restype = ctypes.c_size_t
    n = size(B)
    ws = _guarded(n)
    pool = _Pool(stack.data_ptr(), count.data_ptr(), turn.data_ptr(), pages, P)
    for given, rc in ((n - 1, Bd.ERR_WORKSPACE), (n, Bd.OK)):
        assert Bd.lib().fp4attn_pages_release(ctypes.byref(pool), B, _p(table), per, _p(length), None, None, _p(ws), ctypes.c_size_t(given),
                                              ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == rc
    assert torch.equal(stack[:pages], want) and (stack[pages:] == -7).all() and (table[:pages] == -1).all() and (table[pages:] == -7).all()
    assert count.item() == pages and (ws[n:] == 0xA5).all()


@pytest.mark.parametrize("T", [2, 131])
def test_outputs_of_the_callers(T):
    """O and LSE of the caller's, at every alignment that O may have: the rows behind a count keep what stood there."""
    Bd, g = _bd(), _gen(31 + T)
    B, H, kv, d, P = 2, 4, 2, 64, 16
    cache, table = _filled(Bd, g, "nvfp4", B, kv, P, d, 100 + T)
    q, counts = _randn(g, B, H, T, d), [T, T - 1]
    calls = [lambda **kw: Bd.fp4attn_paged_attention(q, cache, table, _i32([100, 3]), count=_i32(counts), **kw)]
    if T <= 64:
        calls.append(lambda **kw: Bd.fp4attn_shared_prefix_attention(q, cache, table[:1], _i32([40]), _i32([0, 2]), table, _i32([100, 3]), count=_i32(counts), **kw))
    for call in calls:
        want = call()
        for shift in (0, 8):                                        # 32 and 16 bytes
            room = torch.full((B * H * T * d + 8,), 3.0, dtype=q.dtype, device="cuda")
            out, lse = room[shift:shift + B * H * T * d].view(B, H, T, d), torch.full((B, H, T), 5.0, device="cuda")
            got = call(out=out, lse=lse)
            assert got[0] is out and got[1] is lse
            for b, n in enumerate(counts):
                assert torch.equal(out[b, :, :n], want[0][b, :, :n]) and torch.equal(lse[b, :, :n], want[1][b, :, :n])
                assert (out[b, :, n:] == 3.0).all() and (lse[b, :, n:] == 5.0).all()
