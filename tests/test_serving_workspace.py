"""The workspace of tree attention is that of the kernel which will run: two partial results (O, maximum and sum of a row tile) per block."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def size():
    from paper_2609_04105_b200 import build
    call = ctypes.CDLL(build.build()).fp4attn_tree_attention_workspace_bytes
    call.restype = ctypes.c_size_t
    return call


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,T,R,blocks", [(4, 1, 8, 640), (8, 1, 8, 640), (4, 4, 16, 640), (9, 1, 16, 640), (4, 8, 32, 160), (33, 1, 64, 160), (4, 64, 64, 160)])
def test_workspace_is_what_the_call_can_touch(size, heads, T, R, blocks, d):
    for B, kv in ((1, 1), (7, 8)):
        rows = heads * T
        split = 8 * B * kv * -(-rows // R)
        assert 0 < size(B, heads * kv, kv, T, d) <= 2 * blocks * R * (4 * d + 8) + split + 16


class _View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_longlong), ("sh", ctypes.c_longlong), ("sn", ctypes.c_longlong)]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("k_G", ctypes.c_void_p), ("v_G", ctypes.c_void_p), ("fmt", ctypes.c_int),
                ("page_size", ctypes.c_int), ("num_pages", ctypes.c_int), ("kv_heads", ctypes.c_int), ("d", ctypes.c_int)]


@pytest.mark.gpu
@pytest.mark.parametrize("group,T", [(1, 1), (3, 4), (4, 8), (4, 16), (4, 64)])
@pytest.mark.parametrize("fmt,d", [("nvfp4", 128), ("e4m3", 64)])
def test_nothing_behind_the_workspace_is_written(size, fmt, d, group, T):
    """Items that all fall to several blocks, so that every block leaves its two parts; the workspace exactly as long as asked for."""
    import torch
    from test_serving_gpu import _bd, _filled, _gen, _i32, _randn
    Bd, g = _bd(), _gen(d + T)
    B, kv, P, context = 5, 2, 32, 20000
    cache, table = _filled(Bd, g, fmt, 1, kv, P, d, context + T)
    table = table.expand(B, -1).contiguous()
    q = _randn(g, B, group * kv, T, d)
    want = Bd.fp4attn_tree_attention(q, cache, table, _i32([context] * B))
    n = size(B, group * kv, kv, T, d)
    ws = torch.full((n + 65536,), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse, ctx = torch.empty_like(want[0]), torch.empty_like(want[1]), _i32([context] * B)
    p = ctypes.c_void_p
    c = _Cache(cache.pages.data_ptr(), cache.k_G.data_ptr(), cache.v_G.data_ptr(), cache.fmt, P, cache.pages.shape[0], kv, d)
    call = Bd.lib().fp4attn_tree_attention
    call.restype = ctypes.c_int
    for given, rc in ((n - 1, Bd.ERR_WORKSPACE), (n, Bd.OK)):
        assert call(ctypes.byref(_View(q.data_ptr(), *q.stride()[:3])), 0, ctypes.byref(c), B, group * kv, T, p(table.data_ptr()), table.shape[1],
                    p(ctx.data_ptr()), None, None, ctypes.c_float(0.0), p(out.data_ptr()), p(lse.data_ptr()), None, p(ws.data_ptr()),
                    ctypes.c_size_t(given), p(torch.cuda.current_stream().cuda_stream)) == rc
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and (ws[n:] == 0xA5).all() and (ws[:n] != 0xA5).any()
