"""Calls of the serving operators one behind another without a wait of the host between them: each reads what the one before has written,
into memory that earlier calls have read.  The kernels begin before their predecessors end, so what is compared is whether any of them saw old
bytes: the results are those of the same calls with a synchronization behind each, bit by bit."""
import pytest
import torch

from test_serving_gpu import FMTS, _bd, _cache, _gen, _i32, _randn, _table

pytestmark = pytest.mark.gpu


def _chain(Bd, fmt, N, seed):
    g = _gen(seed)
    B, H, kv, d, P, length = 48, 8, 4, 128, 32, 700
    per_seq = -(-(length + N) // P)
    s = {"cache": _cache(Bd, fmt, B * per_seq, kv, P, d), "table": _table(g, B, per_seq, B * per_seq), "zero": _i32([0] * B),
         "start": torch.randint(0, length, (B,), generator=g, device="cuda").to(torch.int32), "f": Bd.fp4attn_rotary_frequencies(d),
         "q": _randn(g, B, H, N, d), "turned": torch.empty(B, kv, N, d, dtype=torch.bfloat16, device="cuda"), "length": length, "N": N,
         "new": [(_randn(g, B, kv, N, d), _randn(g, B, kv, N, d)) for _ in range(6)]}
    s["positions"] = s["start"][:, None] + torch.arange(N, device="cuda", dtype=torch.int32)
    s["first"] = (_randn(g, B, kv, length + N, d), _randn(g, B, kv, length + N, d))
    return s


def _run(Bd, s, between):
    """Contexts written once; then new tokens over the old ones, turned in a buffer that every round uses, each time read back and attended to."""
    out = []

    def done(x=()):
        out.extend(x)
        between()
    Bd.fp4attn_cache_write(s["cache"], *s["first"], s["table"], s["zero"])
    done()
    for k, v in s["new"]:
        done(Bd.fp4attn_cache_read(s["cache"], s["table"], s["zero"], s["length"] + s["N"]))
        Bd.fp4attn_rotary(k, s["positions"], s["f"], q_out=s["turned"])
        done()
        Bd.fp4attn_cache_write(s["cache"], s["turned"], v, s["table"], s["start"])
        done()
        done(Bd.fp4attn_cache_read(s["cache"], s["table"], s["start"], s["N"]))
        done(Bd.fp4attn_tree_attention(s["q"], s["cache"], s["table"], s["start"]))
    done(Bd.fp4attn_cache_read(s["cache"], s["table"], s["zero"], s["length"] + s["N"]))
    return out


@pytest.mark.parametrize("N", [1, 5, 33])
@pytest.mark.parametrize("fmt", FMTS)
def test_new_data_between_reads(fmt, N):
    Bd = _bd()
    s = _chain(Bd, fmt, N, 60 + N)
    want = [x.clone() for x in _run(Bd, s, torch.cuda.synchronize)]
    assert not torch.equal(want[2], want[6])
    for _ in range(3):
        got = _run(Bd, s, lambda: None)
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run(Bd, s, lambda: None)
    for _ in range(2):
        for x in got:
            x.zero_()
        s["cache"].pages.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
