"""Rotary positions under autograd: recorded, differentiated again, refused where a result could not carry a gradient."""
import pytest
import torch


def _formula(x, positions, f, interleaved, sign, factor):
    pairs = f.numel()
    th = positions.double()[:, None, :, None] * f.double()
    c, s = factor * th.cos(), sign * factor * th.sin()
    a, b = (x[..., :2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    p, r = a * c - b * s, b * c + a * s
    return torch.cat((torch.stack((p, r), -1).flatten(-2) if interleaved else torch.cat((p, r), -1), x[..., 2 * pairs:]), -1)


class _Fake:
    """The native module's call in 64 bits on the CPU, with its answer where gradients are recorded."""

    def rotary(self, q, k, positions, f, interleaved, transposed, factor, q_out, k_out):
        if torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in (q, k)):
            return NotImplemented
        assert all(x is None or x.stride(-1) == 1 for x in (q, k))
        out = [_formula(x, positions, f, interleaved, -1.0 if transposed else 1.0, factor) for x in (q, k) if x is not None]
        return out[0] if k is None else tuple(out)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("with_k", [False, True])
def test_recorded_function(monkeypatch, interleaved, with_k):
    """Its gradients, and theirs, against differences; an input that takes none gives an output that needs none."""
    from paper_2609_04105_b200 import binding as Bd
    monkeypatch.setattr(Bd, "_native_module", _Fake())
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(2, h, 3, 10, generator=g, dtype=torch.float64, requires_grad=True) for h in (2, 1))
    pos, f = torch.tensor([[0, 5, 1000], [3, 2, 1]], dtype=torch.int32), torch.tensor([1.0, 0.1, 0.01])
    for call in (Bd.fp4attn_rotary, Bd.fp4attn_rotary_backward):
        def fn(q, k=None):
            return call(q, pos, f, k=k, interleaved=interleaved, attention_factor=0.8)
        inputs = (q, k) if with_k else (q,)
        assert torch.autograd.gradcheck(fn, inputs) and torch.autograd.gradgradcheck(fn, inputs)
        fn(q).sum().backward()                              # a gradient broadcast along every axis
    if with_k:
        a, b = fn(q.detach(), k)
        assert not a.requires_grad and b.requires_grad
        a, b = fn(q, k)
        assert torch.autograd.grad(b.sum(), (q, k), allow_unused=True)[0] is None
    with torch.no_grad():
        assert not fn(q).requires_grad


def _inputs(seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, N, d = 2, 37, 64
    q = torch.randn(B, N, 3, d, generator=g, device="cuda").to(dtype).transpose(1, 2).requires_grad_()
    k = torch.randn(B, 1, N, d, generator=g, device="cuda").to(dtype).requires_grad_()
    pos = torch.randint(0, 1 << 17, (B, N), generator=g, device="cuda").to(torch.int32)
    w = [torch.randn(B, h, N, d, generator=g, device="cuda").to(dtype) for h in (3, 1)]
    return q, k, pos, w


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_are_those_of_the_formula(dtype, interleaved):
    """Those of the call by hand, bit by bit; and the formula's within three roundings of fp32 of the pair and the type's rounding."""
    from paper_2609_04105_b200 import binding as Bd
    q, k, pos, w = _inputs(3, dtype)
    f = Bd.fp4attn_rotary_frequencies(48)
    how = dict(interleaved=interleaved, attention_factor=1.25)
    a, b = Bd.fp4attn_rotary(q, pos, f, k=k, **how)
    with torch.no_grad():
        plain = Bd.fp4attn_rotary(q, pos, f, k=k, **how)
    assert a.requires_grad and b.requires_grad and torch.equal(a, plain[0]) and torch.equal(b, plain[1]) and not plain[0].requires_grad
    dq, dk = torch.autograd.grad((a, b), (q, k), w)
    hand = Bd.fp4attn_rotary_backward(w[0], pos, f, k=w[1], **how)
    assert torch.equal(dq, hand[0]) and torch.equal(dk, hand[1])
    for x, y, dx in ((q, w[0], dq), (k, w[1], dk)):
        z = x.detach().double().requires_grad_()
        _formula(z, pos, f, interleaved, 1.0, 1.25).backward(y.double())
        half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
        assert ((dx.double() - z.grad).abs() <= half * z.grad.abs() + 4 * 2.0 ** -24 * 2 * 1.25 * y.double().abs().max() + 2.0 ** -25).all()
    # of one output alone, of a sum (a gradient of stride 0), through a broadcast input, and again
    c, e = Bd.fp4attn_rotary(q, pos, f, k=k, **how)
    assert torch.autograd.grad(e.sum(), q, allow_unused=True, retain_graph=True)[0] is None
    ones = torch.ones_like(k)
    assert torch.equal(torch.autograd.grad(e.sum(), k)[0], Bd.fp4attn_rotary_backward(ones, pos, f, **how))
    one = q.detach()[:1, :1].clone().requires_grad_()
    got = torch.autograd.grad(Bd.fp4attn_rotary(one.expand(2, 3, 37, 64), pos, f, **how), one, w[0])[0]
    assert torch.allclose(got.double(), hand[0].double().sum((0, 1), keepdim=True), rtol=0, atol=6 * 2 * half * 1.25 * 2 * w[0].double().abs().max().item())
    if dtype == torch.float32:
        dy = w[0].clone().requires_grad_()
        dx = torch.autograd.grad(Bd.fp4attn_rotary(q, pos, f, **how), q, dy, create_graph=True)[0]
        again = torch.autograd.grad(dx, dy, q.detach())[0]
        assert torch.equal(again, Bd.fp4attn_rotary(q.detach(), pos, f, **how))


@pytest.mark.gpu
def test_refused_where_a_result_could_not_carry_a_gradient():
    from paper_2609_04105_b200 import binding as Bd
    q, k, pos, _ = _inputs(4, torch.bfloat16)
    f = Bd.fp4attn_rotary_frequencies(64)
    out = torch.zeros_like(q.detach())
    for call in (lambda: Bd.fp4attn_rotary(q, pos, f, q_out=out), lambda: Bd.fp4attn_rotary(q.detach(), pos, f, k=k, q_out=out),
                 lambda: Bd.fp4attn_rotary(q, pos, f, q_out=q), lambda: Bd.fp4attn_rotary_backward(q, pos, f, q_out=out),
                 lambda: Bd.fp4attn_rotary(q.detach(), pos, f.clone().requires_grad_())):
        with pytest.raises(AssertionError, match="gradient"):
            call()
    assert not out.any()
    with torch.no_grad():
        assert Bd.fp4attn_rotary(q, pos, f, q_out=out) is out and out.any()


@pytest.mark.gpu
def test_captured_step():
    """Forward and gradient in one graph, replayed with new contents."""
    from paper_2609_04105_b200 import binding as Bd
    q, k, pos, w = _inputs(5, torch.bfloat16)
    f = Bd.fp4attn_rotary_frequencies(64)

    def step():
        return torch.autograd.grad(Bd.fp4attn_rotary(q, pos, f, k=k), (q, k), w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        pos.add_(11)
        w[0].mul_(-1.5)
        graph.replay()
        want = Bd.fp4attn_rotary_backward(w[0], pos, f, k=w[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
