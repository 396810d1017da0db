"""Serving over a quantized, paged key/value cache: what its operators cost, and their plain forms.

  rotary   rotary positions on Q and K, and the backward pass
  write    K (with or without its rotary positions) and V quantized into the pages of a batch, and read back
  read     a batch's K and V out of its pages
  tree     attention of one token, or of a tree of drafted tokens, of every sequence over its pages

A page holds `page` tokens of every KV head; a (page, head) record is K codes, K scales, V codes, V scales:
  nvfp4  K codes [d/32][page][16]: byte j of chunk c = elements 32c+2j (bits 0-3) and 32c+2j+1; K scales [page][d/16], E4M3;
         V codes [page/16][d/2][16]: byte (g, i, t) = elements 2i, 2i+1 of token 16g+t; V scales [d/16][page], E4M3, the tokens of
         each eight in the order 0 4 1 5 2 6 3 7.  A value is code * scale / G.
  e4m3   K [d/16][page][16]: byte j of chunk c = element 16c+j; V [page/16][d][16]: byte (g, i, t) = element i of token 16g+t.
         A value is byte / G.
G is one factor per KV head, fixed beforehand.
"""
import math
import random

import torch

own = False

MOST_KV = 32 * 8 * 32768 * 128          # cached elements of K of one case
MOST_PAIRS = 4 * 32 * 64 * 8192 * 128   # batch x heads x query tokens x keys x head dimension
MOST_ROWS = 2 * 40 * 4096 * 128         # elements of Q and K that are rotated


def _rotary(B, H, kv_heads, N, d, rot, interleaved=False, backward=False, far=131072, dtype="bf16"):
    return {"op": "rotary", "B": B, "H": H, "kv_heads": kv_heads, "N": N, "d": d, "rot": rot, "interleaved": interleaved,
            "backward": backward, "far": far, "dtype": dtype}


def _cached(op, B, kv_heads, N, d, fmt, page, context=0, rotary=False, dtype="bf16", H=0):
    return {"op": op, "B": B, "H": H or kv_heads, "kv_heads": kv_heads, "N": N, "d": d, "fmt": fmt, "page": page,
            "context": context, "rotary": rotary, "dtype": dtype}


def listed():
    return [
        # one new token of every sequence of a batch, far into long contexts
        dict(_rotary(32, 32, 8, 1, 128, 128), name="rotary_step"),
        # a prompt of two sequences, Q and K as they come out of one projection
        dict(_rotary(2, 32, 8, 4096, 128, 128), name="rotary_prompt"),
        # the gradients of a training step: neighbouring pairs, half of each head, an odd length
        dict(_rotary(4, 16, 16, 4095, 64, 32, interleaved=True, backward=True, far=8192), name="rotary_backward"),
        # one new token of every sequence of a batch, its K rotated as it is written
        dict(_cached("write", 32, 8, 1, 128, "nvfp4", 64, context=8192, rotary=True), name="write_step"),
        # prompts, or chunks of them, behind contexts of unlike odd lengths
        dict(_cached("write", 4, 8, 4096, 128, "nvfp4", 64, context=1024), name="write_prompt"),
        # eight bits, small heads, small pages, an odd length
        dict(_cached("write", 1, 16, 8191, 64, "e4m3", 16, dtype="fp16"), name="write_e4m3"),
        # whole contexts back in 16 bits, for a step that reads them so
        dict(_cached("read", 4, 8, 8192, 128, "nvfp4", 64), name="read_context"),
        # a few tokens out of the middle of short sequences
        dict(_cached("read", 3, 4, 130, 64, "e4m3", 32, context=77), name="read_part"),
        # one token of one sequence of ordinary length: launches and the host's share of them
        dict(_cached("tree", 1, 8, 1, 128, "nvfp4", 64, context=1000, H=32), name="token_1k"),
        # one token of every sequence of a serving batch, contexts of up to 32768 tokens
        dict(_cached("tree", 32, 8, 1, 128, "nvfp4", 64, context=32767, H=32), name="token_batch"),
        # sixteen drafted tokens a sequence, eight bits, small heads and pages
        dict(_cached("tree", 8, 4, 16, 64, "e4m3", 16, context=4096, dtype="fp16", H=16), name="tree_16"),
        # the largest trees: as much arithmetic as reading
        dict(_cached("tree", 4, 8, 64, 128, "nvfp4", 64, context=8128, H=32), name="tree_64"),
    ]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    while True:
        op = rng.choices(("rotary", "write", "read", "tree"), (3, 3, 2, 4))[0]
        d = rng.choice((64, 128))
        kv = rng.choice((1, 2, 3, 4, 5, 8, 16))
        group = rng.choice((1, 2, 3, 4, 5, 8))
        B = _log(rng, 1, 64)
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        if op == "rotary":
            N = _log(rng, 1, 8192)
            rot = rng.choice((d, d, d // 2, d // 4, d - 8))
            if B * (group + 1) * kv * N * d > MOST_ROWS:
                continue
            return _rotary(B, group * kv, kv, N, d, rot, rng.random() < 0.5, rng.random() < 0.4, rng.choice((8192, 131072, 1 << 20)),
                           rng.choice((dtype, dtype, "fp32")))
        fmt, page = rng.choice(("nvfp4", "nvfp4", "e4m3")), rng.choice((16, 32, 64, 128))
        if op == "tree":
            N, context = rng.choice((1, 1, 2, 3, 5, 8, 13, 16, 31, 48, 64)), _log(rng, 1, 32768)
            if B * kv * (context + N) * d > MOST_KV or B * kv * group * N * (context + N) * d > MOST_PAIRS:
                continue
            return _cached(op, B, kv, N, d, fmt, page, context, False, dtype, kv * group)
        N, context = _log(rng, 1, 8192), rng.choice((0, _log(rng, 1, 8192)))
        if B * kv * N * d > (4 * 8 * 4096 * 128 if op == "write" else 4 * 8 * 8192 * 128) or B * kv * (N + context) * d > MOST_KV // 4:
            continue
        return _cached(op, B, kv, N, d, fmt, page, context, op == "write" and rng.random() < 0.4, dtype)


_TYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _starts(case):
    """How many tokens each sequence of the batch has behind it: one `context`, the others any number of them."""
    r = random.Random(case["B"] * 1000003 + case["context"])
    most = case["context"]
    return [most] + [r.randint(min(most, max(1, most // 8)), most) for _ in range(case["B"] - 1)]


def _parents(case):
    """A tree of drafted tokens per sequence: the parent of each token, -1 for the roots."""
    r = random.Random(case["B"] * 7919 + case["N"])
    return [[r.randint(max(-1, t - 5), t - 1) for t in range(case["N"])] for _ in range(case["B"])]


def _tree_bits(case):
    """int64 [B, N]: bit j of row t where drafted token t sees token j (its ancestors and itself)."""
    rows = []
    for parents in _parents(case):
        bits = []
        for t, p in enumerate(parents):
            bits.append((bits[p] if p >= 0 else 0) | 1 << t)
        rows.append([b - (1 << 64) if b >> 63 else b for b in bits])
    return torch.tensor(rows, dtype=torch.int64, device="cuda")


def _record(case):
    """Bytes of a (page, head) record, and where K codes, K scales, V codes and V scales begin in it."""
    P, d = case["page"], case["d"]
    codes, scales = (P * d // 2, P * d // 16) if case["fmt"] == "nvfp4" else (P * d, 0)
    return 2 * (codes + scales), (0, codes, codes + scales, 2 * codes + scales)


def _frequencies(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, H, kv, N, d, dtype = case["B"], case["H"], case["kv_heads"], case["N"], case["d"], _TYPE[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"] == "rotary":
        # one projection's output, Q and K side by side
        x = torch.randn((B, N, (H + kv) * d), generator=gen, device="cuda").to(dtype)
        s["q"] = x[..., :H * d].unflatten(2, (H, d)).transpose(1, 2)
        s["k"] = x[..., H * d:].unflatten(2, (kv, d)).transpose(1, 2)
        first = torch.randint(0, max(1, case["far"] - N), (B, 1), generator=gen, device="cuda")
        s["positions"] = (first + torch.arange(N, device="cuda")).to(torch.int32)
        s["inv_freq"] = _frequencies(case["rot"])
        return s
    P = case["page"]
    starts = _starts(case)
    per_seq = -(-(case["context"] + N) // P)
    pages = B * per_seq + 1
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    # the sequences' pages lie where they were free: in no order
    s["table"] = torch.randperm(pages, generator=gen, device="cuda")[:B * per_seq].reshape(B, per_seq).to(torch.int32)
    s["start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    if case["op"] == "write":
        # channels of unlike size, as keys have them
        spread = torch.exp(0.5 * torch.randn((1, 1, kv, d), generator=gen, device="cuda"))
        s["k"] = (spread * torch.randn((B, N, kv, d), generator=gen, device="cuda")).to(dtype).transpose(1, 2)
        s["v"] = torch.randn((B, N, kv, d), generator=gen, device="cuda").to(dtype).transpose(1, 2)
        s["pages"] = torch.zeros((pages, kv, size), dtype=torch.uint8, device="cuda")
        full = 2688.0 if case["fmt"] == "nvfp4" else 448.0
        s["k_G"] = full / (4.5 * spread.reshape(kv, d).amax(1))          # from a calibration: about the largest value
        s["v_G"] = full / (4.5 * torch.ones(kv, device="cuda"))
        s["inv_freq"] = _frequencies(d) if case["rotary"] else None
        return s
    # a cache as it is after earlier steps: every code as often as normally distributed values have it
    s["pages"] = torch.empty((pages, kv, size), dtype=torch.uint8, device="cuda")
    if case["fmt"] == "nvfp4":
        for at, until in ((k_at, ks_at), (v_at, vs_at)):
            x = 2.5 * torch.randn((pages, kv, until - at, 2), generator=gen, device="cuda")
            c = _e2m1_codes(x)
            s["pages"][:, :, at:until] = (c[..., 0] + 16 * c[..., 1]).to(torch.uint8)
        for at, until in ((ks_at, v_at), (vs_at, size)):
            x = 160.0 * torch.exp(0.25 * torch.randn((pages, kv, until - at), generator=gen, device="cuda"))
            s["pages"][:, :, at:until] = _e4m3_bytes(x)
    else:
        s["pages"][:] = _e4m3_bytes(100.0 * torch.randn((pages, kv, size), generator=gen, device="cuda"))
    full = 2688.0 if case["fmt"] == "nvfp4" else 448.0
    s["k_G"] = (full / 4.5) * torch.exp(0.2 * torch.randn(kv, generator=gen, device="cuda"))
    s["v_G"] = (full / 4.5) * torch.exp(0.2 * torch.randn(kv, generator=gen, device="cuda"))
    if case["op"] == "tree":
        # logits a few units apart, as trained heads have them
        s["q"] = (3.0 * torch.randn((B, N, H, d), generator=gen, device="cuda")).to(dtype).transpose(1, 2)
        s["bits"] = _tree_bits(case)
    return s


# ---------------------------------------------------------------- plain forms
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _e2m1_codes(x):
    """To nearest, ties to even: fp32 -> int32 codes, the sign in bit 3."""
    a = x.abs()
    c = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()
    return c + 8 * (x < 0).int()


def _e4m3_bytes(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _e4m3_values(b):
    return b.contiguous().view(torch.float8_e4m3fn).float()


def _e2m1_values(b):
    """uint8 [...] -> fp32 [..., 2]."""
    table = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=b.device)
    pair = torch.stack((table.repeat(16), table.repeat_interleave(16)), 1)
    return pair[b.int()]


def _cos_sin(positions, inv_freq):
    angle = positions.double()[:, None, :, None] * inv_freq.double()
    return angle.cos().float(), angle.sin().float()


def _rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    y = x[..., :rot].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:])
    p, q = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((y.to(x.dtype), x[..., rot:]), -1)


def _scale_place(t):
    """Where in a page's row of V scales token t of the page is."""
    return t - t % 8 + 2 * (t % 4) + t % 8 // 4


def _token_bytes(case, s):
    """Flat offsets in the pages of the bytes of each written token: K codes and scales, V codes and scales; [B, kv, N, bytes]."""
    P, d, kv = case["page"], case["d"], case["kv_heads"]
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    position = s["start"].long()[:, None] + torch.arange(case["N"], device="cuda")
    page = s["table"].long().gather(1, position // P)
    base = ((page[:, None] * kv + torch.arange(kv, device="cuda")[None, :, None]) * size)[..., None]
    t = (position % P)[:, None, :, None]
    n = d // 2 if case["fmt"] == "nvfp4" else d
    j, b = torch.arange(n, device="cuda"), torch.arange(d // 16, device="cuda")
    return (base + k_at + ((j // 16) * P + t) * 16 + j % 16, base + ks_at + t * (d // 16) + b,
            base + v_at + (t // 16 * n + j) * 16 + t % 16, base + vs_at + b * P + _scale_place(t))


def _nvfp4(x, G):
    x = x.float().nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf).unflatten(3, (-1, 16))
    G = G[None, :, None, None]
    scales = _e4m3_bytes(x.abs().amax(-1) * G / 6.0)
    S = _e4m3_values(scales)
    ratio = torch.where(S > 0, G / S, torch.zeros_like(S))
    codes = _e2m1_codes(x * ratio[..., None]).flatten(3)
    return (codes[..., 0::2] + 16 * codes[..., 1::2]).to(torch.uint8), scales


def _plain_write(s):
    case = s["case"]
    k, v, flat = s["k"], s["v"], s["pages"].view(-1)
    if s["inv_freq"] is not None:
        positions = s["start"][:, None] + torch.arange(case["N"], device="cuda", dtype=torch.int32)
        k = _rotate(k, *_cos_sin(positions, s["inv_freq"]), False)
    kc, ks, vc, vs = _token_bytes(case, s)
    out = []
    for x, G, at, scales_at in ((k, s["k_G"], kc, ks), (v, s["v_G"], vc, vs)):
        if case["fmt"] == "nvfp4":
            flat[at], flat[scales_at] = _nvfp4(x, G)
            values = _e2m1_values(flat[at]).flatten(3).unflatten(3, (-1, 16)) * _e4m3_values(flat[scales_at])[..., None]
        else:
            flat[at] = _e4m3_bytes(x.float().nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf) * G[None, :, None, None])
            values = _e4m3_values(flat[at]).unflatten(3, (-1, 16))
        out.append((values.flatten(3) / G[None, :, None, None]).to(x.dtype))
    return out


def _plain_pages(s):
    """Every token of the batch's pages: K and V fp32 [B, kv, pages * page, d]."""
    case = s["case"]
    P, d = case["page"], case["d"]
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    r = s["pages"][s["table"].int()].transpose(1, 2)                    # [B, kv, pages, bytes]
    k, v = r[..., k_at:ks_at], r[..., v_at:vs_at]
    if case["fmt"] == "nvfp4":
        k = _e2m1_values(k.unflatten(3, (d // 32, P, 16)).transpose(3, 4)).flatten(4)            # [B, kv, pages, P, d]
        v = _e2m1_values(v.unflatten(3, (P // 16, d // 2, 16)).transpose(4, 5)).flatten(5).flatten(3, 4)
        ks = _e4m3_values(r[..., ks_at:v_at]).unflatten(3, (P, d // 16))
        place = _scale_place(torch.arange(P, device=r.device))
        vs = _e4m3_values(r[..., vs_at:]).unflatten(3, (d // 16, P))[..., place].transpose(3, 4)
        k = (k.unflatten(4, (-1, 16)) * ks[..., None]).flatten(4)
        v = (v.unflatten(4, (-1, 16)) * vs[..., None]).flatten(4)
    else:
        k = _e4m3_values(k.unflatten(3, (d // 16, P, 16)).transpose(3, 4).flatten(4))
        v = _e4m3_values(v.unflatten(3, (P // 16, d, 16)).transpose(4, 5).flatten(3, 4))
    return k.flatten(2, 3) / s["k_G"][None, :, None, None], v.flatten(2, 3) / s["v_G"][None, :, None, None]


def _plain_read(s):
    case = s["case"]
    at = (s["start"].long()[:, None] + torch.arange(case["N"], device="cuda"))[:, None, :, None].expand(-1, case["kv_heads"], -1, case["d"])
    return [x.gather(2, at).to(_TYPE[case["dtype"]]) for x in _plain_pages(s)]


def _seen(s, keys):
    """Truth values [B, N, keys]: the context, and of the drafted tokens those whose bit is set."""
    case = s["case"]
    drafted = torch.arange(keys, device="cuda")[None] - s["start"].long()[:, None]           # [B, keys]
    bit = (s["bits"][:, :, None] >> drafted.clamp(0, case["N"] - 1)[:, None]) & 1
    return ((drafted < 0)[:, None]) | ((drafted < case["N"])[:, None] & (bit == 1))


def _plain_tree(s):
    case = s["case"]
    B, H, kv, N, d = case["B"], case["H"], case["kv_heads"], case["N"], case["d"]
    k, v = _plain_pages(s)
    q = s["q"].float().unflatten(1, (kv, H // kv)).flatten(2, 3)                               # [B, kv, group * N, d]
    scores = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    scores = scores.unflatten(2, (-1, N)).masked_fill(~_seen(s, k.shape[2])[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul((p / total).flatten(2, 3), v).unflatten(2, (-1, N)).flatten(1, 2)
    return out.to(s["q"].dtype), (top + torch.log(total)).squeeze(-1).flatten(1, 2)


def run(state):
    s, case = state, state["case"]
    if not own:
        if case["op"] == "rotary":
            cos, sin = _cos_sin(s["positions"], s["inv_freq"])
            sin = -sin if case["backward"] else sin
            return [_rotate(x, cos, sin, case["interleaved"]) for x in (s["q"], s["k"])]
        return {"write": _plain_write, "read": _plain_read, "tree": _plain_tree}[case["op"]](s)
    from paper_2609_04105_b200 import binding as fp4
    if case["op"] == "rotary":
        call = fp4.fp4attn_rotary_backward if case["backward"] else fp4.fp4attn_rotary
        return call(s["q"], s["positions"], s["inv_freq"], k=s["k"], interleaved=case["interleaved"])
    if "cache" not in s:                # a program makes it once
        fmt = fp4.FMT_NVFP4 if case["fmt"] == "nvfp4" else fp4.FMT_E4M3
        s["cache"] = fp4.QuantizedCache(s["pages"], s["k_G"], s["v_G"], fmt, case["page"], case["d"])
    if case["op"] == "tree":
        return fp4.fp4attn_tree_attention(s["q"], s["cache"], s["table"], s["start"], tree_mask=s["bits"])
    if case["op"] == "write":
        fp4.fp4attn_cache_write(s["cache"], s["k"], s["v"], s["table"], s["start"], inv_freq=s["inv_freq"])
    return fp4.fp4attn_cache_read(s["cache"], s["table"], s["start"], case["N"], dtype=_TYPE[case["dtype"]])


def work(case):
    B, H, kv, N, d = case["B"], case["H"], case["kv_heads"], case["N"], case["d"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "rotary":
        return {"bytes": 2.0 * size * B * (H + kv) * N * d + 4.0 * B * N, "flops": 3.0 * B * (H + kv) * N * case["rot"]}
    held = 9 / 16 if case["fmt"] == "nvfp4" else 1.0       # bytes of a kept element
    if case["op"] == "write":                               # in, into the cache, out of it, out
        return {"bytes": 2 * B * kv * N * d * (2.0 * size + 2 * held), "flops": 0.0}
    if case["op"] == "read":
        return {"bytes": 2 * B * kv * N * d * (size + held), "flops": 0.0}
    keys = sum(_starts(case)) + B * N
    return {"bytes": 2 * keys * kv * d * held + B * H * N * (2.0 * size * d + 4), "flops": 4.0 * keys * N * H * d}


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_e2m1(y):
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=y.device)
    a = y.abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0)).double()
    q = torch.round(a / step) * step                        # ties to an even multiple: the even code
    assert grid.numel() == 8
    return torch.copysign(q, y)


def _exact_e4m3(y):
    a = y.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    e = torch.where(2.0 ** e > a.clamp(min=2.0 ** -6), e - 1, e)
    step = 2.0 ** (e - 3)
    return torch.copysign((torch.round(a / step) * step).clamp(max=448.0), y)


def _f32(x):
    return x.float().double()


def _exact_rotated(x, positions, inv_freq, interleaved, sign=1.0):
    rot = 2 * inv_freq.numel()
    z = positions.double()[:, None, :, None] * inv_freq.double()
    i = torch.arange(rot // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    x = x.double()
    y = x.clone()
    y[..., first] = x[..., first] * z.cos() - sign * x[..., second] * z.sin()
    y[..., second] = x[..., second] * z.cos() + sign * x[..., first] * z.sin()
    return y


def _exact_held(x, G, fmt):
    """The values that the cache stands for; what the format defines with fp32 roundings is rounded so."""
    G = G.double()[None, :, None, None]
    if fmt == "e4m3":
        return _exact_e4m3(_f32(x * G)) / G
    blocks = x.unflatten(3, (-1, 16))
    S = _exact_e4m3(_f32(_f32(blocks.abs().amax(-1) * G) / 6.0))
    ratio = torch.where(S > 0, _f32(G / S.clamp(min=2.0 ** -9)), torch.zeros_like(S))
    return (_exact_e2m1(_f32(blocks * ratio[..., None])) * S[..., None]).flatten(3) / G


def _exact_pages(s):
    """Byte by byte, from the places that the layout gives each element."""
    case = s["case"]
    P, d, kv = case["page"], case["d"], case["kv_heads"]
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    t, e = torch.arange(P, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    records = s["pages"][s["table"].long()]                              # [B, pages, kv, bytes]

    def e4m3(b):
        b = b.int()
        exponent, mantissa = b >> 3 & 15, b & 7
        a = torch.where(exponent > 0, (8 + mantissa) * 2.0 ** (exponent.double() - 10), mantissa * 2.0 ** -9)
        return torch.where(b > 127, -a, a)

    if case["fmt"] == "e4m3":
        k = e4m3(records[..., k_at + (e // 16 * P + t) * 16 + e % 16])
        v = e4m3(records[..., v_at + (t // 16 * d + e) * 16 + t % 16])
    else:
        def e2m1(b):
            c = b.int() >> (4 * (e % 2)).int() & 15
            a = torch.where((c & 6) > 0, (2 + (c & 1)) * 2.0 ** ((c >> 1 & 3).double() - 2), (c & 1) * 0.5)
            return torch.where(c > 7, -a, a)
        eighth = t % 8
        k = e2m1(records[..., k_at + (e // 32 * P + t) * 16 + e % 32 // 2]) * e4m3(records[..., ks_at + t * (d // 16) + e // 16])
        v = e2m1(records[..., v_at + (t // 16 * (d // 2) + e // 2) * 16 + t % 16]) * \
            e4m3(records[..., vs_at + e // 16 * P + t - eighth + (eighth % 4) * 2 + eighth // 4])
    return [x.permute(0, 2, 1, 3, 4).flatten(2, 3) / G.double()[None, :, None, None] for x, G in ((k, s["k_G"]), (v, s["v_G"]))]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return [_exact_rotated(x, s["positions"], s["inv_freq"], case["interleaved"], -1.0 if case["backward"] else 1.0) for x in (s["q"], s["k"])]
    if case["op"] == "write":
        k, v = s["k"].double(), s["v"].double()
        if s["inv_freq"] is not None:                       # a rotated key is one of the inputs' type
            at = s["start"].long()[:, None] + torch.arange(case["N"], device="cuda")
            k = _exact_rotated(k, at, s["inv_freq"], False).to(s["k"].dtype).double()
        return [_exact_held(k, s["k_G"], case["fmt"]), _exact_held(v, s["v_G"], case["fmt"])]
    starts, N = _starts(case), case["N"]
    if case["op"] == "read":
        k, v = _exact_pages(s)
        return [torch.stack([x[b, :, n:n + N] for b, n in enumerate(starts)]) for x in (k, v)]
    group = case["H"] // case["kv_heads"]
    bits, out, lse = s["bits"].tolist(), [], []
    j = torch.arange(N, device="cuda")
    table = s["table"]
    for b, n in enumerate(starts):                          # a sequence at a time: the doubles of a whole batch are too many
        s["table"] = table[b:b + 1, :-(-(n + N) // case["page"])]
        k, v = (x[0, :, :n + N] for x in _exact_pages(s))
        q = s["q"][b].double().unflatten(0, (-1, group))
        z = torch.einsum("hgtd,hkd->hgtk", q, k) / math.sqrt(case["d"])
        seen = torch.tensor(bits[b], device="cuda")[:, None] >> j & 1
        z[..., n:] = torch.where(seen > 0, z[..., n:], -math.inf)
        lse.append(torch.logsumexp(z, -1).flatten(0, 1))
        out.append(torch.einsum("hgtk,hkd->hgtd", torch.softmax(z, -1), v).flatten(0, 1))
    return torch.stack(out), torch.stack(lse)
