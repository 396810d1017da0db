"""Serving whole prompts and shared prefixes over the quantized, paged key/value cache: what its operators cost, and their plain forms.

  paged    attention of any number of tokens of every sequence over its pages: a token, a prompt's chunk, a whole prompt; scores capped
           by a tanh or with a bias by distance, rows that see a document, a window or a prefix
  shared   attention of a batch whose sequences share long prefixes: a prefix is read once for all of its sequences
  pages    pages out of a stack of free ones for the next tokens of a batch, the tokens' slots and positions, and the pages back

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

MOST_KV = 32 * 8 * 32768 * 128          # cached elements of K that the sequences of one case see, a shared one once for each
MOST_SCORES = 32 * 2048 * 32768         # heads x query tokens x keys of one case
MOST_SLOTS = 48 * 16384                 # tokens that get slots


def _paged(B, H, kv_heads, N, d, fmt, page, context, mask="causal", cap=0.0, bias=False, ragged=False, dtype="bf16"):
    return {"op": "paged", "B": B, "H": H, "kv_heads": kv_heads, "N": N, "d": d, "fmt": fmt, "page": page, "context": context,
            "mask": mask, "cap": cap, "bias": bias, "ragged": ragged, "dtype": dtype}


def _shared(B, groups, H, kv_heads, N, d, fmt, page, prefix, context, dtype="bf16"):
    return {"op": "shared", "B": B, "groups": groups, "H": H, "kv_heads": kv_heads, "N": N, "d": d, "fmt": fmt, "page": page,
            "prefix": prefix, "context": context, "dtype": dtype}


def _pages(B, N, page, context, ragged=False):
    return {"op": "pages", "B": B, "N": N, "page": page, "context": context, "ragged": ragged}


def listed():
    return [
        # one token of every sequence of a serving batch, a model that caps its scores
        dict(_paged(32, 32, 8, 1, 128, "nvfp4", 64, 32767, cap=50.0), name="step_capped"),
        # one token of a few sequences, layers that look back over a window, a bias by distance
        dict(_paged(8, 16, 4, 1, 64, "e4m3", 16, 30000, mask="window", bias=True, dtype="fp16"), name="step_window"),
        # the rest of a short prompt behind what is cached already: launches and the host's share of them
        dict(_paged(1, 32, 8, 131, 128, "nvfp4", 64, 1000), name="chunk_short"),
        # whole prompts
        dict(_paged(2, 32, 8, 4096, 128, "nvfp4", 64, 0), name="prompt"),
        # documents packed into sequences of odd lengths, capped scores
        dict(_paged(2, 32, 8, 4095, 128, "nvfp4", 64, 0, mask="documents", cap=30.0, ragged=True), name="prompt_documents"),
        # a prefix that sees itself whole, a bias by distance, small heads, eight bits
        dict(_paged(4, 16, 4, 2047, 64, "e4m3", 32, 500, mask="prefix", bias=True, dtype="fp16"), name="prompt_prefix"),
        # a chunk of a long prompt, far into it
        dict(_paged(1, 32, 8, 2048, 128, "nvfp4", 128, 30720), name="chunk_long"),
        # a few sequences behind a short common prefix
        dict(_shared(4, 1, 32, 8, 1, 128, "nvfp4", 64, 1000, 100), name="shared_small"),
        # one token of every sequence of a batch behind one long prompt (a system's, a book's)
        dict(_shared(48, 1, 32, 8, 1, 128, "nvfp4", 64, 16000, 900), name="shared_batch"),
        # drafted tokens of sequences in groups of unlike sizes, each with a prefix of its own
        dict(_shared(40, 6, 16, 4, 5, 64, "e4m3", 16, 4100, 333, dtype="fp16"), name="shared_groups"),
        # the next token of a large batch: few new pages, in the order of the sequences
        dict(_pages(1024, 1, 64, 8000), name="pages_step"),
        # prompts of unlike lengths
        dict(_pages(48, 16384, 16, 900, ragged=True), name="pages_prompt"),
    ]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    while True:
        op = rng.choices(("paged", "shared", "pages"), (6, 4, 2))[0]
        if op == "pages":
            B, N = _log(rng, 1, 4096), rng.choice((1, 1, _log(rng, 2, 16384)))
            if B * N > MOST_SLOTS:
                continue
            return _pages(B, N, rng.choice((16, 32, 64, 128)), _log(rng, 1, 30000), rng.random() < 0.5)
        d, fmt, page = rng.choice((64, 128)), rng.choice(("nvfp4", "nvfp4", "e4m3")), rng.choice((16, 32, 64, 128))
        kv, group = rng.choice((1, 2, 3, 4, 5, 8)), rng.choice((1, 2, 3, 4, 5, 8))
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        if op == "paged":
            B, N, context = _log(rng, 1, 32), rng.choice((1, 2, _log(rng, 2, 64), _log(rng, 65, 4096), _log(rng, 65, 4096))), rng.choice((0, _log(rng, 1, 32000)))
            if B * kv * (context + N) * d > MOST_KV or B * kv * group * N * (context + N) > MOST_SCORES:
                continue
            return _paged(B, kv * group, kv, N, d, fmt, page, context, rng.choice(("causal", "window", "documents", "prefix")),
                          rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.3, rng.random() < 0.4, dtype)
        groups = rng.choice((1, 1, 2, 5))
        B, N = groups - 1 + _log(rng, 1, 64), rng.choice((1, 1, 1, 4, 7, 16))
        prefix, context = _log(rng, 100, 20000), _log(rng, 1, 2000)
        if B * kv * (prefix + context + N) * d > MOST_KV or B * kv * group * N * (prefix + context + N) > MOST_SCORES:
            continue
        return _shared(B, groups, kv * group, kv, N, d, fmt, page, prefix, context, dtype)


_TYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- what a case is made of, the same for every seed
def _spread(case, most, n, salt):
    """`most`, and n - 1 other numbers up to it."""
    r = random.Random(case["B"] * 1000003 + most * 31 + salt)
    return [most] + [r.randint(min(most, max(1, most // 8)), most) for _ in range(n - 1)]


def _starts(case):
    return _spread(case, case["context"], case["B"], 1)


def _counts(case):
    """How many of the N tokens each sequence has."""
    return _spread(case, case["N"], case["B"], 2) if case.get("ragged") else [case["N"]] * case["B"]


def _seen(case):
    """Lists [B][N]: the first position that a token sees, and the one behind the last."""
    firsts, lasts = [], []
    for b, (start, n) in enumerate(zip(_starts(case), _counts(case))):
        r = random.Random(b * 7919 + start)
        first, last = [0] * case["N"], [start + t + 1 for t in range(case["N"])]
        if case["mask"] == "window":
            first = [max(0, x - 4096) for x in last]
        elif case["mask"] == "documents":
            bounds = [0]
            while bounds[-1] < start + case["N"]:
                bounds.append(bounds[-1] + _log(r, 16, 3000))
            i = 0
            for t in range(case["N"]):
                while bounds[i + 1] <= start + t:
                    i += 1
                first[t] = bounds[i]
        elif case["mask"] == "prefix":
            prefix = r.randint(0, start + n)
            last = [max(x, prefix) for x in last]
        firsts.append(first)
        lasts.append(last)
    return firsts, lasts


def _members(case):
    """Where the sequences of each group begin, and B."""
    r = random.Random(case["B"] * 31 + case["groups"])
    return [0] + sorted(r.sample(range(1, case["B"]), case["groups"] - 1)) + [case["B"]]


def _prefixes(case):
    return _spread(case, case["prefix"], case["groups"], 3)


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
        rows.append(bits)
    return rows


def _record(case):
    """Bytes of a (page, head) record, and where K codes, K scales, V codes and V scales begin in it."""
    P, d = case["page"], case["d"]
    codes, scales = (P * d // 2, P * d // 16) if case["fmt"] == "nvfp4" else (P * d, 0)
    return 2 * (codes + scales), (0, codes, codes + scales, 2 * codes + scales)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, N, P = case["B"], case["N"], case["page"]
    s = {"case": dict(case), "start": _i32(_starts(case)), "count": _i32(_counts(case))}
    per_seq = -(-(case["context"] + N) // P)
    if case["op"] == "pages":
        # what is held already, and the rest of the pool, in the order in which pages have come back
        held = [-(-x // P) for x in _starts(case)]
        new = sum(-(-(x + n) // P) for x, n in zip(_starts(case), _counts(case))) - sum(held)
        total = sum(held) + new + 7
        order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.full((B, per_seq), -1, dtype=torch.int32, device="cuda")
        has = torch.arange(per_seq, device="cuda")[None] < _i32(held)[:, None]
        s["table"][has] = order[:sum(held)]
        s["free"] = torch.cat((order[sum(held):], order[:sum(held)] * 0))
        s["free_count"] = _i32([total - sum(held)])
        return s
    H, kv, d, dtype = case["H"], case["kv_heads"], case["d"], _TYPE[case["dtype"]]
    groups = case.get("groups", 0)
    per_group = -(-case["prefix"] // P) if groups else 0
    pages = B * per_seq + groups * per_group + 1
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    # the sequences' pages lie where they were free: in no order
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    s["table"] = order[:B * per_seq].reshape(B, per_seq)
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
    # logits a few units apart, as trained heads have them; heads side by side, as a projection leaves them
    s["q"] = (3.0 * torch.randn((B, N, H, d), generator=gen, device="cuda")).to(dtype).transpose(1, 2)
    if groups:
        s["prefix_table"] = order[B * per_seq:B * per_seq + groups * per_group].reshape(groups, per_group)
        s["prefix_length"], s["group_start"] = _i32(_prefixes(case)), _i32(_members(case))
        s["bits"] = torch.tensor(_tree_bits(case), dtype=torch.int64, device="cuda")
        return s
    if not case["ragged"]:
        s["count"] = None
    s["first"] = s["last"] = s["slopes"] = None
    if case["mask"] in ("window", "documents"):
        s["first"] = _i32(_seen(case)[0])
    elif case["mask"] == "prefix":
        s["last"] = _i32(_seen(case)[1])
    if case["bias"]:
        # a slope per head, from steep to flat
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(H, device="cuda") + 1.0) / H)
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


def _scale_place(t):
    """Where in a page's row of V scales token t of the page is."""
    return t - t % 8 + 2 * (t % 4) + t % 8 // 4


def _plain_pages(s, table):
    """Every token of a table's pages: K and V fp32 [rows of the table, kv, pages * page, d]."""
    case = s["case"]
    P, d = case["page"], case["d"]
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    r = s["pages"][table].transpose(1, 2)                               # [B, kv, pages, bytes]
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


def _attend(q, k, v, visible, kv, change=None):
    """q [B,H,N,d], k, v fp32 [B,kv,keys,d], visible [B,N,keys] -> O of q's type, LSE."""
    N = q.shape[2]
    x = q.float().unflatten(1, (kv, -1)).flatten(2, 3)                                       # [B, kv, group * N, d]
    scores = torch.matmul(x, k.transpose(2, 3)).mul_(1.0 / math.sqrt(q.shape[3])).unflatten(2, (-1, N))
    if change is not None:
        scores = change(scores)
    scores.masked_fill_(~visible[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top.nan_to_num(neginf=0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul((p.div_(total.clamp(min=1e-30))).flatten(2, 3), v).unflatten(2, (-1, N)).flatten(1, 2)
    return out.to(q.dtype), (top + torch.log(total)).squeeze(-1).flatten(1, 2)


def _plain_paged(s):
    case = s["case"]
    kv, N = case["kv_heads"], case["N"]
    k, v = _plain_pages(s, s["table"])
    key = torch.arange(k.shape[2], device="cuda", dtype=torch.int32)
    t = torch.arange(N, device="cuda", dtype=torch.int32)
    position = s["start"][:, None] + t                                                       # [B, N]
    there = t < (N if s["count"] is None else s["count"][:, None])                            # [B or 1, N]
    last = position + 1 if s["last"] is None else s["last"]
    last = torch.minimum(last, s["start"][:, None] + (N if s["count"] is None else s["count"][:, None]))
    visible = (key < last[..., None]) & there.expand(case["B"], N)[..., None]
    if s["first"] is not None:
        visible &= key >= s["first"][..., None]

    def change(scores):
        if case["cap"]:
            scores = scores.mul_(1.0 / case["cap"]).tanh_().mul_(case["cap"])
        if s["slopes"] is not None:
            distance = (position[..., None] - key).abs().float()[:, None, None]
            scores = scores.sub_(s["slopes"].view(1, kv, -1, 1, 1) * distance)
        return scores

    return _attend(s["q"], k, v, visible, kv, change)


def _plain_shared(s):
    case = s["case"]
    N = case["N"]
    kp, vp = _plain_pages(s, s["prefix_table"])
    k, v = _plain_pages(s, s["table"])
    member = torch.arange(case["B"], device="cuda")
    group = (member[:, None] >= s["group_start"][None, 1:]).sum(1)                            # of each sequence
    prefix, key = torch.arange(kp.shape[2], device="cuda"), torch.arange(k.shape[2], device="cuda")
    drafted = key - s["start"].long()[:, None]                                               # [B, keys]
    bit = (s["bits"][:, :, None] >> drafted.clamp(0, N - 1)[:, None]) & 1
    visible = (drafted < 0)[:, None] | ((drafted < N)[:, None] & (bit == 1))
    before = (prefix < s["prefix_length"][group][:, None])[:, None].expand(-1, N, -1)
    return _attend(s["q"], torch.cat((kp[group], k), 2), torch.cat((vp[group], v), 2), torch.cat((before, visible), 2), case["kv_heads"])


def _plain_assign(s):
    case = s["case"]
    P, N, table = case["page"], case["N"], s["table"]
    has = (s["start"] + P - 1) // P
    new = ((s["start"] + s["count"] + P - 1) // P).clamp(max=table.shape[1]).sub(has).clamp(min=0)
    before = new.cumsum(0) - new
    k = torch.arange(table.shape[1], device="cuda")[None] - has[:, None]                      # which of the new ones
    left = s["free_count"]
    place = left - 1 - (before[:, None] + k)
    taken = torch.where(place >= 0, s["free"][place.clamp(0, s["free"].numel() - 1)], -1)
    table.copy_(torch.where((k >= 0) & (k < new[:, None]), taken, table))
    left.copy_((left - new.sum()).clamp(min=0))
    n = torch.arange(N, device="cuda", dtype=torch.int32)
    positions = s["start"][:, None] + n
    page = table.gather(1, (positions // P).clamp(max=table.shape[1] - 1).long()).long()
    slots = page * P + positions % P
    fine = (n < s["count"][:, None]) & (page >= 0) & (positions < P * table.shape[1])
    return torch.where(fine, slots, -1), positions


def _plain_release(s, length, keep):
    case = s["case"]
    P, table = case["page"], s["table"]
    i = torch.arange(table.shape[1], device="cuda")[None]
    gone = (i >= ((keep + P - 1) // P)[:, None]) & (i < ((length + P - 1) // P)[:, None]) & (table >= 0)
    pages = table[gone]
    at = (s["free_count"] + pages.numel() - 1 - torch.arange(pages.numel(), device="cuda")).long()
    s["free"][at] = pages                               # the last page of the last sequence first
    table[gone] = -1
    s["free_count"] += pages.numel()


def run(state):
    s, case = state, state["case"]
    if not own:
        if case["op"] == "pages":
            slots, positions = _plain_assign(s)
            _plain_release(s, s["start"] + s["count"], s["start"])
            return slots, positions, s["table"], s["free"], s["free_count"]
        return {"paged": _plain_paged, "shared": _plain_shared}[case["op"]](s)
    from paper_2609_04105_b200 import binding as fp4
    if case["op"] == "pages":
        if "pool" not in s:             # a program makes it once
            s["pool"] = fp4.PagePool(s["free"], s["free_count"], case["page"])
        # tokens that come, and go again because they were turned down
        slots, positions = fp4.fp4attn_pages_assign(s["pool"], s["table"], s["start"], s["count"], N=case["N"])
        fp4.fp4attn_pages_release(s["pool"], s["table"], s["start"] + s["count"], keep=s["start"])
        return slots, positions, s["table"], s["free"], s["free_count"]
    if "cache" not in s:
        fmt = fp4.FMT_NVFP4 if case["fmt"] == "nvfp4" else fp4.FMT_E4M3
        s["cache"] = fp4.QuantizedCache(s["pages"], s["k_G"], s["v_G"], fmt, case["page"], case["d"])
    if case["op"] == "shared":
        return fp4.fp4attn_shared_prefix_attention(s["q"], s["cache"], s["prefix_table"], s["prefix_length"], s["group_start"],
                                                   s["table"], s["start"], tree_mask=s["bits"])
    return fp4.fp4attn_paged_attention(s["q"], s["cache"], s["table"], s["start"], count=s["count"], first=s["first"], last=s["last"],
                                       soft_cap=case["cap"], slopes=s["slopes"])


def work(case):
    B, N = case["B"], case["N"]
    if case["op"] == "pages":
        P = case["page"]
        new = sum(-(-(x + n) // P) - -(-x // P) for x, n in zip(_starts(case), _counts(case)))
        # starts and counts in; a slot and a position per token out; a new page: off the stack, into the table, out of it, onto the stack
        return {"bytes": 8.0 * B + 12.0 * B * N + 20.0 * new, "flops": 0.0}
    H, kv, d = case["H"], case["kv_heads"], case["d"]
    held = 9 / 16 if case["fmt"] == "nvfp4" else 1.0       # bytes of a kept element
    rows = B * H * N * (4.0 * d + 4)
    if case["op"] == "shared":
        bounds, prefixes = _members(case), _prefixes(case)
        keys = sum(prefixes) + sum(_starts(case)) + B * N
        seen = sum(p * (e - b) for p, b, e in zip(prefixes, bounds, bounds[1:])) * N + sum(_starts(case)) * N
        seen += sum(bin(x).count("1") for bits in _tree_bits(case) for x in bits)
        return {"bytes": 2 * keys * kv * d * held + rows, "flops": 4.0 * seen * H * d}
    keys = seen = 0
    for first, last, start, n in zip(*_seen(case), _starts(case), _counts(case)):
        keys += start + n - min(first[:n])
        seen += sum(min(x, start + n) - f for f, x in zip(first[:n], last))
    return {"bytes": 2 * keys * kv * d * held + rows, "flops": 4.0 * seen * H * d}


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_sequence(s, row):
    """K and V float64 [kv, tokens, d] of one row of a table: byte by byte, from the places that the layout gives each element."""
    case = s["case"]
    P, d = case["page"], case["d"]
    size, (k_at, ks_at, v_at, vs_at) = _record(case)
    t, e = torch.arange(P, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    records = s["pages"][row.long()]                                     # [pages, kv, bytes]

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
    return [x.transpose(0, 1).flatten(1, 2) / G.double()[:, None, None] for x, G in ((k, s["k_G"]), (v, s["v_G"]))]


def exact(case, seed):
    if case["op"] == "pages":
        return None
    s = prepare(case, seed)
    B, N, H, kv = case["B"], case["N"], case["H"], case["kv_heads"]
    group = H // kv
    out = torch.zeros((B, H, N, case["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, N), -math.inf, dtype=torch.float64, device="cuda")
    starts = _starts(case)

    def one(b, h, n, k, v, see, far=None):
        """Head h of n tokens of sequence b over keys k, v [keys, d]; see [n, keys]; far: distances [n, keys]."""
        z = s["q"][b, h, :n].double() @ k.T / math.sqrt(case["d"])
        if case.get("cap"):
            z = case["cap"] * torch.tanh(z / case["cap"])
        if far is not None:
            z = z - s["slopes"][h].double() * far
        z = torch.where(see, z, -math.inf)
        lse[b, h, :n] = torch.logsumexp(z, -1)
        out[b, h, :n] = torch.softmax(z, -1) @ v

    if case["op"] == "shared":
        bounds, prefixes, bits = _members(case), _prefixes(case), _tree_bits(case)
        j = torch.arange(N, device="cuda")
        for g, length in enumerate(prefixes):
            kp, vp = (x[:, :length] for x in _exact_sequence(s, s["prefix_table"][g]))
            for b in range(bounds[g], bounds[g + 1]):
                k, v = (torch.cat((p, x[:, :starts[b] + N]), 1) for p, x in zip((kp, vp), _exact_sequence(s, s["table"][b])))
                see = torch.ones((N, length + starts[b] + N), dtype=torch.bool, device="cuda")
                see[:, length + starts[b]:] = (torch.tensor(bits[b], device="cuda")[:, None] >> j & 1) > 0
                for h in range(H):
                    one(b, h, N, k[h // group], v[h // group], see)
        return out, lse
    firsts, lasts = _seen(case)
    for b, n in enumerate(_counts(case)):
        keys = starts[b] + n
        k, v = (x[:, :keys] for x in _exact_sequence(s, s["table"][b]))
        at = torch.arange(keys, device="cuda")
        see = (at >= torch.tensor(firsts[b][:n], device="cuda")[:, None]) & (at < torch.tensor(lasts[b][:n], device="cuda")[:, None])
        far = (starts[b] + torch.arange(n, device="cuda")[:, None] - at).abs().double() if case["bias"] else None
        for h in range(H):
            one(b, h, n, k[h // group], v[h // group], see, far)
    return out, lse
