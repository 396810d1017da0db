"""Serving operators (oracle side, test infrastructure only): rotary positions, the bytes of a paged cache, attention of a tree
of tokens over it.  fp64 NumPy, element by element from the layout that include/fp4attn.h states; what the cache's formats define with
fp32 roundings is rounded so.  Pinned by tests/test_oracle_serving.py: closed forms, round trips, brute force."""
from __future__ import annotations

import numpy as np

from . import formats as F
from . import quantize as Qz


def rotary(x, positions, inv_freq, interleaved=False, transposed=False, factor=1.0):
    """x [B,H,N,d]; positions [B,N]; inv_freq float32 [pairs]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    f = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    pairs = f.size
    theta = np.asarray(positions, dtype=np.float64)[:, None, :, None] * f
    c, s = factor * np.cos(theta), factor * np.sin(theta)
    if transposed:
        s = -s
    i = np.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def encode(x, G, fmt):
    """x float [T,d] of one head -> (codes, scale bytes): E2M1 nibbles [T,d] and E4M3 bytes [T,d/16], or E4M3 bytes [T,d] and None."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), 0.0, x)
    G = np.float32(G)
    with np.errstate(over="ignore", invalid="ignore"):
        if fmt == "e4m3":
            return F.e4m3_encode((x.astype(np.float32) * G).astype(np.float64)), None
        blocks = x.astype(np.float32).reshape(x.shape[0], -1, 16)
        t = (np.abs(blocks).max(-1) * G).astype(np.float32) / np.float32(6.0)
        sb = F.e4m3_encode_unsigned(t.astype(np.float64))
        S = F.e4m3_decode(sb).astype(np.float32)
        r = np.where(S > 0, G / np.where(S > 0, S, np.float32(1)), np.float32(0)).astype(np.float32)
        v = np.where(r[..., None] > 0, blocks * r[..., None], np.float32(0)).astype(np.float32)
    return F.e2m1_encode(v.astype(np.float64)).reshape(x.shape), sb


def record_bytes(fmt, P, d):
    return 2 * P * (d // 2 + d // 16 if fmt == "nvfp4" else d)


def places(fmt, P, d):
    """Byte offsets in a record, by token and element (or block): K codes [P,d], K scales [P,d/16], V codes, V scales; and the shift of
    an element's code inside its byte."""
    t, e, b = np.arange(P)[:, None], np.arange(d)[None], np.arange(d // 16)[None]
    if fmt == "e4m3":
        return (e // 16 * P + t) * 16 + e % 16, None, P * d + (t // 16 * d + e) * 16 + t % 16, None, 0 * e
    codes, scales = P * d // 2, P * d // 16
    order = np.array([0, 4, 1, 5, 2, 6, 3, 7])
    place = np.empty(8, dtype=np.int64)
    place[order] = np.arange(8)
    return ((e // 32 * P + t) * 16 + e % 32 // 2, codes + t * (d // 16) + b, codes + scales + (t // 16 * (d // 2) + e // 2) * 16 + t % 16,
            2 * codes + scales + b * P + t // 8 * 8 + place[t % 8], 4 * (e % 2))


def write(pages, k, v, table, start, count, k_G, v_G, fmt, P):
    """pages u8 [num_pages,kv,record] in place; k, v float [B,kv,N,d].  True if every token had a page."""
    B, kv, N, d = k.shape
    kc, ks, vc, vs, shift = places(fmt, P, d)
    fine = True
    for b in range(B):
        for n in range(N if count is None else min(max(int(count[b]), 0), N)):
            pos = int(start[b]) + n
            page = int(table[b][pos // P]) if 0 <= pos < P * len(table[b]) else -1
            if not 0 <= page < len(pages):
                fine = False
                continue
            t = pos % P
            for h in range(kv):
                rec = pages[page, h]
                for x, G, at, scales_at in ((k, k_G[h], kc, ks), (v, v_G[h], vc, vs)):
                    codes, sb = encode(x[b, h, n][None], G, fmt)
                    if fmt == "e4m3":
                        rec[at[t]] = codes[0]
                    else:
                        rec[at[t][0::2]] = codes[0][0::2] | codes[0][1::2] << 4
                        rec[scales_at[t]] = sb[0]
    return fine


def values(pages, table_row, h, length, k_G, v_G, fmt, P, d):
    """K and V float64 [length,d] of a sequence, and which positions have a page."""
    kc, ks, vc, vs, shift = places(fmt, P, d)
    k, v, held = np.zeros((length, d)), np.zeros((length, d)), np.zeros(length, dtype=bool)
    for pos in range(length):
        page = int(table_row[pos // P]) if pos < P * len(table_row) else -1
        if not 0 <= page < len(pages):
            continue
        held[pos] = True
        rec, t = pages[page, h], pos % P
        if fmt == "e4m3":
            k[pos], v[pos] = F.e4m3_decode(rec[kc[t]]), F.e4m3_decode(rec[vc[t]])
        else:
            k[pos] = F.e2m1_decode(rec[kc[t]] >> shift[0] & 15) * np.repeat(F.e4m3_decode(rec[ks[t]]), 16)
            v[pos] = F.e2m1_decode(rec[vc[t]] >> shift[0] & 15) * np.repeat(F.e4m3_decode(rec[vs[t]]), 16)
    return k / np.float64(np.float32(k_G[h])), v / np.float64(np.float32(v_G[h])), held


def seen(context, T, bits, held):
    """Truth values [T, context + T]."""
    ctx = max(0, int(context))
    m = np.zeros((T, ctx + T), dtype=bool)
    m[:, :ctx] = True
    for t in range(T):
        for j in range(T):
            m[t, ctx + j] = (int(bits[t]) >> j & 1) if bits is not None else j <= t
    return m & held[None]


def attend(q, k, v, mask, scale):
    """q [T,d], k, v [n,d], mask [T,n] -> O, LSE, and per row what the tolerances of a test need: sum of p |v| [T,d], and the largest
    sum of |q k| * scale over the keys seen."""
    z = (q @ k.T) * scale
    z = np.where(mask, z, -np.inf)
    any_seen = mask.any(1)
    top = np.where(any_seen, z.max(1, initial=-np.inf), 0.0)
    p = np.exp(z - top[:, None])
    total = p.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(any_seen, top + np.log(total), -np.inf)
    p = p / np.where(any_seen, total, 1.0)[:, None]
    size = np.where(mask, (np.abs(q) @ np.abs(k).T) * scale, 0.0).max(1, initial=0.0)
    return p @ v, lse, p @ np.abs(v), size
