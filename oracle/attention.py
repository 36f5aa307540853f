"""Attention and the 4-bit rows of the paged cache in fp64, from their definitions.

``attend`` is the softmax-weighted mean itself, one query row and head at a time;
beside the result it returns what the error bounds of the tests are made of.
``quantise`` and ``dequantise`` are the row format's arithmetic; ``pack_page`` and
``unpack_page`` its byte order, one nibble at a time.
"""

from __future__ import annotations

import numpy as np

GROUP = 32


def attend(q, k, v, scale, causal=True, seen=None):
    """q [n, H_q, d], k and v [t, H, d] -> dict of out [n, H_q, d], lse [n, H_q],
    mag [n, H_q, d] (the weighted mean of |v|) and arg [n, H_q] (the largest
    scale * sum |q_e k_e| of a key that the row sees).  Row i sees key j <= i + t - n
    (causal), of those the ones that `seen` [t] names."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, Hq, d = q.shape
    t, H = k.shape[0], k.shape[1]
    G = Hq // H
    r = dict(out=np.zeros((n, Hq, d)), lse=np.full((n, Hq), -np.inf), mag=np.zeros((n, Hq, d)),
             arg=np.zeros((n, Hq)), weights={})
    for i in range(n):
        ok = np.ones(t, bool) if seen is None else np.array(seen, bool)
        if causal:
            ok = ok & (np.arange(t) <= i + t - n)
        js = np.nonzero(ok)[0]
        if js.size == 0:
            continue
        for h in range(Hq):
            with np.errstate(invalid="ignore", over="ignore"):
                kk, vv = k[js, h // G], v[js, h // G]
                s = scale * (kk @ q[i, h])
                m = s.max()
                w = np.exp(s - m)
                r["lse"][i, h] = m + np.log(w.sum())
                w = w / w.sum()
                r["out"][i, h] = w @ vv
                r["mag"][i, h] = w @ np.abs(vv)
                r["arg"][i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
            r["weights"][i, h] = (js, w)
    return r


def _bf16(x):
    """fp64 -> fp32 -> bf16, to nearest even; as fp32."""
    u = np.asarray(x, np.float32).view(np.uint32)
    up = ((u >> 16) & 1) + 0x7fff
    with np.errstate(over="ignore"):
        r = ((u + up) & 0xffff0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(np.asarray(x, np.float32)), np.float32(np.nan), r)


def quantise(x):
    """x [..., d] (fp32 values) -> codes [..., d] int, s and o [..., d/32] fp32."""
    x = np.asarray(x, np.float32)
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    with np.errstate(invalid="ignore", over="ignore"):
        lo, hi = g.min(-1), g.max(-1)   # (NaN where a value is)
        o = _bf16(lo)
        s = _bf16((hi - lo) / np.float32(15))
        bad = ~(np.isfinite(s) & np.isfinite(o))
        s = np.where(s < 2.0 ** -100, np.float32(0), s).astype(np.float32)
        # in 64 bits: the quotients of fp32 numbers that lie halfway between codes are exact there
        c = np.rint((g - o[..., None]).astype(np.float64) / np.where(s > 0, s, np.inf)[..., None])
    c = np.where(bad[..., None], 0, np.clip(np.nan_to_num(c), 0, 15)).astype(np.int64)
    s, o = (np.where(bad, np.float32(np.nan), y).astype(np.float32) for y in (s, o))
    return c.reshape(x.shape), s, o


def dequantise(c, s, o):
    g = np.asarray(c, np.float64).reshape(c.shape[:-1] + (c.shape[-1] // GROUP, GROUP))
    return (g * np.asarray(s, np.float64)[..., None] + np.asarray(o, np.float64)[..., None]).reshape(c.shape)


def key_nibble(d, e):
    """Where channel e of a token's keys lies among its d nibbles."""
    g, m, j = e // 32, e % 32 // 8, e % 8
    return (m * (d // 32) + g) * 8 + j


def value_nibble(d, tok, e):
    """Where channel e of token tok of a block of 32 lies among its 32 d nibbles."""
    u, m, j = tok // 16, tok % 16 // 4, tok % 4
    n, c = e // 16, e % 16
    return ((m * 16 + c) * (d // 16) + n) * 8 + 4 * u + j


def page_bytes(H, d, P):
    return H * P * (d + d // 4)


def unpack_page(page, H, d, P):
    """bytes of one page -> dict of codes [role][P, H, d] and words s, o [role][P, H, d/32]."""
    page = np.asarray(page, np.uint8).reshape(H, -1)
    G = d // 32
    nib = np.stack([page & 15, page >> 4], axis=-1).reshape(H, -1).astype(np.int64)
    c = np.zeros((2, P, H, d), np.int64)
    e = np.arange(d)
    kn = key_nibble(d, e)
    for t in range(P):
        c[0, t] = nib[:, t * d + kn]
        c[1, t] = nib[:, P * d + (t // 32) * 32 * d + value_nibble(d, t % 32, e)]
    w = np.ascontiguousarray(page[:, P * d:]).view(np.uint32).reshape(H, 2, P, G).transpose(1, 2, 0, 3)
    s = (w & np.uint32(0xffff0000)).view(np.float32)
    o = (w << np.uint32(16)).astype(np.uint32).view(np.float32)
    return c, s, o


def pack_page(c, s, o, H, d, P):
    """The inverse of unpack_page."""
    nib = np.zeros((H, 2 * P * d), np.uint8)
    e = np.arange(d)
    kn = key_nibble(d, e)
    for t in range(P):
        nib[:, t * d + kn] = c[0, t]
        nib[:, P * d + (t // 32) * 32 * d + value_nibble(d, t % 32, e)] = c[1, t]
    codes = nib[:, 0::2] | (nib[:, 1::2] << 4)
    w = np.asarray(s, np.float32).view(np.uint32) & np.uint32(0xffff0000)
    w = w | (np.asarray(o, np.float32).view(np.uint32) >> np.uint32(16))
    w = np.ascontiguousarray(w.transpose(2, 0, 1, 3)).reshape(H, -1).view(np.uint8).reshape(H, -1)
    return np.concatenate([codes, w], axis=1).reshape(-1)
