"""Windowed attention and the 4-bit K / V cache in float64, from their
definitions (include/svl.h): one sample at a time, whole score matrices."""
from __future__ import annotations

import numpy as np

GROUP, TILE = 64, 16


def visible(pos, n_keys, window, sinks, key_mask=None):
    """[rows][keys]: whether the query at each position sees each key."""
    p, j = np.asarray(pos)[:, None], np.arange(n_keys)[None, :]
    ok = j <= p
    if window > 0:
        ok &= (j > p - window) | (j < sinks)
    if key_mask is not None:
        ok &= np.asarray(key_mask, bool)[None, :]
    return ok


def attention(q, k, v, ok, scale, grad=None):
    """q [n][A][d], k and v [m][KV][d], ok [n][m] -> dict of out [n][A][d], lse [n][A], p
    [A][n][m] and, with grad (of out), dq, dk, dv and ds [A][n][m]."""
    n, A, d = q.shape
    m, H = k.shape[:2]
    rep = A // H
    kh = np.repeat(k, rep, axis=1).transpose(1, 2, 0)          # [A][d][m]
    vh = np.repeat(v, rep, axis=1).transpose(1, 0, 2)          # [A][m][d]
    qh = q.transpose(1, 0, 2)
    s = np.where(ok[None], qh @ kh * scale, -np.inf)
    top = np.max(s, axis=-1, keepdims=True, initial=-np.inf)
    e = np.where(ok[None], np.exp(s - np.where(np.isneginf(top), 0.0, top)), 0.0)
    total = e.sum(-1, keepdims=True)
    p = e / np.where(total > 0, total, 1.0)
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(total), -np.inf)[..., 0]
    out = {"p": p, "lse": lse.T, "out": (p @ vh).transpose(1, 0, 2)}
    if grad is not None:
        g = grad.transpose(1, 0, 2)
        dp = g @ vh.transpose(0, 2, 1)
        ds = p * (dp - (g * (p @ vh)).sum(-1, keepdims=True))
        out["dp"], out["ds"] = dp, ds
        out["dq"] = (ds @ kh.transpose(0, 2, 1)).transpose(1, 0, 2) * scale
        dk, dv = ds.transpose(0, 2, 1) @ qh * scale, p.transpose(0, 2, 1) @ g
        out["dk"] = dk.reshape(H, rep, m, d).sum(1).transpose(1, 0, 2)
        out["dv"] = dv.reshape(H, rep, m, d).sum(1).transpose(1, 0, 2)
    return out


def _round_down(x, bits, low):
    """x >= 0 cut to `bits` significant bits (below 2^low: to the unit there)."""
    m, e = np.frexp(x)
    unit = np.ldexp(1.0, np.maximum(e, low + 1) - bits)
    return np.floor(x / unit) * unit


def quantise(x, f16):
    """Rows [..., d] of fp16 (or bf16) values -> codes [..., d], scales and minima
    [..., d / 64]; a group with an inf or NaN: codes 0, scale and minimum NaN."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    lo = g.min(-1)
    s = _round_down((g.max(-1) - lo) / 15.0, 11 if f16 else 8, -14 if f16 else -126)
    flat = s == 0
    c = np.rint((g - lo[..., None]) / np.where(flat, 1.0, s)[..., None])     # ties to even
    c = np.where(flat[..., None], 0.0, np.clip(c, 0, 15)).astype(np.int64)
    s, lo = np.where(bad, np.nan, s), np.where(bad, np.nan, lo)
    return c.reshape(x.shape), s, lo


def stands_for(codes, s, lo):
    return np.repeat(lo, GROUP, -1) + np.repeat(s, GROUP, -1) * codes


def tile_words(kc, vc, d):
    """K and V codes [16][d] of one tile -> its code words, as uint32."""
    G = d // GROUP
    k = np.zeros((TILE, d // 8), np.uint32)
    v = np.zeros((4, 16, G, 2), np.uint32)
    for p in range(TILE):
        for x in range(d):
            w, i = x // 8, x % 8
            k[p, (w % 4) * (d // 32) + w // 4] |= np.uint32(int(kc[p, x]) << (4 * i))
            g, lane, t, odd = x // GROUP, x % GROUP // 4, x % 4 // 2, x % 2
            i = 2 * odd + p % 4 // 2 + 4 * (p % 2)
            v[p // 4, lane, g, t] |= np.uint32(int(vc[p, x]) << (4 * i))
    return np.concatenate([k.reshape(-1), v.reshape(-1)])
