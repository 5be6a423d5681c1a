"""Shared by the tests of the windowed attention and of the 4-bit cache: inputs,
the oracle sample by sample, and error bounds from the operators' roundings."""
import numpy as np
import torch

import paper_2607_20357_amd as svl
from oracle import attention as oa

U32 = 2.0 ** -24          # a float32 rounding


def dtype_of(compute):
    return torch.float16 if compute == "f16" else torch.bfloat16


def half_step(compute):
    return torch.finfo(dtype_of(compute)).eps / 2


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def draw(gen, shape, compute, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype_of(compute))


def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def score_error(q, k, scale):
    """How far a softmax weight may be off, relatively: the sums of a score (d products
    and the scaling, in float32), the maximum taken off and the power, with headroom of
    two roundings for each."""
    H, rep = k.shape[1], q.shape[1] // k.shape[1]
    top = max((float((np.abs(q[:, h]) @ np.abs(k[:, h // rep]).T).max()) for h in range(q.shape[1])
               if q.shape[0] and k.shape[0]), default=0.0) * scale
    return (q.shape[2] + 16) * U32 * top + 2.0 ** -20


def worst(err, bound):
    """Largest error over its bound."""
    return float(np.max(err / np.maximum(bound, 1e-300), initial=0.0))


# ---------------------------------------------------------------- forward, backward
def run_window(att, cu_q, cu_k, q, k, v, mask=None, grad=None, pad=0):
    """Device call(s); outputs start as NaN so that a row left out shows."""
    n = q.shape[0]
    out = torch.full_like(q, float("nan"))
    lse = torch.full((n, att.n_heads), float("nan"), device="cuda")
    svl.svl_window_attention(att, cu_q, cu_k, q, k, v, out, lse=lse, key_mask=mask)
    if grad is None:
        return out, lse
    dq, dk, dv = (torch.full_like(x, float("nan")) for x in (q, k, v))
    ws = svl.alloc_window_workspace(att, cu_q, cu_k)
    ws.fill_(0xff)
    svl.svl_window_attention_backward(att, cu_q, cu_k, q, k, v, out, lse, grad, dq, dk, dv, ws, key_mask=mask)
    return out, lse, dq, dk, dv


def check_window(att, compute, cu_q, cu_k, q, k, v, got, mask=None, grad=None):
    """Every sample of `got` against the oracle, within the bounds of the roundings."""
    u, scale = half_step(compute), att.scale
    rep = att.n_heads // att.n_kv_heads
    Q, K, V = f64(q), f64(k), f64(v)
    G = None if grad is None else f64(grad)
    M = None if mask is None else mask.cpu().numpy()
    got = [f64(x) for x in got]
    tiny = 2.0 ** -25 if compute == "f16" else 0.0      # half of fp16's smallest step
    ratios = {}
    for b in range(len(cu_q) - 1):
        rq, rk = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        if m == 0:
            continue
        ok = oa.visible(np.arange(m - n, m), m, att.window, att.sinks, None if M is None else M[rk])
        qs, ks, vs = Q[rq], K[rk], V[rk]
        ref = oa.attention(qs, ks, vs, ok, scale, None if G is None else G[rq])
        de = score_error(qs, ks, scale)
        p = ref["p"]
        av = np.repeat(np.abs(vs), rep, axis=1).transpose(1, 0, 2)
        pav = (p @ av).transpose(1, 0, 2)
        # P rounded once, its subnormals, the weights' own error, the output rounded once
        tol = u * (np.abs(ref["out"]) + pav) * (1 + 2 * u) + 3 * de * pav + tiny * (1 + m * np.abs(vs).max())
        res = {"out": worst(np.abs(got[0][rq] - ref["out"]), tol)}
        empty = ~ok.any(1)
        assert (got[0][rq][empty] == 0).all() and np.isneginf(got[1][rq][empty]).all()
        l = ref["lse"][~empty]
        res["lse"] = worst(np.abs(got[1][rq][~empty] - l), de + (m + 8) * U32 + 4 * U32 * np.abs(l))
        if G is not None:
            gs = G[rq]
            ag, ak, aq = np.abs(gs).transpose(1, 0, 2), np.repeat(np.abs(ks), rep, axis=1).transpose(1, 0, 2), \
                np.abs(qs).transpose(1, 0, 2)
            # weights from the kernel's log-sum: its error comes on top
            dw = de + (m + 8) * U32 + 4 * U32 * np.abs(np.where(empty[None], 0, ref["lse"].T)).max(initial=0.0)
            delta = (ag * (tol + u * np.abs(ref["out"])).transpose(1, 0, 2)).sum(-1, keepdims=True)
            sums = (att.head_dim + 8) * U32 * (ag @ av.transpose(0, 2, 1))
            es = p * (delta + sums) + (u * (1 + 2 * u) + 3 * dw) * np.abs(ref["ds"]) + 3 * dw * p * delta
            # fp16: dS is held with its row's (dk: the sample's) largest gradient in
            # [1, 2) at worst 2^-14 below what overflows: half a subnormal step
            sub = 2.0 ** -24 * np.abs(gs).max(initial=0.0) if compute == "f16" else 0.0
            big = np.abs(ref["dp"]).max(initial=0.0) / max(np.abs(gs).max(initial=0.0), 1e-300)
            sub *= max(1.0, big * 2.0 ** -9)
            es = es + np.where(ok[None], sub, 0.0)
            tq = scale * (es @ ak).transpose(1, 0, 2) + u * np.abs(ref["dq"]) + tiny
            fold = lambda x: x.reshape(att.n_kv_heads, rep, m, -1).sum(1).transpose(1, 0, 2)
            tk = scale * fold(es.transpose(0, 2, 1) @ aq) + u * np.abs(ref["dk"]) + tiny
            pe = p * (u * (1 + 2 * u) + 3 * dw) + np.where(ok[None], tiny, 0.0)
            tv = fold(pe.transpose(0, 2, 1) @ ag) + u * np.abs(ref["dv"]) + tiny
            n32 = n * rep * U32       # the sums over rows
            tk, tv = tk + n32 * scale * fold(np.abs(ref["ds"]).transpose(0, 2, 1) @ aq), \
                tv + n32 * fold(p.transpose(0, 2, 1) @ ag)
            for name, x, t, r in (("dq", got[2], tq, rq), ("dk", got[3], tk, rk), ("dv", got[4], tv, rk)):
                res[name] = worst(np.abs(x[r] - ref[name]), t)
        for key, val in res.items():
            ratios[key] = max(ratios.get(key, 0.0), val) if val == val else float("nan")
    print("  error / bound:", {k: round(x, 3) for k, x in ratios.items()}, flush=True)
    for name, x in ratios.items():
        assert x <= 1.0, (name, x)
    return ratios


# ---------------------------------------------------------------- the 4-bit cache
def cached_rows(k, v, compute):
    """(codes, scales, minima) of K and V rows and what they stand for, float64."""
    f16 = compute == "f16"
    a, b = oa.quantise(f64(k), f16), oa.quantise(f64(v), f16)
    return a, b, oa.stands_for(*a), oa.stands_for(*b)


def fill_cache(att, k, v, max_len, batch=None):
    """k, v [B][positions][KV][d] appended from position 0 into a cache of 0xff bytes."""
    B, P = k.shape[:2]
    cache = svl.alloc_kv4_cache(att, B, max_len)
    cache.fill_(0xff)
    cu = offsets([P] * B)
    svl.svl_kv4_append(att, cu, [0] * B, k.flatten(0, 1), v.flatten(0, 1), cache, max_len)
    return cache


def check_cached(att, compute, cu, pos, q, k, v, got):
    """got [rows][A][d] of svl_kv4_attention against the oracle on what the cache
    stands for; k, v [B][positions][KV][d] are the appended 16-bit rows."""
    u, rep = half_step(compute), att.n_heads // att.n_kv_heads
    Q, got = f64(q), f64(got)
    worst_ratio = 0.0
    for b in range(len(cu) - 1):
        n, m = cu[b + 1] - cu[b], pos[b] + cu[b + 1] - cu[b]
        if n == 0:
            continue
        (kc, ks, kl), (vc, vs, vl), kk, vv = cached_rows(k[b, :m], v[b, :m], compute)
        ok = oa.visible(np.arange(pos[b], m), m, att.window, att.sinks)
        qs = Q[cu[b]:cu[b + 1]]
        ref = oa.attention(qs, kk, vv, ok, att.scale)
        # a score is s (q . c) + lo sum(q): its terms are bounded by |q| (|lo| + 15 s)
        ak = np.repeat(np.abs(kl) + 15 * ks, oa.GROUP, -1)
        de = score_error(qs, ak, att.scale)
        r = lambda x: np.repeat(x, rep, axis=1).transpose(1, 0, 2)
        sv = r(np.repeat(vs, oa.GROUP, -1) * vc)
        psv = (ref["p"] @ sv).transpose(1, 0, 2)
        pav = (ref["p"] @ r(np.abs(vv))).transpose(1, 0, 2)
        # P s rounded to fp16 once (its subnormals: 15 codes times half a step, after the
        # factor of 4), the weights' own error on both terms, the sums, the output
        sub = 15 * 2.0 ** -25 / 4 * m if compute == "f16" else 15 * 2.0 ** -25 * 2.0 ** -13 * m * vs.max()
        big = (ref["p"] @ r(np.repeat(np.abs(vl), oa.GROUP, -1))).transpose(1, 0, 2) + psv
        tol = u * np.abs(ref["out"]) + 2.0 ** -11 * (1 + 2.0 ** -10) * psv + 3 * de * (big + pav) + \
            (m + 64) * U32 * big + sub + (2.0 ** -25 if compute == "f16" else 0.0)
        worst_ratio = max(worst_ratio, worst(np.abs(got[cu[b]:cu[b + 1]] - ref["out"]), tol))
        assert np.isfinite(got[cu[b]:cu[b + 1]]).all()
    print("  error / bound:", round(worst_ratio, 3), flush=True)
    assert worst_ratio <= 1.0
    return worst_ratio
