"""Inputs, runs and derived error bounds of the tests of embedding, row norm,
language-model loss and optimizer step.

U is float32's half step.  A sum of float32 values whose longest chain of
additions has k links is off by at most k U times the sum of magnitudes (to
first order; the factor 1.01 below covers the rest).
"""
import numpy as np
import torch

import paper_2607_20357_amd as svl
from oracle import learning as ol

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}   # half the smallest subnormal


def half(name):
    return torch.finfo(TYPES[name]).eps / 2


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(gen, shape, name="f32", std=1.0):
    return (torch.randn(shape, generator=gen, device=gen.device) * std).to(TYPES[name])


def gen_of(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def strided(t, extra=8):
    """The same values in rows that are further apart; what lies between is NaN."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def assert_within(got, want, bound, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} values out of bounds, worst "
                           f"{np.nanmax(np.where(bad, off / np.maximum(bound, 1e-300), 0)):.3g} times the bound, first at "
                           f"{np.argwhere(bad)[0]}: {got[tuple(np.argwhere(bad)[0])]} for {want[tuple(np.argwhere(bad)[0])]}")


# ------------------------------------------------------------------ norm
# a row's sum: up to 16 values of a thread, 6 steps in a wave, 16 waves; a product before
DEPTH = 16 + 6 + 16 + 2


def norm_bounds(x, gain, bias, layer, eps, y_type):
    """(bound of y, of z, relative bound of r)."""
    y, mean, r = ol.norm(x, gain, bias, layer, eps)
    dm = DEPTH * U * np.abs(x).mean(1, keepdims=True) * 1.01 if layer else np.zeros_like(mean)
    er = dm * r + (DEPTH / 2 + 6) * U          # of 1 / sqrt(mean square): the mean's error, half the sum's
    z = (x - mean) * r
    dz = np.abs(z) * (er + 3 * U) + r * dm + U * r * np.abs(mean)
    g = 1.0 if gain is None else np.abs(gain)
    dy = dz * g + U * (np.abs(z) * g + np.abs(y))
    return y, dy + half(y_type) * (np.abs(y) + dy) + TINY[y_type], dz, er


def norm_grad_bounds(x, gy, gain, layer, eps, x_type, dz, er):
    gx, gg, gb = ol.norm_grad(x, gy, gain, layer, eps)
    _, mean, r = ol.norm(x, layer=layer, eps=eps)
    z = (x - mean) * r
    h = gy if gain is None else gy * gain
    hz = np.abs((h * z).mean(1, keepdims=True))
    d_hz = DEPTH * U * np.abs(h * z).mean(1, keepdims=True) + (np.abs(h) * dz).mean(1, keepdims=True)
    d_h = DEPTH * U * np.abs(h).mean(1, keepdims=True) if layer else 0.0
    hm = np.abs(h.mean(1, keepdims=True)) if layer else 0.0
    d = r * (np.abs(z) * d_hz + dz * (hz + d_hz) + d_h + 6 * U * (np.abs(h) + np.abs(z) * hz + hm)) + (er + U) * np.abs(gx)
    d *= 1.01
    links = -(-len(x) // 512) + 8 + 64          # rows of a piece, pieces of a group, groups
    dgg = (np.abs(gy) * (dz + 2 * U * np.abs(z))).sum(0) + links * U * np.abs(gy * z).sum(0)
    dgb = links * U * np.abs(gy).sum(0)
    return (gx, d + half(x_type) * (np.abs(gx) + d) + TINY[x_type]), (gg, 1.01 * dgg), (gb, 1.01 * dgb)


# ------------------------------------------------------------------ loss
def loss_bounds(x, w, labels, weight, compute, ref):
    """Bounds of lse, loss, grad_x and grad_w of oracle result `ref`."""
    n, d = x.shape
    v = len(w)
    wt = np.ones(n) if weight is None else weight
    ds = d * 2 * U * (np.abs(x) @ np.abs(w).T)               # of a logit: d products, added in any order
    top = ds.max(1)
    s = x @ w.T
    b_lse = top + (64 + v / 8192) * U + 4 * U * np.abs(ref.lse)
    b_loss = b_lse + top + 2 * U * np.abs(ref.loss)
    far = np.where(ref.p > 0, np.abs(s - ref.lse[:, None]), 0.0)
    # the exponential's own error, its fp16 digits, then P's rounding (and fp16's smallest steps)
    rel = (ds + b_lse[:, None] + 8 * U * (far + 8)) + 2.0 ** -11
    most = np.abs(wt[(labels >= 0) & (labels < v)]).max(initial=0.0)
    dp = np.abs(wt)[:, None] * ref.p * rel * 1.01
    dp = dp + half(compute) * (np.abs(ref.ds) + dp) + (ref.p > 0) * most * 2.0 ** -37
    links = 2 * U * max(n, v)
    bx = dp @ np.abs(w) + links * (np.abs(ref.ds) @ np.abs(w))
    bw = dp.T @ np.abs(x) + links * (np.abs(ref.ds).T @ np.abs(x))
    bx = 1.01 * bx + half(compute) * (np.abs(ref.grad_x) + bx) + TINY[compute]
    bw = 1.01 * bw + half(compute) * (np.abs(ref.grad_w) + bw) + TINY[compute]
    return b_lse, b_loss, bx, bw


def run_loss(head, x, w, labels, weight=None, want_x=True, want_w=True, held=None, ws=None, stream=None):
    n = x.shape[0]
    loss = torch.full((n,), float("nan"), device="cuda")
    lse = torch.full((n,), float("nan"), device="cuda")
    gx = torch.full((n, x.shape[1]), float("nan"), dtype=x.dtype, device="cuda") if want_x else None
    gw = None
    if want_w:
        gw = held if held is not None else torch.full(w.shape, float("nan"), dtype=w.dtype, device="cuda")
    if ws is None:
        ws = svl.alloc_lm_loss_workspace(head, n, want_x, want_w)
        ws.fill_(255)                      # a workspace needs no state
    svl.svl_lm_loss(head, x, w, labels, loss, ws, lse=lse, row_weight=weight, grad_x=gx, grad_w=gw,
                    accumulate=held is not None, stream=stream)
    return loss, lse, gx, gw
