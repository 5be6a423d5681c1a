"""Embedding, row norm, language-model loss and AdamW step with their gradients,
plainly and in float64 (numpy), written from their definitions.

8-bit optimizer states are the exception: their codes depend on every bit of
float32 moments, so the moments are rounded where the definition rounds them.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np

WORD = np.uint64(0xFFFFFFFF)
LOW_M, LOW_V = -13, -29    # lowest exponents with all digits, under scale 1
BLOCK = 256


def embed(tokens, table, scale=1.0):
    """Rows of the table; zeros for a token outside it."""
    out = np.zeros((len(tokens), table.shape[1]))
    for r, t in enumerate(tokens):
        if 0 <= t < len(table):
            out[r] = scale * table[t]
    return out


def embed_grad(tokens, grad_rows, vocab, scale=1.0):
    """(gradient, sum of magnitudes, rows) of each table row."""
    g = np.zeros((vocab, grad_rows.shape[1]))
    size, count = np.zeros_like(g), np.zeros(vocab, dtype=np.int64)
    for r, t in enumerate(tokens):
        if 0 <= t < vocab:
            g[t] += scale * grad_rows[r]
            size[t] += abs(scale) * np.abs(grad_rows[r])
            count[t] += 1
    return g, size, count


def norm(x, gain=None, bias=None, layer=False, eps=1e-6):
    """(y, mean, r)"""
    mean = x.mean(1, keepdims=True) if layer else np.zeros((len(x), 1))
    r = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) * r
    if gain is not None:
        y = y * gain
    if bias is not None:
        y = y + bias
    return y, mean, r


def norm_grad(x, grad_y, gain=None, layer=False, eps=1e-6):
    """(grad_x, grad_gain, grad_bias)"""
    _, mean, r = norm(x, layer=layer, eps=eps)
    z = (x - mean) * r
    h = grad_y if gain is None else grad_y * gain
    gx = h - z * (h * z).mean(1, keepdims=True)
    if layer:
        gx = gx - h.mean(1, keepdims=True)
    return gx * r, (grad_y * z).sum(0), grad_y.sum(0)


class Loss(NamedTuple):
    loss: np.ndarray
    lse: np.ndarray
    p: np.ndarray        # softmax of the rows with a label, zeros elsewhere
    ds: np.ndarray       # gradient of sum(weight * loss) with respect to the logits
    grad_x: np.ndarray
    grad_w: np.ndarray


def lm_loss(x, w, labels, weight=None) -> Loss:
    n, v = len(x), len(w)
    loss, lse = np.zeros(n), np.zeros(n)
    p, ds = np.zeros((n, v)), np.zeros((n, v))
    gx, gw = np.zeros((n, x.shape[1])), np.zeros(w.shape)
    for r in range(n):
        if not 0 <= labels[r] < v:
            continue
        s = w @ x[r]
        top = s.max()
        e = np.exp(s - top)
        lse[r] = top + np.log(e.sum())
        loss[r] = lse[r] - s[labels[r]]
        p[r] = e / e.sum()
        ds[r] = p[r]
        ds[r, labels[r]] -= 1.0
        ds[r] *= 1.0 if weight is None else weight[r]
        gx[r] = ds[r] @ w
        gw += np.outer(ds[r], x[r])
    return Loss(loss, lse, p, ds, gx, gw)


def f32(x):
    return np.asarray(x, dtype=np.float32).astype(np.float64)


def moments(grad, m, v, beta1, beta2, grad_scale=1.0):
    """The moments after a step: float32 values, every product and sum rounded once."""
    b1, b2, r1, r2 = (f32(t) for t in (beta1, beta2, 1.0 - beta1, 1.0 - beta2))
    g = f32(grad * f32(grad_scale))
    return f32(f32(b1 * m) + f32(r1 * g)), f32(f32(b2 * v) + f32(f32(r2 * g) * g))


def adamw(param, m, v, step, lr, beta1, beta2, eps, decay):
    """The parameter after a step, from the moments after it."""
    rate = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return param - lr * decay * param - lr * rate, lr * rate


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & WORD
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x6A09E667)) & WORD
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0xBB67AE85)) & WORD
    return x ^ (x >> np.uint64(16))


def random_bits(n, seed, number, first=0):
    """(low, high) 16 bits for elements first .. first + n - 1 of tensor `number`."""
    i = np.arange(first, first + n, dtype=np.uint64)
    key = mix(np.uint64(seed) + np.uint64(0x9E3779B9) * np.uint64(number + 1)
              + np.uint64(0xBB67AE85) * (i >> np.uint64(32)))
    r = mix(((i & WORD) * np.uint64(0x9E3779B9) & WORD) + key)
    return (r & np.uint64(0xFFFF)).astype(np.int64), (r >> np.uint64(16)).astype(np.int64)


def code_value(code, low):
    """What magnitude codes stand for under scale 1."""
    e, f = code >> 3, code & 7
    return np.where(e > 0, (1 + f / 8.0) * 2.0 ** (np.maximum(e, 1) - 1 + low), f / 8.0 * 2.0 ** low)


def decode(code, scale, second):
    code = np.asarray(code).astype(np.int64)
    scale = np.repeat(np.asarray(scale, dtype=np.float64), BLOCK)[:len(code)]
    if second:
        return f32(f32(scale * code_value(code, LOW_V)) ** 2)
    return np.where(code > 127, -1.0, 1.0) * scale * code_value(code & 127, LOW_M)


def encode(x, bits, low, signed):
    """(codes, scales) of float32 values, by the neighbours' places and the random bits."""
    code = np.zeros(len(x), dtype=np.int64)
    scales = []
    grid = code_value(np.arange(128 if signed else 256), low)
    for a in range(0, len(x), BLOCK):
        size = np.abs(x[a:a + BLOCK])
        if not np.all(np.isfinite(size)):
            scales.append(np.nan)
            continue
        top = size.max()
        s = 0.0 if top == 0 else 2.0 ** max(np.frexp(top)[1] - 1, -90)
        scales.append(s)
        if s == 0:
            continue
        for i, y in enumerate(size / s):
            below = int(np.searchsorted(grid, y, side="right")) - 1
            place = np.floor((y - grid[below]) / (grid[below + 1] - grid[below]) * 2.0 ** 20)
            code[a + i] = below + (place + 16 * bits[a + i] >= 2 ** 20)
    if signed:
        code += 128 * (x < 0) * np.repeat(np.isfinite(scales) & (np.asarray(scales) != 0), BLOCK)[:len(x)]
    return code.astype(np.uint8), np.asarray(scales, dtype=np.float32)
