"""Pins of oracle.learning: gradients against central differences and torch's
float64 autograd, the moments and codes against their definition's properties."""
import numpy as np
import pytest
import torch

from oracle import learning as ol


def _diff(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        y = x.copy()
        y[i] += h
        up = f(y)
        y[i] -= 2 * h
        g[i] = (up - f(y)) / (2 * h)
    return g


def test_embed_gradient_is_the_lookups():
    rng = np.random.default_rng(0)
    tokens = np.array([3, 0, 3, -1, 7, 8, 3])
    table, up = rng.standard_normal((8, 5)), rng.standard_normal((7, 5))
    want = _diff(lambda t: (ol.embed(tokens, t, 1.5) * up).sum(), table)
    got, _, count = ol.embed_grad(tokens, up, 8, 1.5)
    assert np.allclose(got, want, atol=1e-8) and count.tolist() == [1, 0, 0, 3, 0, 0, 0, 1]
    assert np.array_equal(ol.embed(tokens, table)[3], np.zeros(5))


@pytest.mark.parametrize("layer", [False, True])
def test_norm_gradient(layer):
    rng = np.random.default_rng(1)
    x, up = rng.standard_normal((3, 6)) * 2 + 0.3, rng.standard_normal((3, 6))
    gain, bias = rng.standard_normal(6), rng.standard_normal(6)
    f = lambda x, g, b: (ol.norm(x, g, b, layer, 1e-3)[0] * up).sum()
    gx, gg, gb = ol.norm_grad(x, up, gain, layer, 1e-3)
    assert np.allclose(gx, _diff(lambda t: f(t, gain, bias), x), atol=1e-7)
    assert np.allclose(gg, _diff(lambda t: f(x, t, bias), gain), atol=1e-7)
    assert np.allclose(gb, _diff(lambda t: f(x, gain, t), bias), atol=1e-7)
    if layer:
        want = torch.nn.functional.layer_norm(torch.from_numpy(x), (6,), torch.from_numpy(gain),
                                              torch.from_numpy(bias), 1e-3).numpy()
        assert np.allclose(ol.norm(x, gain, bias, True, 1e-3)[0], want, atol=1e-12)


def test_loss_is_torchs_cross_entropy():
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((6, 4)), rng.standard_normal((9, 4))
    labels, weight = np.array([0, 8, 3, -100, 3, 9]), rng.random(6) + 0.5
    tx, tw = (torch.from_numpy(t).requires_grad_() for t in (x, w))
    tl = torch.from_numpy(np.where((labels < 0) | (labels > 8), -100, labels))
    loss = torch.nn.functional.cross_entropy(tx @ tw.T, tl, reduction="none", ignore_index=-100)
    (loss * torch.from_numpy(weight)).sum().backward()
    r = ol.lm_loss(x, w, labels, weight)
    assert np.allclose(r.loss, loss.detach().numpy(), atol=1e-12)
    assert np.allclose(r.grad_x, tx.grad.numpy(), atol=1e-12) and np.allclose(r.grad_w, tw.grad.numpy(), atol=1e-12)
    want = _diff(lambda t: (ol.lm_loss(t, w, labels).loss * weight).sum(), x)
    assert np.allclose(r.grad_x, want, atol=1e-7)


def test_adamw_is_torchs():
    rng = np.random.default_rng(3)
    p = torch.from_numpy(rng.standard_normal(50)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    mine, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        m, v = ol.moments(g, m, v, 0.9, 0.95)      # float32 moments beside float64 ones
        mine, _ = ol.adamw(mine, m, v, step, 1e-2, 0.9, 0.95, 1e-8, 0.1)
        assert np.abs(mine - p.detach().numpy()).max() < 1e-6


def test_codes_grow_with_their_values():
    for low, n in ((ol.LOW_M, 128), (ol.LOW_V, 256)):
        grid = ol.code_value(np.arange(n), low)
        assert grid[0] == 0 and np.all(np.diff(grid) > 0) and grid[-1] < 4 and 1.875 in grid and 2.0 in grid
        step = np.diff(grid)[8:] / grid[8:-1]
        assert np.all((step <= 1 / 8) & (step >= 1 / 15))


def test_codes_are_right_on_average():
    """10000 seeds: a value's mean code value is the value, within 5 deviations of the mean."""
    x = np.array([1.0, 0.77, -0.0301, 1.3e-3, 2.1e-5])
    for low, signed in ((ol.LOW_M, True), (ol.LOW_V, False)):
        vals = np.abs(x) if not signed else x
        seen = []
        for seed in range(2000):
            bits = ol.random_bits(5, seed, 3)[0 if signed else 1]
            c, s = ol.encode(vals, bits, low, signed)
            seen.append(ol.decode(c, s, not signed))
        seen = np.asarray(seen)
        if not signed:
            seen = np.sqrt(seen)
        dev = seen.std(0) / np.sqrt(len(seen)) + 1e-9
        assert np.all(np.abs(seen.mean(0) - vals) < 5 * dev)


def test_random_bits_are_even():
    low, high = ol.random_bits(100000, 7, 0)
    for b in (low, high):
        counts = np.bincount(b >> 8, minlength=256)
        assert abs(counts - 100000 / 256).max() < 6 * np.sqrt(100000 / 256)
    assert abs(np.corrcoef(low, high)[0, 1]) < 0.02
    other = ol.random_bits(100000, 8, 0)[0]
    assert abs(np.corrcoef(low, other)[0, 1]) < 0.02
    assert np.array_equal(ol.random_bits(8, 7, 2, first=(1 << 32) + 4)[0][:4], ol.random_bits(4, 7, 2, first=(1 << 32) + 4)[0])
