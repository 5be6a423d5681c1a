"""The windowed attention over packed rows and its backward, against the float64
oracle within the bounds of their roundings (attention_helpers)."""
import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from attention_helpers import check_window, draw, dtype_of, f64, half_step, offsets, run_window
from oracle import attention as oa

pytestmark = pytest.mark.gpu
COMPUTES = ["f16", "bf16"]


def _inputs(heads, compute, nq, nk, seed, spread=1.0, masked=False):
    A, H, d = heads
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cu_q, cu_k = offsets(nq), offsets(nk)
    q = draw(gen, (int(cu_q[-1]), A, d), compute)
    k = draw(gen, (int(cu_k[-1]), H, d), compute)
    v = draw(gen, (int(cu_k[-1]), H, d), compute)
    grad = draw(gen, q.shape, compute, spread)
    mask = (torch.rand(int(cu_k[-1]), generator=gen, device="cuda") > 0.3).to(torch.uint8) if masked else None
    return cu_q, cu_k, q, k, v, grad, mask


def _check(heads, compute, nq, nk, window, sinks, seed=0, spread=1.0, masked=False):
    att = svl.make_attention(*heads, window=window, sinks=sinks, compute=compute)
    cu_q, cu_k, q, k, v, grad, mask = _inputs(heads, compute, nq, nk, seed, spread, masked)
    got = run_window(att, cu_q, cu_k, q, k, v, mask, grad)
    torch.cuda.synchronize()
    check_window(att, compute, cu_q, cu_k, q, k, v, got, mask, grad)
    return att, cu_q, cu_k, q, k, v, grad, mask, got


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("heads", [(4, 4, 128), (4, 4, 64), (7, 1, 128), (8, 2, 64), (8, 8, 128)])
def test_ragged_causal(heads, compute):
    n = [1, 2, 33, 0, 64, 65, 131, 200]
    _check(heads, compute, n, n, 0, 0, seed=heads[0])


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 2), (32, 0), (64, 64), (100, 7), (130, 200), (9999, 5)])
def test_windows_and_sinks(window, sinks, compute):
    n = [300, 129, 7]
    _check((4, 2, 128), compute, n, n, window, sinks, seed=window)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_queries_behind_earlier_keys(window, sinks, compute):
    """A chunk of a prompt: the queries are the last rows of longer keys; samples without queries."""
    _check((4, 2, 64), compute, [1, 100, 0, 37, 64], [300, 150, 40, 37, 65], window, sinks, seed=3)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (50, 4)])
def test_key_mask_and_rows_that_see_nothing(window, sinks, compute):
    att, cu_q, cu_k, q, k, v, grad, mask, got = _check((4, 2, 128), compute, [150, 70], [150, 90], window, sinks,
                                                       seed=5, masked=True)
    if window == 3:
        assert torch.isneginf(got[1]).any()
    # what a hidden row holds does not matter
    hidden = mask == 0
    k2, v2 = k.clone(), v.clone()
    k2[hidden], v2[hidden] = float("nan"), float("inf")
    again = run_window(att, cu_q, cu_k, q, k2, v2, mask, grad)
    for x, y in zip(got, again):
        assert torch.equal(x, y)
    # a mask of truth values is the same mask
    assert torch.equal(run_window(att, cu_q, cu_k, q, k, v, mask.bool())[0], got[0])


def test_everything_hidden():
    att = svl.make_attention(2, 1, 64)
    cu, _, q, k, v, grad, _ = _inputs((2, 1, 64), "f16", [70], [70], 1)
    out, lse, dq, dk, dv = run_window(att, cu, None, q, k, v, torch.zeros(70, dtype=torch.uint8, device="cuda"), grad)
    assert torch.isneginf(lse).all()
    for x in (out, dq, dk, dv):
        assert (x == 0).all()


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("n,heads,window,sinks", [([700], (2, 1, 128), 0, 0), ([900, 400], (4, 2, 64), 64, 10)])
def test_long_rows_in_pieces(n, heads, window, sinks, compute):
    """Key tiles cut into pieces that are joined, and 128-row tiles of queries."""
    _check(heads, compute, n, n, window, sinks, seed=2)


def test_many_heads_take_the_taller_tiles():
    _check((32, 32, 64), "bf16", [260, 129, 385, 520, 130, 257], [260, 129, 385, 520, 130, 257], 0, 0, seed=12)


def test_a_batch_of_more_than_one_launch():
    rng = np.random.default_rng(0)
    n = [int(x) for x in rng.integers(0, 60, 140)]
    _check((2, 2, 64), "f16", n, n, 17, 2, seed=6)


@pytest.mark.parametrize("compute,spread", [("f16", 1e-5), ("f16", 3e3), ("bf16", 1e-12), ("bf16", 1e10)])
def test_gradients_of_other_sizes(compute, spread):
    """Unscaled small gradients and large scaled ones keep their digits."""
    _check((4, 2, 128), compute, [130, 40], [130, 40], 50, 2, seed=7, spread=spread)


@pytest.mark.parametrize("compute", COMPUTES)
def test_packed_projections_and_rows_outside(compute):
    """Q, K and V as slices of one array, offsets that do not start at 0, outputs with gaps."""
    A, H, d, n = 4, 2, 64, 100
    att = svl.make_attention(A, H, d, window=30, sinks=1, compute=compute)
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = draw(gen, (n, A + 2 * H, d), compute)
    q, k, v = qkv[:, :A], qkv[:, A:A + H], qkv[:, A + H:]
    cu = np.array([3, 50, 50, 97], np.int32)
    g = draw(gen, (n, A, d), compute)
    out = torch.full((n, A + 1, d), 7.0, dtype=q.dtype, device="cuda")[:, :A]
    lse = torch.full((n, A), 7.0, device="cuda")
    grads = torch.full((n, A + 2 * H, d), 7.0, dtype=q.dtype, device="cuda")
    dq, dk, dv = grads[:, :A], grads[:, A:A + H], grads[:, A + H:]
    ws = svl.alloc_window_workspace(att, cu)
    svl.svl_window_attention(att, cu, None, q, k, v, out, lse=lse)
    svl.svl_window_attention_backward(att, cu, None, q, k, v, out, lse, g, dq, dk, dv, ws)
    torch.cuda.synchronize()
    check_window(att, compute, cu, cu, q, k, v, (out, lse, dq, dk, dv), None, g)
    for x in (out, lse, dq, dk, dv):
        assert (x[:3] == 7).all() and (x[97:] == 7).all()


@pytest.mark.parametrize("compute", COMPUTES)
def test_an_inf_stays_with_those_that_see_it(compute):
    """Rows and keys with an inf or NaN, and those that are masked from them."""
    heads, n = (2, 1, 128), 300
    att = svl.make_attention(*heads, window=40, sinks=2, compute=compute)
    cu, _, q, k, v, grad, _ = _inputs(heads, compute, [n], [n], 4)
    base = run_window(att, cu, None, q, k, v, None, grad)
    ok = oa.visible(np.arange(n), n, 40, 2)
    for name, at, value in (("v", 100, "inf"), ("k", 131, "nan"), ("grad", 200, "nan"), ("q", 77, "inf"), ("v", 250, "nan")):
        x = {"q": q.clone(), "k": k.clone(), "v": v.clone(), "grad": grad.clone()}
        x[name][at, 0, 5] = float(value)
        out, lse, dq, dk, dv = run_window(att, cu, None, x["q"], x["k"], x["v"], None, x["grad"])
        if name in "kv":
            rows = ok[:, at]                              # the queries that see it
            keys = ok[rows].any(0)                        # and the keys that those see
        else:
            rows = np.arange(n) == at
            keys = ok[at]
        heads_hit = [0, 1] if name in "kv" else [0]
        if name != "grad":
            assert torch.equal(out[~rows], base[0][~rows]), name
            assert (~np.isfinite(f64(out)[rows][:, heads_hit])).any(-1).all(), name
        assert torch.equal(dq[~rows], base[2][~rows]), name
        assert torch.equal(dk[~keys], base[3][~keys]) and torch.equal(dv[~keys], base[4][~keys]), name
        assert (~np.isfinite(f64(dq)[rows][:, heads_hit])).any(-1).all(), name
        assert (~np.isfinite(f64(dk)[keys])).any((1, 2)).all(), name


def test_same_bits_on_every_call_and_in_graphs():
    heads, n = (8, 2, 128), [500, 130]
    att = svl.make_attention(*heads, window=100, sinks=4, compute="bf16")
    cu, _, q, k, v, grad, _ = _inputs(heads, "bf16", n, n, 8)
    base = run_window(att, cu, None, q, k, v, None, grad)
    again = run_window(att, cu, None, q, k, v, None, grad)
    for x, y in zip(base, again):
        assert torch.equal(x, y)
    outs = [torch.empty_like(x) for x in base]
    ws = svl.alloc_window_workspace(att, cu)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        svl.svl_window_attention(att, cu, None, q, k, v, outs[0], lse=outs[1])
        svl.svl_window_attention_backward(att, cu, None, q, k, v, outs[0], outs[1], grad, *outs[2:], ws)
    for _ in range(3):
        for x in outs:
            x.fill_(5)
        g.replay()
        other = run_window(att, cu, None, q, k, v, None, grad)     # eager work between replays
        torch.cuda.synchronize()
        for x, y, z in zip(base, outs, other):
            assert torch.equal(x, y) and torch.equal(x, z)


def test_gradient_against_differences():
    """Along random directions: (L(x + e u) - L(x - e u)) / 2e of the kernel's own forward."""
    heads, n = (4, 2, 64), [90]
    att = svl.make_attention(*heads, window=30, sinks=2)
    cu, _, q, k, v, grad, _ = _inputs(heads, "f16", n, n, 9)
    _, _, dq, dk, dv = run_window(att, cu, None, q, k, v, None, grad)
    loss = lambda a, b, c: float((run_window(att, cu, None, a, b, c)[0].double() * grad.double()).sum())
    gen = torch.Generator(device="cuda").manual_seed(3)
    for i, (x, g) in enumerate(((q, dq), (k, dk), (v, dv))):
        u = torch.randn(x.shape, generator=gen, device="cuda").half()
        e = 0.25 if i == 2 else 0.03125
        args = [[q, k, v], [q, k, v]]
        args[0][i], args[1][i] = (x + e * u), (x - e * u)
        got = (loss(*args[0]) - loss(*args[1])) / float(2 * e)
        step = (args[0][i].double() - args[1][i].double()) / (2 * e)      # what was moved, after rounding
        want = float((g.double() * step).sum())
        # outputs of about 1 rounded at 2^-11 (random, over the root of their number), the
        # third derivative e^2 / 6 of a sum of about |u| sized terms
        size = float((grad.double() ** 2).sum() ** 0.5)
        tol = size * (2.0 ** -11 / e + 4 * e * e * (0 if i == 2 else 1)) + 2.0 ** -10 * abs(want)
        assert abs(got - want) <= tol, (i, got, want, tol)


@pytest.mark.parametrize("compute", COMPUTES)
def test_key_gradient_under_large_outputs(compute):
    """Values near 100, so that the output's rounding is large beside the differences that
    the gradient is made of: it must not reach the key gradient."""
    heads, n, d = (2, 1, 64), 150, 64
    att = svl.make_attention(*heads, window=60, sinks=2, compute=compute)
    gen = torch.Generator(device="cuda").manual_seed(11)
    q, k, grad = (draw(gen, (n, h, d), compute) for h in (2, 1, 2))
    v = (100 + torch.randn((n, 1, d), generator=gen, device="cuda")).to(dtype_of(compute))
    cu = np.array([0, n], np.int32)
    dk = run_window(att, cu, None, q, k, v, None, grad)[3]
    w = oa.attention(f64(q), f64(k), f64(v), oa.visible(np.arange(n), n, 60, 2), d ** -0.5, f64(grad))
    # dS is rounded once as an operand and dK once as the result.  What float32 leaves of D
    # is some 2^-18 of the terms of the products grad . v, in every dS by its P
    h, aq = half_step(compute), np.abs(f64(q)).transpose(1, 0, 2)                  # [A][n][d]
    terms = (np.abs(f64(grad)) * np.abs(f64(v))).sum(-1).max(0)                    # [A]
    each = h * np.abs(w["ds"]) + 2.0 ** -18 * terms[:, None, None] * w["p"]        # [A][n][m]
    bound = 1.01 * ((each.transpose(0, 2, 1) @ aq).sum(0)[:, None] * d ** -0.5 + h * np.abs(w["dk"]))
    err = np.abs(f64(dk) - w["dk"])
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("compute", COMPUTES)
def test_the_largest_window_is_no_window(compute):
    """window and sinks at the largest integer: the causal range, bit for bit."""
    heads, n = (2, 1, 64), [150, 70]
    cu, _, q, k, v, grad, _ = _inputs(heads, compute, n, n, 12)
    most = 2 ** 31 - 1
    base = run_window(svl.make_attention(*heads, compute=compute), cu, None, q, k, v, None, grad)
    for window, sinks in ((most, 0), (most, most), (2 ** 30, 1), (5, most)):
        att = svl.make_attention(*heads, window=window, sinks=sinks, compute=compute)
        for x, y in zip(base, run_window(att, cu, None, q, k, v, None, grad)):
            assert torch.equal(x, y), (window, sinks)
