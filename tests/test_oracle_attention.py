"""The float64 oracle of the windowed attention and of the 4-bit cache: the
gradient against differences, the mask and the quantisation against their
definitions one value at a time."""
import numpy as np
import pytest

from oracle import attention as oa


@pytest.mark.parametrize("window,sinks,masked", [(0, 0, False), (3, 0, False), (1, 0, True), (2, 1, True)])
def test_gradient_is_the_difference_quotient(window, sinks, masked):
    rng = np.random.default_rng(window + 10 * sinks)
    n, m, A, H, d, scale = 5, 7, 4, 2, 6, 0.6
    q, k, v, g = (rng.standard_normal(s) for s in ((n, A, d), (m, H, d), (m, H, d), (n, A, d)))
    mask = (np.arange(m) % 3 != 0) if masked else None
    ok = oa.visible(np.arange(m - n, m), m, window, sinks, mask)
    if masked and window == 1:
        assert (~ok.any(1)).any()     # a row that sees nothing is among them
    got = oa.attention(q, k, v, ok, scale, g)
    f = lambda q, k, v: float((oa.attention(q, k, v, ok, scale)["out"] * g).sum())
    h = 1e-5
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for i in list(np.ndindex(x.shape))[::5]:
            x0 = x[i]
            x[i] = x0 + h
            up = f(q, k, v)
            x[i] = x0 - h
            dn = f(q, k, v)
            x[i] = x0
            # truncation h^2 times a third derivative of order 10, cancellation 1e-16 / h
            assert abs((up - dn) / (2 * h) - got[name][i]) < 1e-8, (name, i)


def test_visibility_one_pair_at_a_time():
    for window in (0, 1, 2, 5, 100):
        for sinks in (0, 1, 3):
            ok = oa.visible(np.arange(4, 12), 12, window, sinks)
            for r, p in enumerate(range(4, 12)):
                for j in range(12):
                    want = j <= p and (window == 0 or p - j < window or j < sinks)
                    assert ok[r, j] == want


@pytest.mark.parametrize("f16", [True, False])
def test_quantised_values_keep_their_bounds(f16):
    rng = np.random.default_rng(3)
    bits, low = (11, -14) if f16 else (8, -126)
    x = rng.standard_normal((40, 128)) * np.exp2(rng.integers(-10, 4, (40, 1)).astype(np.float64))
    m, e = np.frexp(x)
    x = np.ldexp(np.rint(m * 2.0 ** bits), e - bits)          # values of the type
    c, s, lo = oa.quantise(x, f16)
    y = oa.stands_for(c, s, lo)
    g = x.reshape(40, 2, 64)
    assert (y.reshape(g.shape).max(-1) <= g.max(-1)).all() and (y.reshape(g.shape).min(-1) >= g.min(-1)).all()
    # half a step, or what rounding the step down took off fifteen of them
    bound = np.maximum(s / 2, 15 * s * 2.0 ** (1 - bits))
    assert (np.abs(y - x).reshape(g.shape) <= bound[..., None]).all()
    assert ((c >= 0) & (c <= 15)).all()


def test_quantised_ties_and_flat_groups():
    x = np.zeros((3, 64))
    x[0, :4] = [0, 15, 0.5, 1.5]       # step 1: ties to even
    x[1] = -2.5
    x[2, 5] = np.nan
    c, s, lo = oa.quantise(x, True)
    assert list(c[0, :4]) == [0, 15, 0, 2] and s[0, 0] == 1
    assert (c[1] == 0).all() and s[1, 0] == 0 and lo[1, 0] == -2.5
    assert np.isnan(s[2, 0]) and np.isnan(lo[2, 0]) and (c[2] == 0).all()


def test_tile_words_hold_every_nibble_once():
    for d in (64, 128):
        kc = np.arange(16 * d).reshape(16, d) % 16
        vc = (np.arange(16 * d).reshape(16, d) * 7 + 3) % 16
        w = oa.tile_words(kc, vc, d)
        n = np.array([(int(x) >> (4 * i)) & 15 for x in w for i in range(8)])
        assert len(n) == 2 * 16 * d
        assert np.array_equal(np.bincount(n[:16 * d], minlength=16), np.bincount(kc.ravel(), minlength=16))
        assert np.array_equal(np.bincount(n[16 * d:], minlength=16), np.bincount(vc.ravel(), minlength=16))
