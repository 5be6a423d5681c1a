"""Digits of the language-model loss where the float32 logits are known exactly, so
that nothing but the softmax itself is judged: large logits, sure rows, and rows whose
weights differ by decades."""
import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from learn_helpers import TYPES, f64, run_loss

pytestmark = pytest.mark.gpu
COMPUTES = ["bf16", "f16"]
D = 64


def _exact(compute, vocab, at, tops, labels):
    """Rows whose logits are tops[r] - gap[v]: at gives the gaps {entry: gap} of some entries, all others'
    is 1000.  tops[r] = (a, b): the product a b, of 16-bit values as all that is here; products and sums are
    whole multiples of what float32 resolves."""
    x, w = np.zeros((len(tops), D)), np.zeros((vocab, D))
    b = tops[0][1]
    w[:, 0], w[:, 1] = b, -1000.0
    for v, gap in at.items():
        w[v, 1] = -gap
    for r, (a, same) in enumerate(tops):
        assert same == b
        x[r, :2] = a, 1.0
    t = [torch.from_numpy(m).to(TYPES[compute]).cuda() for m in (x, w)]
    assert all(np.array_equal(f64(m), n) for m, n in zip(t, (x, w)))
    s = x @ w.T
    assert np.array_equal(s, s.astype(np.float32))
    return x, w, t[0], t[1], torch.tensor(labels, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("a, b", [(125.0, 80.0), (-125.0, 80.0), (1.5 * 2 ** 10, 2.0 ** 10), (3.0 * 2 ** 11, 2.0 ** 11),
                                  (3.0 * 2 ** 12, 2.0 ** 12), (-3.0 * 2 ** 12, 2.0 ** 12)])
@pytest.mark.parametrize("vocab, rows", [(300, 3), (33000, 200)])
def test_large_logits_of_one_entry(compute, a, b, vocab, rows):
    """One entry has all the probability, whatever its logit's size: P is 0 or +-1 exactly, and so is what the
    gradients add up.  (Both sizes of tiles.)"""
    top, other = 137, vocab - 2
    labels = [top if r % 2 else other for r in range(rows)]
    x, w, tx, tw, tl = _exact(compute, vocab, {top: 0.0}, [(a, b)] * rows, labels)
    loss, lse, gx, gw = run_loss(svl.make_lm_head(D, vocab, compute), tx, tw, tl)
    away = np.array([l == other for l in labels])
    assert np.array_equal(f64(lse), np.full(rows, a * b))
    assert np.array_equal(f64(loss), np.where(away, 1000.0, 0.0))
    want = np.where(away[:, None], w[top] - w[other], 0.0)
    assert np.array_equal(f64(gx), want)
    want = np.zeros((vocab, D))
    want[top] = x[away].sum(0)
    want[other] = -want[top]
    assert np.array_equal(f64(gw), f64(torch.from_numpy(want).to(TYPES[compute])))
