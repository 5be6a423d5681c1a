"""Digits of the language-model loss where the float32 logits are known exactly, so
that nothing but the softmax itself is judged: large logits, sure rows, and rows whose
weights differ by decades."""
import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from learn_helpers import (TINY, TYPES, U, assert_within, f64, gen_of, half, loss_bounds, randn, run_loss)
from oracle import learning as ol

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


def _sum_bound(s, top):
    """Relative error of a row's sum of exponentials under its largest logit.  Each exponential: its argument's
    difference, two products and a sum (3 U far + 14 U log 2), the exponential itself (2 U), and the slab's to the
    row's (far U + 4 U and a product).  Sums: at most as many inexact additions as there are entries beside the
    largest, and no more than 32 of a lane, 2 + 6 between lanes, and the slabs of a lane."""
    far = top - s
    p = np.exp(-far)
    others = (p > 2.0 ** -150).sum(1, keepdims=True) - 1
    p[far == 0] = 0.0
    return 1.01 * U * (np.minimum(others, 40 + s.shape[1] / 4096) + (p * (4 * far + 18)).sum(1, keepdims=True))


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("b", [1.0, 64.0])
@pytest.mark.parametrize("vocab, rows", [(3, 1), (700, 40), (33000, 200)])
def test_sure_rows_keep_their_small_losses(compute, b, vocab, rows):
    """A loss of 1e-6 beside logits of hundreds: its error is the sum's, not the log-sum's rounding, and P of the
    label balances P of the others."""
    top, near, last = 0, 1, vocab - 1
    at = {top: 0.0, near: 13.75, last: 9.25}
    tops = [((30.0, 200.0, -200.0, 2000.0, 0.0)[r % 5], b) for r in range(rows)]
    labels = [(top, top, top, near)[r // 5 % 4] for r in range(rows)]
    x, w, tx, tw, tl = _exact(compute, vocab, at, tops, labels)
    weight = np.full(rows, 1024.0)
    loss, lse, gx, _ = run_loss(svl.make_lm_head(D, vocab, compute), tx, tw, tl,
                                torch.from_numpy(weight).float().cuda(), want_w=False)
    ref = ol.lm_loss(x, w, labels, weight)
    s = x @ w.T
    most = s.max(1, keepdims=True)
    far, e = most - s, _sum_bound(s, most)
    log_sum = np.log(np.exp(-far).sum(1))
    away = far[np.arange(rows), labels]
    # the logarithm (2 U of itself), the label's distance and the sum of both
    b_loss = e[:, 0] + U * (2 * log_sum + away + 2 * (away + log_sum)) + U * 2 ** -20
    want = away + log_sum              # (as ref.loss, without float64's own cancellation)
    assert np.abs(want - ref.loss).max() < 1e-10
    assert_within(loss, want, b_loss, "loss")
    assert_within(lse, ref.lse, e[:, 0] + U * (2 * log_sum + 2 * np.abs(ref.lse)), "lse")
    # P: exponentials in fp16 digits but for the largest (2^14), their own errors, the sum's and its quotient's, then
    # P's rounding
    dp = ref.p * (e + 2 * U + (far > 0) * (2.0 ** -11 + U * (4 * far + 30))) * 1.01
    dp = weight[:, None] * dp
    dp = dp + half(compute) * (np.abs(ref.ds) + dp) + (ref.p > 0) * weight[:, None] * 2.0 ** -37
    bx = dp @ np.abs(w) + 6 * U * (np.abs(ref.ds) @ np.abs(w))       # (three entries count: few inexact sums)
    bx = 1.01 * bx + half(compute) * (np.abs(ref.grad_x) + bx) + TINY[compute]
    bx[:, 2:] = 0.0
    assert_within(gx, ref.grad_x, bx, "grad_x")


@pytest.mark.parametrize("grad_w", [False, True])
@pytest.mark.parametrize("rows, ignored", [(40, 0), (300, 3)])
def test_fp16_rows_of_small_weights_keep_their_gradient(grad_w, rows, ignored):
    """Weights 2^20 apart over a vocabulary of small and even probabilities, whose roundings do not cancel (the head's
    entries have a mean in common): each row's gradient is judged by its own size."""
    vocab = 70001
    gen = gen_of(rows)
    w = (1.0 + randn(gen, (vocab, D), "f32", 1.0 / 8)).half()
    x = randn(gen, (rows, D), "f16", 1.0 / 64)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda").to(torch.int32)
    if ignored:
        labels[::ignored] = -1
    weight = torch.where(torch.arange(rows, device="cuda") % 5 == 1, 2.0 ** 12 * 1.1, 2.0 ** -8 * 1.3)
    weight[::11] = 0.0
    _, _, gx, gw = run_loss(svl.make_lm_head(D, vocab, "f16"), x, w, labels, weight, want_w=grad_w)
    x64, w64, wt, l = f64(x), f64(w), f64(weight), labels.cpu().numpy().astype(np.int64)
    for size in (wt > 1, (wt > 0) & (wt < 1), wt == 0):
        own = np.where(size, l, -1)              # rows of one size alone
        ref = ol.lm_loss(x64, w64, own, wt)
        _, _, bx, _ = loss_bounds(x64, w64, own, wt, "f16", ref)
        assert_within(f64(gx)[size & (l >= 0)], ref.grad_x[size & (l >= 0)], bx[size & (l >= 0)], "grad_x")
    if grad_w:
        ref = ol.lm_loss(x64, w64, l, wt)
        assert_within(gw, ref.grad_w, loss_bounds(x64, w64, l, wt, "f16", ref)[3], "grad_w")


def test_fp16_weights_that_differ_over_several_passes():
    """A vocabulary whose passes are of 1280 rows: rows of both passes keep their gradients beside larger weights of
    their own and of the other pass, and the head's gradient sums them all."""
    vocab, rows = 400001, 1400
    gen = gen_of(9)
    w, x = randn(gen, (vocab, D), "f16", 1.0 / 8), randn(gen, (rows, D), "f16")
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda").to(torch.int32)
    weight = torch.exp2(-(torch.arange(rows, device="cuda") % 21).float()) * 1.7 * 2 ** 10
    _, _, gx, gw = run_loss(svl.make_lm_head(D, vocab, "f16"), x, w, labels, weight)
    w64, want_w = w.double(), torch.zeros((vocab, D), dtype=torch.float64, device="cuda")
    for a in range(0, rows, 200):
        p = torch.softmax(x[a:a + 200].double() @ w64.t().contiguous(), 1)
        p[torch.arange(200, device="cuda"), labels[a:a + 200].long()] -= 1
        p *= weight[a:a + 200, None].double()
        want = p @ w64
        # norms: half a step of 16 bits for the exponentials, P and the result, so at most their sum
        off = (gx[a:a + 200].double() - want).norm(dim=1) / want.norm(dim=1)
        assert off.max().item() < 3 * half("f16"), a
        want_w += p.t().contiguous() @ x[a:a + 200].double()
    assert ((gw.double() - want_w).norm() / want_w.norm()).item() < 3 * half("f16")


@pytest.mark.parametrize("weight", [1.01, 1.3, 1.0 / 3000, -1.01])
@pytest.mark.parametrize("grad_w", [False, True])
def test_fp16_equal_weights_cost_no_digits(weight, grad_w):
    """P of a label that is not sure is just under 1, where fp16 rounds by 2^-12 at most, and equal weights leave it
    there: they are multiplied back in float32."""
    vocab, rows = 1000, 300
    gen = gen_of(1)
    x, w = np.zeros((rows, D)), np.zeros((vocab, D))
    w[7, 0] = 1.9375                                   # the label's alone: grad_x[:, 0] is P of the label times it
    w[:, 1] = f64(torch.randint(-64, 64, (vocab,), generator=gen, device="cuda")) / 32
    x[:, 1] = f64(torch.randint(0, 256, (rows,), generator=gen, device="cuda")) / 256
    tx, tw = (torch.from_numpy(t).half().cuda() for t in (x, w))
    labels = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    wt = torch.full((rows,), weight, device="cuda")
    _, _, gx, _ = run_loss(svl.make_lm_head(D, vocab, "f16"), tx, tw, labels, wt, want_w=grad_w)
    s = x @ w.T
    p = np.exp(s - s.max(1, keepdims=True))
    p = (p / p.sum(1, keepdims=True))[:, 7]
    assert 0 < p.min() and p.max() < 0.2
    want = f64(wt) * (p - 1.0) * 1.9375
    # P: half a step under 1, and p's own digits; float32's are some U; then half a step of the result
    bound = np.abs(f64(wt)) * 1.9375 * (2.0 ** -12 + p * 2.0 ** -11 + 100 * U)
    step = np.exp2(np.floor(np.log2(np.abs(want) + bound)) - 11)
    assert step.min() > TINY["f16"]
    assert_within(f64(gx)[:, 0], want, bound + step, "grad_x")


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("want", [(False, False), (True, False), (False, True), (True, True)])
def test_a_large_workspace_serves_fewer_rows(compute, want):
    """A workspace made for more rows serves calls on both sides of the choice of tiles, with the same bits."""
    for d, vocab, most, sizes in ((64, 65537, 300, (1, 65, 128, 129, 256, 257)), (64, 10240, 1024, (705, 768, 769))):
        gen = gen_of(vocab)
        head = svl.make_lm_head(d, vocab, compute)
        x, w = randn(gen, (most, d), compute), randn(gen, (vocab, d), compute, d ** -0.5)
        labels = torch.randint(0, vocab, (most,), generator=gen, device="cuda").to(torch.int32)
        ws = svl.alloc_lm_loss_workspace(head, most, *want)
        for n in sizes:
            ws.fill_(255)
            got = run_loss(head, x[:n], w, labels[:n], None, *want, ws=ws)
            own = run_loss(head, x[:n], w, labels[:n], None, *want)
            assert all(a is None or torch.equal(a, b) for a, b in zip(got, own)), n
