"""The language-model loss and its gradients against the float64 oracle within the
bounds of their roundings (learn_helpers), its refusals of nothing that it allows,
and the operators of a training step together, eagerly and captured."""
import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from learn_helpers import (TYPES, U, assert_within, f64, gen_of, half, loss_bounds, randn, run_loss, strided)
from oracle import learning as ol

pytestmark = pytest.mark.gpu
COMPUTES = ["bf16", "f16"]


def _inputs(rows, d, vocab, compute, ignored=0.0, seed=0, std=1.0, weights="mean"):
    gen = gen_of(seed)
    w = randn(gen, (vocab, d), compute, 1.0 / d ** 0.5)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda").to(torch.int32)
    sure = torch.rand((rows, 1), generator=gen, device="cuda") * 6
    x = (torch.randn((rows, d), generator=gen, device="cuda") * std + sure * w[labels.long()].float()).to(TYPES[compute])
    if ignored:
        gone = torch.rand(rows, generator=gen, device="cuda") < ignored
        bad = torch.tensor([-1, vocab, -100, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
        labels = torch.where(gone, bad[torch.arange(rows, device="cuda") % 4], labels)
        x[gone] = float("nan")
    weight = None
    if weights == "mean":
        weight = torch.full((rows,), (1024.0 if compute == "f16" else 1.0) / rows, device="cuda")
    elif weights == "any":
        weight = torch.exp2(torch.randint(-12, 1, (rows,), generator=gen, device="cuda").float())
        weight *= torch.rand(rows, generator=gen, device="cuda") - 0.3
        weight[::7] = 0.0
    return x, w, labels, weight


def _check(rows, d, vocab, compute, ignored=0.0, seed=0, std=1.0, weights="mean", spread=False, held=False, want_x=True,
           want_w=True):
    x, w, labels, weight = _inputs(rows, d, vocab, compute, ignored, seed, std, weights)
    head = svl.make_lm_head(d, vocab, compute)
    if spread:
        x, w = strided(x, 16), strided(w, 72)
    old = randn(gen_of(seed + 1), (vocab, d), compute, 1e-2) if held else None
    old64 = None if old is None else f64(old)
    loss, lse, gx, gw = run_loss(head, x, w, labels, weight, want_x, want_w, held=old)
    torch.cuda.synchronize()
    l = labels.cpu().numpy().astype(np.int64)
    has = (l >= 0) & (l < vocab)
    x64 = np.where(has[:, None], np.nan_to_num(f64(x)), 0.0)
    w64, wt = f64(w), None if weight is None else f64(weight)
    ref = ol.lm_loss(x64, w64, l, wt)
    b_lse, b_loss, bx, bw = loss_bounds(x64, w64, l, wt, compute, ref)
    assert_within(lse, ref.lse, np.where(has, b_lse, 0.0), "lse")
    assert_within(loss, ref.loss, np.where(has, b_loss, 0.0), "loss")
    if want_x:
        assert_within(gx, ref.grad_x, np.where(has[:, None], bx, 0.0), "grad_x")
    if want_w:
        want = ref.grad_w
        if held:
            want = want + old64
            bw = bw + (half(compute) + 2 * U) * np.abs(want)
        assert_within(gw, want, bw, "grad_w")
    return head, x, w, labels, weight, (loss, lse, gx, gw)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("vocab", [1, 2, 63, 127, 128, 129, 255, 256, 257, 1000])
def test_vocabularies(compute, vocab):
    _check(67, 128, vocab, compute, ignored=0.2, seed=vocab)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("rows", [1, 2, 8, 16, 17, 63, 64, 65, 255, 256, 257, 700])
def test_rows(compute, rows):
    _check(rows, 64, 333, compute, ignored=0.0 if rows < 3 else 0.3, seed=rows, weights="any")


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("vocab", [16384, 16385, 16640 + 63, 16640 + 127, 16640 + 129, 16640 + 255, 17152])
def test_logits_in_whole_tiles(compute, vocab):
    """More than 128 tiles of logits, and more rows than small tiles are taken for; 16384: the last in small ones."""
    _check(300, 64, vocab, compute, ignored=0.2, seed=vocab, weights="any", held=vocab % 2 == 0)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("rows", [128, 129, 256, 257])
def test_logits_of_rows_at_the_choice_of_tiles(compute, rows):
    _check(rows, 128, 129 * 256 - 5, compute, ignored=0.1, seed=rows)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("d", [64, 192, 256, 320, 1024, 3584])
def test_widths(compute, d):
    _check(40, d, 300, compute, seed=d, spread=d % 128 == 64)


@pytest.mark.parametrize("compute", COMPUTES)
def test_cut_sums(compute):
    """Few tiles with a long sum: grad_x over a wide vocabulary, grad_w over many rows."""
    _check(20, 64, 9001, compute)
    _check(3000, 64, 100, compute, ignored=0.1)
    _check(1100, 128, 700, compute, held=True, weights="any")


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("rows", [5, 90, 768, 769])
def test_added_to_what_is_there(compute, rows):
    """Small tiles of the head's gradient (up to 768 rows) and large ones, edges in both directions."""
    _check(rows, 192, 500, compute, ignored=0.2, held=True, weights="any", seed=rows)


@pytest.mark.parametrize("rows", [60, 1500])
def test_sums_cut_in_more_than_a_round(rows):
    """Tiles of the rows' gradient that fill the CUs' rounds only in pieces, by the rows that have a label."""
    for ignored in (0.0, 0.7):
        _check(rows, 1024, 2100, "bf16", ignored=ignored, want_w=False)


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("want", [(False, False), (True, False), (False, True)])
def test_outputs_alone(compute, want):
    head, x, w, labels, weight, got = _check(90, 128, 500, compute, ignored=0.4, want_x=want[0], want_w=want[1])
    full = run_loss(head, x, w, labels, weight)
    for a, b in zip(got, full):
        assert a is None or torch.equal(a, b)
    # nor without log-sums and weights
    loss = torch.empty(90, device="cuda")
    svl.svl_lm_loss(head, x, w, labels, loss, svl.alloc_lm_loss_workspace(head, 90))
    assert torch.equal(loss, full[0])


def test_unit_weights_by_default():
    _check(50, 128, 400, "bf16", weights=None)


@pytest.mark.parametrize("compute", COMPUTES)
def test_large_logits(compute):
    """Sure and far rows: probabilities of 0 and 1."""
    _check(60, 64, 600, compute, std=12.0)


def test_no_row_has_a_label():
    head = svl.make_lm_head(128, 300)
    x, w, labels, weight = _inputs(70, 128, 300, "bf16")
    labels[:] = -1
    x[:] = float("nan")
    loss, lse, gx, gw = run_loss(head, x, w, labels, weight)
    for t in (loss, lse, gx, gw):
        assert (t == 0).all()
    held = randn(gen_of(3), (300, 128), "bf16")
    assert torch.equal(run_loss(head, x, w, labels, weight, held=held.clone())[3], held)


def test_no_rows():
    head = svl.make_lm_head(128, 300)
    x, w, labels, weight = _inputs(4, 128, 300, "bf16")
    loss, lse, gx, gw = run_loss(head, x[:0], w, labels[:0], weight[:0])
    assert (gw == 0).all()
    held = randn(gen_of(3), (300, 128), "bf16")
    assert torch.equal(run_loss(head, x[:0], w, labels[:0], weight[:0], held=held.clone())[3], held)


def test_weights_of_zero():
    head, x, w, labels, weight, _ = _check(70, 128, 300, "f16")
    _, _, gx, gw = run_loss(head, x, w, labels, torch.zeros_like(weight))
    assert (gx == 0).all() and (gw == 0).all()


@pytest.mark.parametrize("compute", COMPUTES)
def test_nonfinite_rows_stay_their_own(compute):
    head, x, w, labels, weight, got = _check(70, 128, 300, compute)
    bad = x.clone()
    bad[9, 3] = float("nan")
    bad[33, 0] = float("inf")
    loss, lse, gx, gw = run_loss(head, bad, w, labels, weight)
    others = torch.ones(70, dtype=torch.bool, device="cuda")
    others[[9, 33]] = False
    for a, b in ((loss, got[0]), (lse, got[1]), (gx, got[2])):
        assert torch.equal(a[others], b[others])
        assert not torch.isfinite(a[9]).all() and not torch.isfinite(a[33]).all()
    assert torch.isnan(gw).any()


def test_small_fp16_weights_keep_their_digits():
    """A loss that is not scaled: fp16's range does not touch P, only what is given back."""
    x, w, labels, _ = _inputs(64, 128, 2000, "f16")
    weight = torch.full((64,), 2.0 ** -30, device="cuda")
    head = svl.make_lm_head(128, 2000, "f16")
    big = run_loss(head, x, w, labels, weight * 2.0 ** 30)
    small = run_loss(head, x, w, labels, weight)
    assert torch.equal((big[2].double() * 2.0 ** -30).half(), small[2])


def _torch_loss(x, w, labels, weight):
    """In float64 on the GPU, some rows at a time (sizes that numpy would take minutes for)."""
    n, v = x.shape[0], w.shape[0]
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    gx, gw = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (x, w))
    w64 = w.double()
    for a in range(0, n, 128):
        at = torch.arange(a, min(n, a + 128), device="cuda")
        at = at[(labels[at] >= 0) & (labels[at] < v)]
        if len(at) == 0:
            continue
        s = x[at].double() @ w64.t().contiguous()
        k = torch.arange(len(at), device="cuda")
        lab = labels[at].long()
        lse[at] = torch.logsumexp(s, 1)
        loss[at] = lse[at] - s[k, lab]
        p = torch.exp(s - lse[at, None])
        p[k, lab] -= 1
        p *= weight[at, None].double()
        gx[at] = p @ w64
        gw += p.t().contiguous() @ x[at].double()
    return loss, lse, gx, gw


@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_several_passes(compute, accumulate):
    """More rows than a pass takes: the head's gradient is summed over passes, rows without a label move the rest."""
    rows, d, vocab = 2500, 64, 400001
    x, w, labels, weight = _inputs(rows, d, vocab, compute, ignored=0.1)
    head = svl.make_lm_head(d, vocab, compute)
    held = randn(gen_of(8), w.shape, compute, 1e-3) if accumulate else None
    want = _torch_loss(torch.nan_to_num(x), w, labels, weight)
    more = 0.0 if held is None else held.double()
    loss, lse, gx, gw = run_loss(head, x, w, labels, weight, held=held)
    # norms: the roundings of P (2 half steps of 16 bits) and of the result, independent, so at most their sum
    for a, b in ((gx, want[2]), (gw, want[3] + more)):
        assert torch.isfinite(a).all() and ((a.double() - b).norm() / b.norm()).item() < 3 * half(compute)
    for a, b in ((loss, want[0]), (lse, want[1])):
        assert (a.double() - b).abs().max().item() < 64 * 2 * U * 40 + 64 * U * b.abs().max().item()
    # the same bits when it is called again on a used workspace
    again = run_loss(head, x, w, labels, weight)
    twice = run_loss(head, x, w, labels, weight)
    assert all(torch.equal(a, b) for a, b in zip(again, twice)) and torch.equal(again[2], gx)


def test_head_past_2_gib():
    """Offsets of the head's rows past 32 bits of bytes."""
    d, vocab, rows = 4096, 300001, 70
    x, w, labels, weight = _inputs(rows, d, vocab, "bf16")
    labels[:3] = torch.tensor([vocab - 1, 0, 270000], device="cuda", dtype=torch.int32)
    head = svl.make_lm_head(d, vocab)
    loss, lse, gx, gw = run_loss(head, x, w, labels, weight)
    want = _torch_loss(x, w, labels, weight)
    for a, b in ((gx, want[2]), (gw, want[3])):
        assert torch.isfinite(a).all() and ((a.double() - b).norm() / b.norm()).item() < 3 * half("bf16")
    assert (loss.double() - want[0]).abs().max().item() < 1e-3


def test_two_streams():
    """Calls at once, each with its own workspace, on streams that are not the tensors' own."""
    sets = [_inputs(300, 256, 5000, c, ignored=0.2, seed=i) for i, c in enumerate(COMPUTES)]
    heads = [svl.make_lm_head(256, 5000, c) for c in COMPUTES]
    want = [run_loss(h, *s) for h, s in zip(heads, sets)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for _ in range(3):
        got = []
        for h, s, st in zip(heads, sets, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append(run_loss(h, *s))
        torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------ together
class _Step:
    """Embedding, final norm, tied head, loss and optimizer as a program uses them: rows of the table are normed
    and score the next token; the table learns from both of its uses."""

    def __init__(self, bits, rows=200, d=256, vocab=700):
        gen = gen_of(11)
        self.rows, self.d, self.vocab = rows, d, vocab
        self.emb = svl.make_embedding(d, vocab, "bf16", "f32", 2.0)
        self.norm = svl.make_norm(d, "rms", "f32", "bf16", "f32")
        self.head = svl.make_lm_head(d, vocab, "bf16")
        self.adam = svl.make_adamw(1e-2, 0.9, 0.95, 1e-8, 0.01, bits)
        self.table, self.gain = randn(gen, (vocab, d), "bf16", 0.5), torch.ones(d, device="cuda")
        new = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
        self.tokens, self.labels = new(rows, dt=torch.int32), new(rows, dt=torch.int32)
        self.weight = torch.full((rows,), 1.0 / rows, device="cuda")
        self.x, self.gx = new(rows, d), new(rows, d)
        self.y, self.gy = new(rows, d, dt=torch.bfloat16), new(rows, d, dt=torch.bfloat16)
        self.stats, self.loss = new(rows, 2), new(rows)
        self.g_table, self.g_gain = new(vocab, d, dt=torch.bfloat16), new(d)
        self.dev = new(5)
        self.ws = [svl.alloc_embed_workspace(self.emb, rows), svl.alloc_norm_workspace(self.norm, rows),
                   svl.alloc_lm_loss_workspace(self.head, rows, True, True)]
        tensors = []
        for p, g in ((self.table, self.g_table), (self.gain, self.g_gain)):
            t = dict(param=p.view(-1), grad=g.view(-1))
            if bits == 8:
                blocks = -(-p.numel() // 256)
                t.update(m=new(p.numel(), dt=torch.uint8), v=new(p.numel(), dt=torch.uint8), m_scale=new(blocks),
                         v_scale=new(blocks))
            else:
                t.update(m=new(p.numel()), v=new(p.numel()))
            tensors.append(t)
        self.tensors = svl.AdamwTensors(tensors)

    def feed(self, step):
        gen = gen_of(100 + step)
        self.tokens.copy_(torch.randint(-2, self.vocab, (self.rows,), generator=gen, device="cuda"))
        self.labels.copy_(torch.where(self.tokens < 0, self.tokens, (self.tokens * 7 + 3) % self.vocab))
        words = torch.tensor([1e-2, 1 - 0.9 ** step, 1 - 0.95 ** step, 1.0, 0.0])
        words.view(torch.int32)[4] = step
        self.dev.copy_(words)

    def run(self):
        svl.svl_embed(self.emb, self.tokens, self.table, self.x)
        svl.svl_norm_forward(self.norm, self.x, self.gain, self.y, stats=self.stats)
        svl.svl_lm_loss(self.head, self.y, self.table, self.labels, self.loss, self.ws[2], row_weight=self.weight,
                        grad_x=self.gy, grad_w=self.g_table)
        svl.svl_norm_backward(self.norm, self.x, self.gain, self.stats, self.gy, self.gx, self.ws[1],
                              grad_gain=self.g_gain)
        svl.svl_embed_backward(self.emb, self.tokens, self.gx, self.g_table, self.ws[0], accumulate=True)
        svl.svl_adamw_step(self.adam, self.tensors, dev=self.dev)

    def all(self):
        return [self.loss, self.g_table, self.g_gain, self.table, self.gain] + [
            x for t in self.tensors.tensors for k, x in sorted(t.items()) if k in ("m", "v")]


def test_step_gradients_are_autograds():
    s = _Step(32)
    s.feed(1)
    table, gain = (t.double().requires_grad_() for t in (s.table, s.gain))
    s.run()
    torch.cuda.synchronize()
    here = s.tokens >= 0
    x = 2.0 * table[s.tokens.long()[here]]
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * gain
    loss = torch.nn.functional.cross_entropy(y @ table.t(), s.labels.long()[here], reduction="sum") / s.rows
    loss.backward()
    # bf16 roundings on the way: y, P, grad_y, and the two of the table's gradient: norms within their sum
    for got, want in ((s.g_table, table.grad), (s.g_gain, gain.grad)):
        assert ((got.double() - want).norm() / want.norm()).item() < 5 * half("bf16")
    assert abs(s.loss.double().sum().item() / s.rows - loss.item()) < 5 * half("bf16") * abs(loss.item())


@pytest.mark.parametrize("bits", [32, 8])
def test_step_captured_and_replayed(bits):
    """A captured step follows its buffers: each replay equals the eager step, other work in between."""
    eager, captured = _Step(bits), _Step(bits)
    captured.feed(1)
    keep = [t.clone() for t in captured.all()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured.run()                                     # warm
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    fresh = _Step(bits)                                    # the state before the first step
    for mine, new in zip(captured.all()[3:5], fresh.all()[3:5]):
        mine.copy_(new)
    for t, u in zip(captured.tensors.tensors, fresh.tensors.tensors):
        for k in t:
            if k not in ("param", "grad"):
                t[k].copy_(u[k])
    del keep
    for step in range(1, 6):
        for s in (eager, captured):
            s.feed(step)
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.all(), captured.all()):
            assert torch.equal(a, b), step
    assert torch.isfinite(eager.table.float()).all()


def test_decoder_learns_through_the_loss():
    """The masked decoder's forward, the norm, the loss and back: svl_train_step takes the norm's gradient, and its
    token and gate gradients match central differences of the whole loss in the oracle's float64."""
    import workloads as W
    from oracle import training as ot
    w = W.get_workload("tiny_f32")
    inp = W.draw_inputs(w, seed=0, device="cuda")
    layers = [W.draw_layer_weights(w, l, 0, device="cuda") for l in range(w.shape.n_layers)]
    cfg = svl.make_config(w.shape)
    N, T, D, L = w.n_vision, w.n_text, w.shape.d_model, w.shape.n_layers
    vocab, P, units = 500, 1, 4
    rng = np.random.default_rng(5)
    z, g = (rng.normal(0.3, 1.5, s).astype(np.float32) for s in ((1, N), (1, (L - P) * units)))
    gen = gen_of(2)
    table, gain = randn(gen, (vocab, D)), 1 + 0.1 * randn(gen, D)
    head_w = randn(gen, (vocab, D), "bf16", D ** -0.5)
    tokens = torch.randint(0, vocab, (T,), generator=gen, device="cuda").to(torch.int32)
    text = torch.empty((T, D), device="cuda")
    svl.svl_embed(svl.make_embedding(D, vocab, "f32", "f32"), tokens, table, text)
    assert torch.equal(text, table[tokens.long()])
    labels = torch.full((N + T,), -1, dtype=torch.int32, device="cuda")      # image rows carry none
    labels[N:N + T - 1] = tokens[1:]
    norm, head = svl.make_norm(D, "rms", "f32", "bf16", "f32"), svl.make_lm_head(D, vocab)
    prm = svl.svl_train_params(0.7, 1.3, P, units)
    tws = svl.alloc_train_workspace(cfg, prm, 1, N, T)
    tz, tg = torch.from_numpy(z).cuda(), torch.from_numpy(g).cuda()
    run = lambda grad: svl.svl_train_step(cfg, svl.LayerTable(layers), prm, tz, tg, inp.vision[:1], text[None], grad, tws)
    hidden = run(None)["hidden"].view(N + T, D)
    y, stats = torch.empty((N + T, D), dtype=torch.bfloat16, device="cuda"), torch.empty((N + T, 2), device="cuda")
    svl.svl_norm_forward(norm, hidden, gain, y, stats=stats)
    weight = torch.full((N + T,), 1.0 / (T - 1), device="cuda")
    loss, _, gy, _ = run_loss(head, y, head_w, labels, weight, want_w=False)
    gx = torch.empty_like(hidden)
    svl.svl_norm_backward(norm, hidden, gain, stats, gy, gx)
    got = run(gx.view(1, N + T, D))
    torch.cuda.synchronize()
    # the same in float64, from the same hidden rows on
    h = hidden.double().requires_grad_()
    yy = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * gain.double()
    at = torch.arange(N, N + T - 1, device="cuda")
    want = torch.nn.functional.cross_entropy(yy[at] @ head_w.double().t(), labels[at].long())
    want.backward()
    assert (gx[:N] == 0).all()
    assert ((gx.double() - h.grad).norm() / h.grad.norm()).item() < 4 * half("bf16")
    assert abs(loss.double().sum().item() / (T - 1) - want.item()) < 4 * half("bf16") * want.item()
    ref = ot.masked_train_step(w.shape, lambda l: {k: W.as_f32(v) for k, v in layers[l].items()}, W.as_f32(inp.vision)[0],
                               f64(text), z[0].astype(np.float64), g[0].astype(np.float64), f64(gx), P, units, 0.7, 1.3)
    gg = got["grad_gate"].cpu().numpy()[0].astype(np.float64)
    assert np.abs(gg - ref.grad_gate).max() <= 1e-3 * np.abs(ref.grad_gate).max()
