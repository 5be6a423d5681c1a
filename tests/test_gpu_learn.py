"""Embedding, row norm and optimizer step against the float64 oracle, within the
bounds of their roundings (learn_helpers); 8-bit optimizer states bit for bit."""
import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from learn_helpers import (TINY, TYPES, U, assert_within, f64, gen_of, half, norm_bounds, norm_grad_bounds, randn,
                           strided)
from oracle import learning as ol

pytestmark = pytest.mark.gpu
NAMES = ["f32", "bf16", "f16"]


# ------------------------------------------------------------------ embedding
def _tokens(gen, n, vocab, how):
    if how == "one":
        return torch.full((n,), vocab - 1, dtype=torch.int32, device="cuda")
    t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    if how == "skewed":
        t = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.6, torch.full_like(t, vocab // 2), t)
    t = t.to(torch.int32)
    if how == "outside" and n:
        bad = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
        t[::3] = bad[torch.arange(len(t[::3]), device="cuda") % 4]
    return t


def _embed(rows, width, vocab, table, row, how="any", scale=1.0, accumulate=False, seed=0, spread=False):
    gen = gen_of(seed)
    emb = svl.make_embedding(width, vocab, table, row, scale)
    tok = _tokens(gen, rows, vocab, how)
    tab, grad = randn(gen, (vocab, width), table), randn(gen, (rows, width), row)
    inside = ((tok >= 0) & (tok < vocab)).cpu().numpy()
    grad[torch.from_numpy(~inside).cuda()] = float("nan")         # rows without a token may hold anything
    out = torch.full((rows, width), float("nan"), dtype=TYPES[row], device="cuda")
    held = randn(gen, (vocab, width), table)
    got = held.clone() if accumulate else torch.full_like(held, float("nan"))
    if spread:
        tab, grad, out, got = (strided(t, 24) for t in (tab, grad, out, got))
    svl.svl_embed(emb, tok, tab, out)
    ws = svl.alloc_embed_workspace(emb, rows)
    ws.fill_(255)
    svl.svl_embed_backward(emb, tok, grad, got, ws, accumulate=accumulate)
    torch.cuda.synchronize()
    t = tok.cpu().numpy().astype(np.int64)
    want = ol.embed(t, f64(tab), scale)
    assert_within(out, want, (half(row) + U) * np.abs(want) + TINY[row], "rows")
    g64 = np.nan_to_num(f64(grad))
    g, size, count = ol.embed_grad(t, g64, vocab, scale)
    bound = 1.01 * (count[:, None] + 2) * U * size
    if accumulate:
        g = g + f64(held)
        bound += U * np.abs(g)
    bound += half(table) * (np.abs(g) + bound) + TINY[table]
    if accumulate:
        bound[count == 0] = 0.0                                   # not touched
    assert_within(got, g, bound, "table gradient")
    return emb, tok, grad, got


@pytest.mark.parametrize("row", NAMES)
@pytest.mark.parametrize("table", NAMES)
def test_embed_types(table, row):
    _embed(37, 72, 50, table, row, "outside", scale=0.7)
    _embed(37, 72, 50, table, row, "skewed", scale=-3.0, accumulate=True, spread=True)


@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 255, 257, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("how", ["any", "one", "skewed", "outside"])
def test_embed_runs(rows, how):
    """Runs that begin and end on, before and behind the pieces of 32 and of 1024."""
    _embed(rows, 40, 19, "f32", "bf16", how, seed=rows)
    _embed(rows, 8, 300, "bf16", "f32", how, accumulate=True, seed=rows)


@pytest.mark.parametrize("rows,vocab,width,how", [(16384, 700, 8, "skewed"), (16385, 70000, 8, "any"),
                                                 (40000, 257, 8, "skewed"), (20000, 1, 16, "one"), (3, 65536, 2056, "any"),
                                                 (300, 255, 4104, "skewed"), (5, 256, 8200, "outside")])
def test_embed_sizes(rows, vocab, width, how):
    _embed(rows, width, vocab, "f32", "f32", how)


def test_embed_keeps_the_order_of_equal_tokens():
    """The same bits on every call, also where several workgroups sort."""
    for rows in (5000, 40000):
        emb, tok, grad, got = _embed(rows, 64, 97, "f32", "f16", "skewed")
        ws = svl.alloc_embed_workspace(emb, rows)
        for _ in range(3):
            again = torch.empty_like(got)
            svl.svl_embed_backward(emb, tok, grad, again, ws)
            assert torch.equal(again, got)


def test_embed_without_rows():
    emb = svl.make_embedding(64, 9, "bf16", "bf16")
    none = torch.empty((0,), dtype=torch.int32, device="cuda")
    rows = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    g = torch.full((9, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = svl.alloc_embed_workspace(emb, 0)
    svl.svl_embed(emb, none, torch.zeros((9, 64), dtype=torch.bfloat16, device="cuda"), rows)
    svl.svl_embed_backward(emb, none, rows, g, ws, accumulate=True)
    assert torch.isnan(g).all()
    svl.svl_embed_backward(emb, none, rows, g, ws)
    assert (g == 0).all()


def test_embed_table_past_2_gib():
    emb = svl.make_embedding(4096, 300000, "bf16", "bf16")
    table = torch.zeros((300000, 4096), dtype=torch.bfloat16, device="cuda")
    tok = torch.tensor([299999, 0, 270000, 299999], dtype=torch.int32, device="cuda")
    row = randn(gen_of(1), (4, 4096), "bf16")
    table[299999], table[270000] = row[0], row[2]
    out = torch.empty_like(row)
    svl.svl_embed(emb, tok, table, out)
    assert torch.equal(out, torch.stack([row[0], torch.zeros_like(row[0]), row[2], row[0]]))
    svl.svl_embed_backward(emb, tok, row, table, svl.alloc_embed_workspace(emb, 4))
    assert torch.equal(table[299999], (row[0].float() + row[3].float()).bfloat16())
    assert torch.equal(table[270000], row[2]) and torch.equal(table[0], row[1])
    assert not table[1:270000].any()


# ------------------------------------------------------------------ norm
def _norm(rows, width, kind, x_type, y_type, gain_type, gain=True, bias=False, seed=0, offset=0.1, spread=False, size=1.0,
          eps=1e-6, held=False):
    gen = gen_of(seed)
    layer = kind == "layer"
    norm = svl.make_norm(width, kind, x_type, y_type, gain_type, eps)
    x = ((torch.randn((rows, width), generator=gen, device="cuda") + offset) * size).to(TYPES[x_type])
    g = randn(gen, width, gain_type) if gain else None
    b = randn(gen, width, gain_type) if bias else None
    gy = randn(gen, (rows, width), y_type)
    y = torch.full_like(gy, float("nan"))
    gx = torch.full_like(x, float("nan"))
    stats = torch.full((rows, 2), float("nan"), device="cuda")
    gg = randn(gen, width) if held else torch.full((width,), float("nan"), device="cuda")
    gb = randn(gen, width) if held else torch.full((width,), float("nan"), device="cuda")
    held_g, held_b = f64(gg), f64(gb)
    if spread:
        x, gy, y, gx = (strided(t, 16) for t in (x, gy, y, gx))
    svl.svl_norm_forward(norm, x, g, y, bias=b, stats=stats)
    ws = svl.alloc_norm_workspace(norm, rows)
    ws.fill_(255)
    svl.svl_norm_backward(norm, x, g, stats, gy, gx, ws, grad_gain=gg, grad_bias=gb, accumulate=held)
    torch.cuda.synchronize()
    g64, b64 = (None if t is None else f64(t) for t in (g, b))
    want, bound, dz, er = norm_bounds(f64(x), g64, b64, layer, np.float64(np.float32(eps)), y_type)
    assert_within(y, want, bound, "y")
    (wx, bx), (wg, bg), (wb, bb) = norm_grad_bounds(f64(x), f64(gy), g64, layer, np.float64(np.float32(eps)), x_type, dz, er)
    assert_within(gx, wx, bx, "grad_x")
    if held:
        wg, wb = wg + held_g, wb + held_b
        bg, bb = bg + U * np.abs(wg), bb + U * np.abs(wb)
    assert_within(gg, wg, bg, "grad_gain")
    assert_within(gb, wb, bb, "grad_bias")
    return norm, x, g, b, stats, gy, gx, gg


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("x_type", NAMES)
@pytest.mark.parametrize("y_type", NAMES)
def test_norm_types(kind, x_type, y_type):
    for gain_type in NAMES:
        _norm(9, 264, kind, x_type, y_type, gain_type, bias=kind == "layer")


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", [8, 16, 504, 512, 520, 1024, 1032, 2048, 2056, 3584, 4096, 5120, 8192, 8200, 16384])
def test_norm_widths(kind, width):
    _norm(5, width, kind, "f32", "f32", "f32", bias=True, seed=width)


@pytest.mark.parametrize("rows", [1, 2, 3, 63, 511, 512, 513, 1500])
def test_norm_rows(rows):
    _norm(rows, 256, "layer", "bf16", "f16", "bf16", bias=True, seed=rows, held=rows % 2 == 1)
    _norm(rows, 1096, "rms", "f32", "bf16", "bf16", seed=rows, spread=True)


def test_norm_without_gain_and_of_far_rows():
    _norm(7, 512, "rms", "f32", "f32", "f32", gain=False)
    _norm(7, 2560, "layer", "f32", "f32", "f32", gain=False, bias=True, offset=30.0)
    _norm(7, 512, "rms", "f32", "f32", "f32", size=1e-12)
    _norm(7, 512, "rms", "bf16", "bf16", "f32", size=1e15)


def test_norm_zero_rows_and_nonfinite_rows():
    norm = svl.make_norm(1024, "layer", "f32", "f32", "f32", 1e-6)
    x = randn(gen_of(3), (6, 1024))
    x[1] = 0.0
    x[2] = 5.0
    x[4, 7] = float("inf")
    x[5, 100] = float("nan")
    y, stats, gx = torch.empty_like(x), torch.empty((6, 2), device="cuda"), torch.empty_like(x)
    svl.svl_norm_forward(norm, x, None, y, stats=stats)
    svl.svl_norm_backward(norm, x, None, stats, torch.ones_like(x), gx)
    assert (y[1:3] == 0).all() and torch.isfinite(y[:4]).all() and torch.isfinite(gx[:4]).all()
    assert torch.isnan(y[4]).any() and torch.isnan(y[5]).all()


@pytest.mark.parametrize("width", [256, 1024, 4096, 8192, 16384])
def test_norm_in_place_and_repeatable(width):
    norm, x, g, b, stats, gy, gx, gg = _norm(600, width, "rms", "f32", "f32", "f32")
    y = torch.empty_like(x)
    svl.svl_norm_forward(norm, x, g, y)
    over = x.clone()
    svl.svl_norm_forward(norm, over, g, over)
    assert torch.equal(over, y)
    ws = svl.alloc_norm_workspace(norm, 600)
    over, again = gy.clone(), torch.empty_like(gg)
    svl.svl_norm_backward(norm, x, g, stats, over, over, ws, grad_gain=again)
    assert torch.equal(over, gx) and torch.equal(again, gg)


def test_norm_weight_gradients_alone():
    norm, x, g, b, stats, gy, gx, gg = _norm(70, 256, "layer", "f16", "f16", "f32")
    ws = svl.alloc_norm_workspace(norm, 70)
    again, bias = torch.empty_like(gg), torch.zeros_like(gg)
    svl.svl_norm_backward(norm, x, g, stats, gy, None, ws, grad_gain=again)
    svl.svl_norm_backward(norm, x, g, stats, gy, None, ws, grad_bias=bias, accumulate=True)
    assert torch.equal(again, gg)
    assert_within(bias, f64(gy).sum(0), 74 * U * np.abs(f64(gy)).sum(0), "grad_bias")
    svl.svl_norm_backward(norm, x[:0], g, stats[:0], gy[:0], None, ws, grad_gain=again)
    assert (again == 0).all()


# ------------------------------------------------------------------ optimizer
LR, B1, B2, EPS, DECAY = 3e-3, 0.9, 0.99, 1e-8, 0.05


def _state(gen, n, bits, spread):
    if bits == 32:
        return dict(m=randn(gen, n) * spread, v=torch.rand(n, generator=gen, device="cuda") * spread ** 2)
    blocks = -(-n // 256)
    t = dict(m=torch.randint(0, 256, (n,), generator=gen, device="cuda").to(torch.uint8),
             v=torch.randint(0, 256, (n,), generator=gen, device="cuda").to(torch.uint8))
    for k in ("m_scale", "v_scale"):
        t[k] = torch.exp2(torch.randint(-14, 3, (blocks,), generator=gen, device="cuda").float())
    # codes of the top 8 binades: none past what a step leaves
    t["m"] = (t["m"] & 128) | (64 + (t["m"] & 63)).clamp(max=119)
    t["v"] = (176 + (t["v"] & 63)).clamp(max=247)
    return {k: x.to(torch.uint8) if k in ("m", "v") else x for k, x in t.items()}


def _adamw(sizes, param, grad, bits, master=False, steps=3, seed=0, grad_scale=1.0, edit=None, dev=False):
    gen = gen_of(seed)
    adam = svl.make_adamw(LR, B1, B2, EPS, DECAY, bits)
    tensors = []
    for n in sizes:
        t = dict(param=randn(gen, n, param, 0.1), grad=randn(gen, n, grad, 0.02), **_state(gen, n, bits, 0.02))
        if master:
            t["master"] = t["param"].float() * (1 + 2.0 ** -12)
        tensors.append(t)
    if edit:
        edit(tensors)
    table = svl.AdamwTensors(tensors)
    for step in range(1, steps + 1):
        before = [{k: x.cpu() for k, x in t.items()} for t in tensors]
        if dev:
            words = torch.tensor([LR, 1 - B1 ** step, 1 - B2 ** step, grad_scale, 0.0], device="cuda")
            words.view(torch.int32)[4] = 77 + step
            svl.svl_adamw_step(adam, table, step=0, dev=words)
        else:
            svl.svl_adamw_step(adam, table, step=step, seed=77 + step, grad_scale=grad_scale)
        torch.cuda.synchronize()
        for i, (t, old) in enumerate(zip(tensors, before)):
            if t["param"].numel() == 0:
                continue
            if bits == 32:
                m0, v0 = f64(old["m"]), f64(old["v"])
            else:
                m0, v0 = (ol.decode(old[k].numpy(), old[k + "_scale"].numpy(), k == "v") for k in ("m", "v"))
            m, v = ol.moments(f64(old["grad"]), m0, v0, B1, B2, grad_scale)
            p0 = f64(old["master"] if master else old["param"])
            want, rate = ol.adamw(p0, m, v, step, LR, B1, B2, EPS, DECAY)
            # p keep, the corrections, root, sum, two quotients, a product, the difference, lr and eps themselves
            bound = 4 * U * np.abs(p0) + 12 * U * np.abs(rate)
            if master:
                assert_within(t["master"], want, bound, f"master {i}")
                assert torch.equal(t["param"], t["master"].to(TYPES[param]))
            else:
                assert_within(t["param"], want, bound + half(param) * (np.abs(want) + bound) + TINY[param], f"param {i}")
            if bits == 32:
                assert np.array_equal(f64(t["m"]), m) and np.array_equal(f64(t["v"]), v)
                continue
            low, high = ol.random_bits(len(m), 77 + step, i)
            for k, x, r, lo, signed in (("m", m, low, ol.LOW_M, True), ("v", ol.f32(np.sqrt(v)), high, ol.LOW_V, False)):
                code, scale = ol.encode(x, r, lo, signed)
                assert np.array_equal(t[k + "_scale"].cpu().numpy()[:len(scale)], scale, equal_nan=True), k
                assert np.array_equal(t[k].cpu().numpy(), code), k
    return tensors


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", NAMES)
@pytest.mark.parametrize("grad", NAMES)
def test_adamw_types(param, grad, bits):
    _adamw([300, 1, 256, 0, 257, 4096, 4097], param, grad, bits)
    _adamw([511, 2049], param, grad, bits, master=True, steps=2, grad_scale=0.25)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_many_tensors(bits):
    """More tensors than a launch takes, empty ones among them: each keeps its number."""
    _adamw([(37 * i) % 700 for i in range(130)], "bf16", "f32", bits, master=True, steps=2)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_step_values_on_the_device(bits):
    _adamw([700, 5000], "f32", "f32", bits, dev=True, grad_scale=0.5)


def test_adamw_8bit_edges():
    """Blocks of zeros, one value, huge spreads, and the least scale."""
    def edit(tensors):
        t = tensors[0]
        for k in ("m", "v"):
            t[k][:512] = 0
            t[k + "_scale"][:2] = 0.0
        t["grad"][:512] = 0.0
        t["grad"][300] = 1e-3
        t["m"][512:768] = 0
        t["v"][512:768] = 0
        t["grad"][512:768] = 2.0 ** -80
        t["grad"][768:1024] *= torch.exp2(-torch.arange(256, device="cuda").float() / 8)
    _adamw([2000], "f32", "f32", 8, edit=edit, steps=4)


def test_adamw_8bit_nonfinite_block():
    def edit(tensors):
        tensors[0]["grad"][5] = float("inf")
        tensors[0]["grad"][600] = float("nan")
    gen = gen_of(0)
    t = dict(param=randn(gen, 1024), grad=randn(gen, 1024), **_state(gen, 1024, 8, 1.0))
    edit([t])
    svl.svl_adamw_step(svl.make_adamw(LR, state_bits=8), [t])
    for k in ("m", "v"):
        v = torch.empty(1024, device="cuda")
        svl.svl_adamw_read_state(k, t[k], t[k + "_scale"], v)
        bad = torch.isnan(v).view(4, 256)
        assert bad[0].all() and bad[2].all() and not bad[1].any() and not bad[3].any()


@pytest.mark.parametrize("n", [1, 7, 8, 255, 256, 1000])
def test_adamw_read_state(n):
    gen = gen_of(n)
    codes = torch.randint(0, 256, (n,), generator=gen, device="cuda").to(torch.uint8)
    scales = torch.exp2(torch.randint(-30, 3, (-(-n // 256),), generator=gen, device="cuda").float())
    for k in ("m", "v"):
        out = torch.full((n + 8,), -7.0, device="cuda")
        svl.svl_adamw_read_state(k, codes, scales, out)
        want = ol.decode(codes.cpu().numpy(), scales.cpu().numpy(), k == "v")
        assert np.array_equal(f64(out[:n]), want) and (out[n:] == -7.0).all()


def test_adamw_small_changes_are_not_lost():
    """A second moment that only decays follows its decay on average, though a step is a hundredth of a code's."""
    n = 1 << 16
    t = dict(param=torch.zeros(n, device="cuda"), grad=torch.zeros(n, device="cuda"),
             m=torch.zeros(n, dtype=torch.uint8, device="cuda"),
             v=torch.full((n,), 240, dtype=torch.uint8, device="cuda"),
             m_scale=torch.zeros(n // 256, device="cuda"), v_scale=torch.ones(n // 256, device="cuda"))
    adam = svl.make_adamw(0.0, 0.9, 0.99, state_bits=8)
    table = svl.AdamwTensors([t])
    for step in range(1, 201):
        svl.svl_adamw_step(adam, table, step=step, seed=step)
    v = torch.empty(n, device="cuda")
    svl.svl_adamw_read_state("v", t["v"], t["v_scale"], v)
    # the root decays by sqrt(0.99) a step without bias: its mean after 200 is 0.99^100 = 0.366; a value's
    # deviation is under 1/8 of it a step, sqrt(200) steps over 65536 values: under 0.7 percent
    assert abs(v.double().sqrt().mean().item() / 0.99 ** 100 - 1) < 0.01


def test_adamw_touches_nothing_else():
    for bits in (32, 8):
        gen = gen_of(5)
        wide = {k: x for k, x in dict(param=randn(gen, 1000, "bf16"), grad=randn(gen, 1000), master=randn(gen, 1000),
                                      **_state(gen, 1000, bits, 1.0)).items()}
        before = {k: x.clone() for k, x in wide.items()}
        part = {k: x[:1] if k.endswith("scale") else x[:203] for k, x in wide.items()}
        svl.svl_adamw_step(svl.make_adamw(LR, state_bits=bits), [part])
        for k, x in wide.items():
            n = 1 if k.endswith("scale") else 203
            assert torch.equal(x[n:], before[k][n:])
            assert k == "grad" or not torch.equal(x[:n], before[k][:n])
