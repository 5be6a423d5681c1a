"""The decoder on a 4-bit cache with a window and sinks: prefill and decode steps
against the float64 oracle whose attention has the same key range, over the
quantised keys and values once a row is past the prefill."""
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2607_20357_amd as svl
import workloads as W
from attention_helpers import f64
from gpu_helpers import host_layer, rel_err_per_sample, tol_for
from oracle import attention as oa

pytestmark = pytest.mark.gpu


def _oracle_attention(steps, window, sinks, compute):
    """Stands for the oracle's causal_attention: rows of the prefill see its rows as they
    are, later ones what the cache stands for."""
    dt = torch.float16 if compute == "f16" else torch.bfloat16

    def attend(q, k, v, counter=None):
        S, d = q.shape
        held = [oa.stands_for(*oa.quantise(torch.from_numpy(x).to(dt).double().numpy(), compute == "f16"))
                for x in (k, v)]
        ok = oa.visible(np.arange(S), S, window, sinks)
        out = np.zeros((S, d))
        for rows, (kk, vv) in ((slice(0, S - steps), (k, v)), (slice(S - steps, S), held)):
            r = oa.attention(q[rows, None], kk[:, None], vv[:, None], ok[rows], d ** -0.5)
            out[rows] = r["out"][:, 0]
        return out
    return attend


def _run(w, seed, steps, window, sinks, monkeypatch, compute="f16"):
    dev, shape = "cuda", w.shape
    cfg = svl.make_config(shape, compute=compute)
    inp = W.draw_inputs(w, seed, device=dev)
    layers = [W.draw_layer_weights(w, l, seed, device=dev) for l in range(shape.n_layers)]
    table = svl.LayerTable(layers)
    B, N = inp.scores.shape
    seq = (np.asarray(inp.keep) + w.n_text).astype(np.int32)
    R, D, max_len = int(seq.sum()), shape.d_model, int(seq.max()) + steps
    cache = svl.alloc_cache4(cfg, B, max_len)
    cache.fill_(0xff)
    ws = svl.alloc_workspace(cfg, B, R)
    kept = torch.empty((B, N), dtype=torch.int32, device=dev)
    resid = torch.empty((R, D), dtype=torch.float32, device=dev)
    cu = svl.svl_prefill_cache4(cfg, table, inp.keep, torch.from_numpy(inp.scores).to(dev), inp.vision, inp.text,
                                inp.layer_mask, inp.head_mask, inp.ffn_mask, window, sinks, kept, resid, cache,
                                max_len, ws)
    assert svl.svl_workspace_status(ws) == 0
    gen = torch.Generator(device=dev).manual_seed(seed + 100)
    new = torch.randn(steps, B, D, generator=gen, device=dev).to(torch.bfloat16).to(torch.float32)
    dws = svl.alloc_decode4_workspace(cfg, B, max_len)
    outs, cache_len = [], seq.copy()
    for t in range(steps):
        x = new[t].clone()
        svl.svl_decode_step4(cfg, table, x, cache_len, inp.layer_mask, inp.head_mask, inp.ffn_mask, window, sinks,
                             cache, max_len, dws)
        outs.append(f64(x))
        cache_len += 1
    text = np.concatenate([W.as_f32(inp.text), new.permute(1, 0, 2).cpu().numpy()], axis=1)
    monkeypatch.setattr(sys.modules["oracle.prefill"], "causal_attention",
                        _oracle_attention(steps, window, sinks, compute))
    ref = oracle.prefill(shape, lambda l: host_layer(layers[l]), inp.scores, np.asarray(inp.keep),
                         W.as_f32(inp.vision), text, inp.layer_mask, inp.head_mask, inp.ffn_mask)
    first = np.concatenate([ref.resid[ref.cu_seqlens[b]:ref.cu_seqlens[b] + seq[b]] for b in range(B)])
    errs = [max(rel_err_per_sample(f64(resid), first, cu))]
    for t in range(steps):
        rows = ref.resid[[ref.cu_seqlens[b] + seq[b] + t for b in range(B)]]
        errs.append(max(np.abs(outs[t][b] - rows[b]).max() / np.abs(rows[b]).max() for b in range(B)))
    print("  prefill, steps:", [f"{e:.2e}" for e in errs], flush=True)
    assert max(errs) <= tol_for(shape), errs


@pytest.mark.parametrize("compute", ["f16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
def test_ragged_batch(window, sinks, compute, monkeypatch):
    """Samples with their own lengths, head groups and skipped layers."""
    w = W.scaled(W.get_workload("llava7b_b8_ragged"), n_layers=3, d_model=512, n_heads=4, n_kv_heads=4,
                 d_ffn=1024, n_vision=200, name="c4")
    _run(w, 7, 3, window, sinks, monkeypatch, compute)


def test_grouped_heads(monkeypatch):
    w = W.scaled(W.get_workload("gqa7b_hires_b2"), n_layers=2, d_model=512, n_heads=4, n_kv_heads=2, d_ffn=1024,
                 n_vision=400, n_text=24, name="c4g")
    _run(w, 8, 2, 33, 2, monkeypatch)


def test_heads_of_64_across_launches(monkeypatch):
    """More samples than one launch's segments."""
    import dataclasses
    base = W.scaled(W.get_workload("llava7b_b8_ragged"), n_layers=2, d_model=256, d_ffn=512, batch=70, n_vision=24,
                    n_text=5, name="c4w")
    w = dataclasses.replace(base, shape=dataclasses.replace(base.shape, n_heads=4, n_kv_heads=2, head_dim=64))
    _run(w, 9, 1, 7, 1, monkeypatch)


def test_cache_rows_are_those_of_the_16_bit_cache():
    """Layer 0's K / V do not depend on the attention: what the 4-bit cache holds of it is
    the 16-bit cache's rows, quantised."""
    w = W.scaled(W.get_workload("llava7b_b1_keep25"), n_layers=1, d_model=512, n_heads=4, n_kv_heads=4, d_ffn=1024,
                 layers_skipped=0, name="c4r")
    dev, shape = "cuda", w.shape
    cfg = svl.make_config(shape)
    inp = W.draw_inputs(w, 3, device=dev)
    inp.layer_mask[:] = 1
    layers = [W.draw_layer_weights(w, 0, 3, device=dev)]
    S = int(inp.keep[0]) + w.n_text
    kept = torch.empty(inp.scores.shape, dtype=torch.int32, device=dev)
    resid = torch.empty((S, shape.d_model), dtype=torch.float32, device=dev)
    ws, c16, c4 = svl.alloc_workspace(cfg, 1, S), svl.alloc_kv_cache(cfg, 1, S), svl.alloc_cache4(cfg, 1, S)
    args = (cfg, layers, inp.keep, torch.from_numpy(inp.scores).to(dev), inp.vision, inp.text, inp.layer_mask,
            inp.head_mask, inp.ffn_mask)
    c16.zero_()
    c4.zero_()
    svl.svl_prefill_cache(*args, kept, resid, c16, S, ws)
    svl.svl_prefill_cache4(*args, 20, 1, kept, resid, c4, S, ws)
    rows = c16.view(torch.float16).view(4, 2, S, 128)
    att = svl.make_attention(4, 4, 128)
    k, v = torch.empty(S, 4, 128, dtype=torch.float16, device=dev), torch.empty(S, 4, 128, dtype=torch.float16, device=dev)
    svl.svl_kv4_read(att, [0, S], [0], c4[0], S, k, v)
    for got, want in ((k, rows[:, 0]), (v, rows[:, 1])):
        want = oa.stands_for(*oa.quantise(f64(want).transpose(1, 0, 2), True))
        assert (np.abs(f64(got) - want) <= 2.0 ** -11 * (1 + 2.0 ** -11) * np.abs(want) + 2.0 ** -25).all()


def test_refusals():
    w = W.scaled(W.get_workload("llava7b_b8_ragged"), n_layers=2, d_model=512, n_heads=4, n_kv_heads=4, d_ffn=1024,
                 batch=2, name="c4bad")
    cfg = svl.make_config(w.shape)
    layers = [W.draw_layer_weights(w, l, 0, device="cuda") for l in range(2)]
    cache, ws = svl.alloc_cache4(cfg, 2, 32), svl.alloc_decode4_workspace(cfg, 2, 32)
    x = torch.zeros(2, 512, device="cuda")
    lm, hm = np.ones((2, 2), np.uint8), np.ones((2, 2, 4), np.uint8)
    step = lambda **kw: svl.svl_decode_step4(*{**dict(cfg=cfg, layers=layers, x=x, cache_len=[0, 3], layer_mask=lm,
                                                      head_mask=hm, ffn_mask=None, window=0, sinks=0, cache=cache,
                                                      max_len=32, ws=ws), **kw}.values())
    for kw, words in ((dict(window=-1), "window"), (dict(sinks=-1), "sinks"), (dict(cache_len=[32, 0]), "cache_len"),
                      (dict(ws=ws[:-256]), "needed")):
        with pytest.raises(svl.SvlError, match=words):
            step(**kw)
    with pytest.raises(ValueError, match="cache"):
        step(cache=cache.view(-1)[:-1])
    with pytest.raises(svl.SvlError, match="cache shape"):
        svl.svl_cache4_bytes(cfg, 2, 40000)
    with pytest.raises(svl.SvlError, match="cache shape"):
        svl.svl_cache4_bytes(svl.make_config(w.shape, dtype="f32"), 2, 40)
