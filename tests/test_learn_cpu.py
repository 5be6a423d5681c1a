"""Host-side checks of embedding, row norm, language-model loss and optimizer step
(no GPU): exports, workspace sizes, and every refusal, through the C ABI with
pointers that are never followed and through the binding."""
import ctypes
import os
import re

import pytest
import torch

import paper_2607_20357_amd as svl
from paper_2607_20357_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 16 * 4096
NULL, SHAPE, VALUE, WORKSPACE, DTYPE, HIP, ALIGN = 1, 2, 3, 4, 5, 6, 7
BIG = 1 << 50


def test_exports():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "svl.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(svl_(?:embed|norm|lm|adamw)_?[a-z0-9_]*)\s*\(", text))
    assert names == {"svl_embed", "svl_embed_workspace_bytes", "svl_embed_backward", "svl_norm_forward",
                     "svl_norm_workspace_bytes", "svl_norm_backward", "svl_lm_loss_workspace_bytes", "svl_lm_loss",
                     "svl_adamw_step", "svl_adamw_read_state"}
    for n in names:
        assert hasattr(svl.load_library(), n) and hasattr(svl, n)


def _status(name, order, args, **change):
    args = dict(args, **change)
    return getattr(svl.load_library(), name)(*[args[k] for k in order])


def _refused(name, order, args, cases, word=None):
    for change, status in cases:
        assert _status(name, order, args, **change) == status, (change, svl.load_library().svl_last_error())


def _emb(**kw):
    e = svl.make_embedding(64, 100)
    for k, v in kw.items():
        setattr(e, k, v)
    return ctypes.byref(e)


EMBED = ("emb", "rows", "tokens", "table", "ldt", "out", "ldo", "stream")
EMBED_BACK = ("emb", "rows", "tokens", "grad", "ldg", "table", "ldt", "acc", "ws", "nws", "stream")


def test_embed_refusals():
    ok = dict(emb=_emb(), rows=4, tokens=P, table=P, ldt=64, out=P, ldo=64, stream=None)
    descs = [(dict(emb=None), NULL), (dict(emb=_emb(width=0)), SHAPE), (dict(emb=_emb(width=60)), SHAPE),
             (dict(emb=_emb(width=65544)), SHAPE), (dict(emb=_emb(vocab=0)), SHAPE), (dict(emb=_emb(vocab=1 << 24)), SHAPE),
             (dict(emb=_emb(table_type=3)), DTYPE), (dict(emb=_emb(row_type=-1)), DTYPE),
             (dict(emb=_emb(scale=float("inf"))), VALUE), (dict(emb=_emb(scale=float("nan"))), VALUE)]
    _refused("svl_embed", EMBED, ok, descs + [
        (dict(rows=-1), SHAPE), (dict(rows=1 << 24), SHAPE), (dict(tokens=None), NULL), (dict(tokens=P + 2), ALIGN),
        (dict(table=None), NULL), (dict(table=P + 8), ALIGN), (dict(ldt=56), SHAPE), (dict(ldt=68), SHAPE),
        (dict(ldt=(1 << 23) + 8), SHAPE), (dict(out=None), NULL), (dict(out=P + 4), ALIGN), (dict(ldo=60), SHAPE)])
    back = dict(emb=_emb(), rows=4, tokens=P, grad=P, ldg=64, table=P, ldt=64, acc=0, ws=P, nws=BIG, stream=None)
    _refused("svl_embed_backward", EMBED_BACK, back, descs + [
        (dict(rows=-1), SHAPE), (dict(tokens=None), NULL), (dict(grad=None), NULL), (dict(grad=P + 8), ALIGN),
        (dict(ldg=56), SHAPE), (dict(table=None), NULL), (dict(ldt=65), SHAPE), (dict(acc=2), VALUE),
        (dict(ws=None), NULL), (dict(ws=P + 8), ALIGN),
        (dict(nws=svl.svl_embed_workspace_bytes(svl.make_embedding(64, 100), 4) - 1), WORKSPACE)])
    # no work: nothing is asked of the pointers
    assert _status("svl_embed", EMBED, ok, rows=0, tokens=None, table=None, out=None) == 0
    assert _status("svl_embed_backward", EMBED_BACK, back, rows=0, tokens=None, grad=None, acc=1, ws=None, nws=0) == 0


def _nrm(**kw):
    n = svl.make_norm(64)
    for k, v in kw.items():
        setattr(n, k, v)
    return ctypes.byref(n)


NORM = ("norm", "rows", "x", "ldx", "gain", "bias", "y", "ldy", "stats", "stream")
NORM_BACK = ("norm", "rows", "x", "ldx", "gain", "stats", "gy", "ldgy", "gx", "ldgx", "gg", "gb", "acc", "ws", "nws",
             "stream")


def test_norm_refusals():
    ok = dict(norm=_nrm(), rows=4, x=P, ldx=64, gain=P, bias=None, y=2 * P, ldy=64, stats=None, stream=None)
    descs = [(dict(norm=None), NULL), (dict(norm=_nrm(width=0)), SHAPE), (dict(norm=_nrm(width=68)), SHAPE),
             (dict(norm=_nrm(width=16392)), SHAPE), (dict(norm=_nrm(kind=2)), VALUE), (dict(norm=_nrm(x_type=3)), DTYPE),
             (dict(norm=_nrm(y_type=9)), DTYPE), (dict(norm=_nrm(gain_type=-1)), DTYPE),
             (dict(norm=_nrm(eps=-1.0)), VALUE), (dict(norm=_nrm(eps=float("nan"))), VALUE)]
    _refused("svl_norm_forward", NORM, ok, descs + [
        (dict(rows=-1), SHAPE), (dict(x=None), NULL), (dict(x=P + 8), ALIGN), (dict(ldx=56), SHAPE), (dict(ldx=65), SHAPE),
        (dict(y=None), NULL), (dict(y=P + 8), ALIGN), (dict(ldy=60), SHAPE), (dict(gain=P + 8), ALIGN),
        (dict(bias=P + 2), ALIGN), (dict(stats=P + 4), ALIGN), (dict(y=P), VALUE),
        (dict(norm=_nrm(y_type=0), y=P, ldy=72), VALUE)])
    back = dict(norm=_nrm(), rows=4, x=P, ldx=64, gain=P, stats=P, gy=2 * P, ldgy=64, gx=3 * P, ldgx=64, gg=P, gb=P, acc=0,
                ws=P, nws=BIG, stream=None)
    need = svl.svl_norm_workspace_bytes(svl.make_norm(64), 4)
    _refused("svl_norm_backward", NORM_BACK, back, descs + [
        (dict(rows=-1), SHAPE), (dict(x=None), NULL), (dict(ldx=63), SHAPE), (dict(gain=P + 8), ALIGN),
        (dict(stats=None), NULL), (dict(stats=P + 4), ALIGN), (dict(gy=None), NULL), (dict(ldgy=8), SHAPE),
        (dict(gx=P + 8), ALIGN), (dict(ldgx=60), SHAPE), (dict(gx=2 * P), VALUE), (dict(gg=P + 4), ALIGN),
        (dict(gb=P + 8), ALIGN), (dict(acc=-1), VALUE), (dict(ws=None), NULL), (dict(nws=need - 1), WORKSPACE)])
    assert _status("svl_norm_forward", NORM, ok, rows=0, x=None, y=None) == 0
    assert _status("svl_norm_backward", NORM_BACK, back, rows=0, x=None, gy=None, stats=None, gg=None, gb=None) == 0


def _hd(**kw):
    h = svl.make_lm_head(64, 100)
    for k, v in kw.items():
        setattr(h, k, v)
    return ctypes.byref(h)


LOSS = ("head", "rows", "x", "ldx", "w", "ldw", "labels", "weight", "loss", "lse", "gx", "ldgx", "gw", "ldgw", "acc", "ws",
        "nws", "stream")


def test_loss_refusals():
    ok = dict(head=_hd(), rows=4, x=P, ldx=64, w=P, ldw=64, labels=P, weight=P, loss=P, lse=P, gx=P, ldgx=64, gw=P, ldgw=64,
              acc=0, ws=P, nws=BIG, stream=None)
    need = svl.svl_lm_loss_workspace_bytes(svl.make_lm_head(64, 100), 4, True, True)
    _refused("svl_lm_loss", LOSS, ok, [
        (dict(head=None), NULL), (dict(head=_hd(d_model=0)), SHAPE), (dict(head=_hd(d_model=72)), SHAPE),
        (dict(head=_hd(d_model=65600)), SHAPE), (dict(head=_hd(vocab=0)), SHAPE),
        (dict(head=_hd(vocab=(1 << 20) + 1)), SHAPE), (dict(head=_hd(compute=2)), DTYPE), (dict(rows=-1), SHAPE),
        (dict(rows=1 << 24), SHAPE), (dict(x=None), NULL), (dict(x=P + 8), ALIGN), (dict(ldx=56), SHAPE),
        (dict(ldx=(1 << 21) + 8), SHAPE), (dict(w=None), NULL), (dict(ldw=65), SHAPE), (dict(labels=None), NULL),
        (dict(labels=P + 1), ALIGN), (dict(weight=P + 2), ALIGN), (dict(loss=None), NULL), (dict(loss=P + 2), ALIGN),
        (dict(lse=P + 2), ALIGN), (dict(gx=P + 8), ALIGN), (dict(ldgx=56), SHAPE), (dict(gw=P + 8), ALIGN),
        (dict(ldgw=8), SHAPE), (dict(acc=7), VALUE), (dict(ws=None), NULL), (dict(ws=P + 8), ALIGN),
        (dict(nws=need - 1), WORKSPACE)])
    # without gradients less is needed
    less = svl.svl_lm_loss_workspace_bytes(svl.make_lm_head(64, 100), 4)
    assert less < need
    assert _status("svl_lm_loss", LOSS, ok, gx=None, gw=None, nws=less - 1) == WORKSPACE
    assert _status("svl_lm_loss", LOSS, ok, rows=0, x=None, w=None, labels=None, loss=None, gw=None, ws=None) == 0


def test_workspace_is_bounded():
    """Rows beyond a piece cost their own rows, not the vocabulary."""
    head = svl.make_lm_head(4096, 32000)
    a, b = (svl.svl_lm_loss_workspace_bytes(head, n, True, False) for n in (1 << 15, 1 << 17))
    assert b - a < ((1 << 17) - (1 << 15)) * (4096 * 2 + 16) + 4096
    assert a < (1 << 15) * (4096 * 2 + 16) + (5 << 28)
    for bad in (dict(rows=-1), dict(rows=1 << 24)):
        with pytest.raises(svl.SvlError, match="rows"):
            svl.svl_lm_loss_workspace_bytes(head, **bad)
    with pytest.raises(svl.SvlError, match="d_model"):
        svl.svl_lm_loss_workspace_bytes(svl.make_lm_head(100, 5), 1)
    with pytest.raises(svl.SvlError, match="width"):
        svl.svl_embed_workspace_bytes(svl.make_embedding(12, 5), 1)
    with pytest.raises(svl.SvlError, match="width"):
        svl.svl_norm_workspace_bytes(svl.make_norm(12), 1)


ADAM = ("adam", "count", "tensors", "step", "seed", "scale", "dev", "stream")


def _adam(**kw):
    a = svl.make_adamw(1e-3)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


def _tensors(**kw):
    t = dict(n=10, param_type=0, grad_type=0, param=P, grad=P, master=None, m=P, v=P, m_scale=None, v_scale=None)
    t.update(kw)
    return (binding.svl_adamw_tensor * 1)(binding.svl_adamw_tensor(**t))


def test_adamw_refusals():
    ok = dict(adam=_adam(), count=1, tensors=_tensors(n=0), step=1, seed=0, scale=1.0, dev=None, stream=None)
    inf, nan = float("inf"), float("nan")
    _refused("svl_adamw_step", ADAM, ok, [
        (dict(adam=None), NULL), (dict(adam=_adam(lr=inf)), VALUE), (dict(adam=_adam(beta1=1.0)), VALUE),
        (dict(adam=_adam(beta1=-0.1)), VALUE), (dict(adam=_adam(beta2=nan)), VALUE), (dict(adam=_adam(eps=-1.0)), VALUE),
        (dict(adam=_adam(eps=inf)), VALUE), (dict(adam=_adam(weight_decay=-1.0)), VALUE),
        (dict(adam=_adam(state_bits=16)), DTYPE), (dict(count=-1), SHAPE), (dict(tensors=None), NULL),
        (dict(step=0), VALUE), (dict(scale=nan), VALUE), (dict(dev=P + 2), ALIGN),
        (dict(tensors=_tensors(n=-1)), SHAPE), (dict(tensors=_tensors(n=(1 << 40) + 1)), SHAPE),
        (dict(tensors=_tensors(param_type=3)), DTYPE), (dict(tensors=_tensors(grad_type=-1)), DTYPE),
        (dict(tensors=_tensors(param=None)), NULL), (dict(tensors=_tensors(grad=None)), NULL),
        (dict(tensors=_tensors(m=None)), NULL), (dict(tensors=_tensors(v=None)), NULL),
        (dict(tensors=_tensors(param=P + 4)), ALIGN), (dict(tensors=_tensors(grad=P + 8)), ALIGN),
        (dict(tensors=_tensors(master=P + 4)), ALIGN), (dict(tensors=_tensors(m=P + 8)), ALIGN),
        (dict(tensors=_tensors(v=P + 8)), ALIGN), (dict(adam=_adam(state_bits=8), tensors=_tensors()), NULL),
        (dict(adam=_adam(state_bits=8), tensors=_tensors(m_scale=P, v_scale=P + 2)), ALIGN)])
    assert _status("svl_adamw_step", ADAM, ok) == 0                       # a tensor without elements
    assert _status("svl_adamw_step", ADAM, ok, count=0, tensors=None) == 0
    read = ("second", "n", "codes", "scales", "out", "stream")
    good = dict(second=0, n=10, codes=P, scales=P, out=P, stream=None)
    _refused("svl_adamw_read_state", read, good, [
        (dict(second=2), VALUE), (dict(n=-1), SHAPE), (dict(codes=None), NULL), (dict(codes=P + 8), ALIGN),
        (dict(scales=None), NULL), (dict(scales=P + 2), ALIGN), (dict(out=None), NULL), (dict(out=P + 4), ALIGN)])


def test_binding_checks_tensors_before_pointers():
    f, b, i = torch.float32, torch.bfloat16, torch.int32
    z = lambda *s, dtype=f: torch.zeros(s, dtype=dtype)
    ws = z(1 << 20, dtype=torch.uint8)
    emb = svl.make_embedding(64, 10)
    with pytest.raises(ValueError, match="tokens has dtype"):
        svl.svl_embed(emb, z(3, dtype=torch.int64), z(10, 64, dtype=b), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="table has shape"):
        svl.svl_embed(emb, z(3, dtype=i), z(10, 56, dtype=b), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="table holds 9 rows"):
        svl.svl_embed(emb, z(3, dtype=i), z(9, 64, dtype=b), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="out holds 2 rows"):
        svl.svl_embed(emb, z(3, dtype=i), z(10, 64, dtype=b), z(2, 64, dtype=b))
    with pytest.raises(ValueError, match="GPU tensor"):
        svl.svl_embed(emb, z(3, dtype=i), z(10, 64, dtype=b), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="grad_rows has dtype"):
        svl.svl_embed_backward(emb, z(3, dtype=i), z(3, 64), z(10, 64, dtype=b), ws)
    norm = svl.make_norm(64)
    with pytest.raises(ValueError, match="gain has dtype"):
        svl.svl_norm_forward(norm, z(3, 64), z(64), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="y has dtype"):
        svl.svl_norm_forward(norm, z(3, 64), z(64, dtype=b), z(3, 64))
    with pytest.raises(ValueError, match="stride"):
        svl.svl_norm_forward(norm, z(3, 68)[:, :64], z(64, dtype=b), z(3, 64, dtype=b))
    with pytest.raises(ValueError, match="stats"):
        svl.svl_norm_forward(norm, z(3, 64), None, z(3, 64, dtype=b), stats=z(2, 2))
    with pytest.raises(ValueError, match="stats is required"):
        svl.svl_norm_backward(norm, z(3, 64), None, None, z(3, 64, dtype=b), None)
    with pytest.raises(ValueError, match="grad_gain has dtype"):
        svl.svl_norm_backward(norm, z(3, 64), None, z(3, 2), z(3, 64, dtype=b), None, ws, grad_gain=z(64, dtype=b))
    head = svl.make_lm_head(64, 10)
    x, w, l = z(3, 64, dtype=b), z(10, 64, dtype=b), z(3, dtype=i)
    for kw, match in ((dict(x=z(3, 64)), "x has dtype"), (dict(w=z(9, 64, dtype=b)), "w holds 9"),
                      (dict(labels=z(2, dtype=i)), "labels has shape"), (dict(loss=z(3, dtype=b)), "loss has dtype"),
                      (dict(lse=z(2)), "lse has shape"), (dict(row_weight=z(3, 1)), "row_weight has shape"),
                      (dict(grad_x=z(2, 64, dtype=b)), "grad_x holds"), (dict(grad_w=z(10, 64)), "grad_w has dtype"),
                      (dict(ws=z(4)), "ws has dtype"), (dict(), "GPU tensor")):
        args = dict(x=x, w=w, labels=l, loss=z(3), ws=ws)
        args.update(kw)
        with pytest.raises(ValueError, match=match):
            svl.svl_lm_loss(head, **args)
    t = dict(param=z(300), grad=z(300), m=z(300), v=z(300))
    eight = dict(t, m=z(300, dtype=torch.uint8), v=z(300, dtype=torch.uint8), m_scale=z(2), v_scale=z(2))
    for bad, match in ((dict(t, grad=None), "grad is missing"), (dict(t, m=z(299)), "m holds 299"),
                       (dict(t, v=z(300, dtype=b)), "v has dtype"), (dict(t, master=z(300, dtype=b)), "master has dtype"),
                       (dict(t, other=z(3)), "unknown"), (dict(eight, m_scale=z(1)), "m_scale must hold 2"),
                       (dict(eight, v_scale=None), "v_scale must hold"), (dict(t, m_scale=z(2)), "scales belong"),
                       (dict(t, param=z(300, dtype=torch.float64)), "param has dtype"),
                       (dict(t, grad=z(600)[::2]), "contiguous"), (t, "GPU tensor")):
        with pytest.raises(ValueError, match=match):
            svl.AdamwTensors([bad])
    with pytest.raises(ValueError, match="8 and of 32"):
        svl.AdamwTensors([eight, t])
    empty = svl.AdamwTensors([])
    with pytest.raises(ValueError, match="unknown state"):
        svl.svl_adamw_read_state("p", z(3, dtype=torch.uint8), z(1), z(3))
    with pytest.raises(ValueError, match="5 words"):
        svl.svl_adamw_step(svl.make_adamw(1e-3), empty, dev=z(4))
    for make in (lambda: svl.make_embedding(64, 10, table="f64"), lambda: svl.make_norm(64, kind="batch"),
                 lambda: svl.make_lm_head(64, 10, compute="f32")):
        with pytest.raises(ValueError, match="unknown"):
            make()
