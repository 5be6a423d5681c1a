"""Host-side checks of the windowed attention and of the 4-bit cache (no GPU): the
exports, sizes, and every refusal, through the C ABI with pointers that are never
followed and through the binding."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2607_20357_amd as svl
from paper_2607_20357_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 16 * 4096
CALLS = ["append", "read", "cached", "window", "backward"]


def test_exports():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "svl.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(svl_(?:kv4|window)_[a-z0-9_]+)\s*\(", text))
    assert names == {"svl_kv4_cache_bytes", "svl_kv4_append", "svl_kv4_read", "svl_kv4_workspace_bytes",
                     "svl_kv4_attention", "svl_window_attention", "svl_window_workspace_bytes",
                     "svl_window_attention_backward"}
    for n in names | {"svl_cache4_bytes", "svl_prefill_cache4", "svl_decode_step4"}:
        assert hasattr(svl.load_library(), n) and hasattr(svl, n)
    assert hasattr(svl.load_library(), "svl_decode4_workspace_bytes")


def test_cache_bytes():
    """Tiles of 16 positions of 18 head_dim bytes: 4.5 bits a value."""
    for d in (64, 128):
        for length in (1, 16, 17, 1000, 1 << 20):
            att = svl.make_attention(8, 2, d)
            assert svl.svl_kv4_cache_bytes(att, 3, length) == 3 * 2 * -(-length // 16) * 18 * d
    for args in ((0, 5), (2, 0), (2, (1 << 20) + 1)):
        with pytest.raises(svl.SvlError, match="out of range"):
            svl.svl_kv4_cache_bytes(svl.make_attention(8, 2, 128), *args)
    with pytest.raises(svl.SvlError, match="head_dim"):
        svl.svl_kv4_cache_bytes(svl.make_attention(8, 2, 96), 1, 5)


def _call(name, att, cu=(0, 3, 5), pos=(4, 0), cu_k=(0, 9, 12), max_len=64, ld=None, null=None, shift=None,
          ws_bytes=1 << 40, batch=None):
    """The C call with made-up device pointers; null / shift name an argument to be NULL / off by 8."""
    lib, P = svl.load_library(), ctypes.c_void_p
    cu, pos, cu_k = (None if x is None else np.asarray(x, np.int32) for x in (cu, pos, cu_k))
    host = lambda a, n: None if a is None or null == n else a.ctypes.data_as(P)
    dev = lambda n: None if null == n else P(PTR + (8 if shift == n else 0))
    a = None if null == "att" else ctypes.byref(att)
    B = len(cu) - 1 if batch is None else batch
    lq, lk = (att.n_heads * att.head_dim, att.n_kv_heads * att.head_dim) if ld is None else (ld, ld)
    c, p, ck = host(cu, "cu"), host(pos, "pos"), host(cu_k, "cu_k")
    if name == "append":
        return lib.svl_kv4_append(a, B, c, p, dev("k"), lk, dev("v"), lk, dev("cache"), max_len, None)
    if name == "read":
        return lib.svl_kv4_read(a, B, c, p, dev("cache"), max_len, dev("k"), lk, dev("v"), lk, None)
    if name == "cached":
        return lib.svl_kv4_attention(a, B, c, p, dev("q"), lq, dev("cache"), max_len, dev("out"), lq, dev("ws"),
                                     ws_bytes, None)
    if name == "window":
        return lib.svl_window_attention(a, B, c, ck, dev("q"), lq, dev("k"), lk, dev("v"), lk, None, dev("out"),
                                        lq, None, None)
    return lib.svl_window_attention_backward(
        a, B, c, ck, dev("q"), lq, dev("k"), lk, dev("v"), lk, None, dev("out"), lq, dev("lse"),
        dev("grad_out"), lq, dev("grad_q"), lq, dev("grad_k"), lk, dev("grad_v"), lk, dev("ws"), ws_bytes, None)


def _refused(status, code, words):
    assert binding.STATUS[status] == code, (binding.STATUS[status], svl.load_library().svl_last_error())
    assert words in svl.load_library().svl_last_error().decode()


@pytest.mark.parametrize("name", CALLS)
def test_descriptions_are_refused(name):
    good = dict(n_heads=8, n_kv_heads=2, head_dim=128)
    for change, code, words in (
            (dict(n_heads=7), "SVL_E_SHAPE", "multiple of n_kv_heads"), (dict(n_heads=0), "SVL_E_SHAPE", "positive"),
            (dict(n_kv_heads=-1), "SVL_E_SHAPE", "positive"), (dict(head_dim=96), "SVL_E_SHAPE", "64 or 128"),
            (dict(n_heads=1024), "SVL_E_SHAPE", "65536"), (dict(window=-1), "SVL_E_VALUE", "window"),
            (dict(sinks=-2), "SVL_E_VALUE", "sinks"), (dict(scale=0.0), "SVL_E_VALUE", "scale"),
            (dict(scale=float("nan")), "SVL_E_VALUE", "scale"), (dict(scale=float("inf")), "SVL_E_VALUE", "scale"),
            (dict(scale=-1.0), "SVL_E_VALUE", "scale")):
        _refused(_call(name, svl.make_attention(**{**good, **change})), code, words)
    att = svl.make_attention(**good)
    att.compute = 2
    _refused(_call(name, att), "SVL_E_DTYPE", "compute")
    _refused(_call(name, att, null="att"), "SVL_E_NULL", "description")
    with pytest.raises(ValueError, match="compute"):
        svl.make_attention(8, 2, 128, compute="f32")


@pytest.mark.parametrize("name", CALLS)
def test_rows_and_arrays_are_refused(name):
    att = svl.make_attention(8, 2, 128)
    what = "cu_rows" if name in ("append", "read", "cached") else "cu_q"
    _refused(_call(name, att, cu=(0, 3, 2)), "SVL_E_VALUE", f"{what} decreases at 2")
    _refused(_call(name, att, cu=(-1, 3, 4)), "SVL_E_VALUE", "negative")
    _refused(_call(name, att, null="cu"), "SVL_E_NULL", what)
    _refused(_call(name, att, batch=0), "SVL_E_SHAPE", "batch")
    arrays = {"append": "k v cache", "read": "k v cache", "cached": "q out cache ws", "window": "q k v out",
              "backward": "q k v out grad_out grad_q grad_k grad_v ws"}[name].split()
    for a in arrays:
        _refused(_call(name, att, null=a), "SVL_E_NULL", "workspace" if a == "ws" else a)
        _refused(_call(name, att, shift=a), "SVL_E_ALIGN", "workspace" if a == "ws" else a)
    _refused(_call(name, att, ld=248), "SVL_E_SHAPE", "row stride")
    _refused(_call(name, att, ld=2044), "SVL_E_SHAPE", "row stride")
    if name == "backward":
        _refused(_call(name, att, null="lse"), "SVL_E_NULL", "lse")


@pytest.mark.parametrize("name", ["append", "read", "cached"])
def test_positions_are_refused(name):
    att = svl.make_attention(8, 2, 128)
    _refused(_call(name, att, pos=(62, 0)), "SVL_E_VALUE", "sample 0")
    _refused(_call(name, att, pos=(0, 63)), "SVL_E_VALUE", "sample 1")
    _refused(_call(name, att, pos=(0, -1)), "SVL_E_VALUE", "sample 1")
    _refused(_call(name, att, pos=(2 ** 31 - 1, 0)), "SVL_E_VALUE", "sample 0")
    _refused(_call(name, att, null="pos"), "SVL_E_NULL", "pos")
    _refused(_call(name, att, max_len=0), "SVL_E_SHAPE", "max_len")
    _refused(_call(name, att, max_len=(1 << 20) + 1), "SVL_E_SHAPE", "max_len")
    if name == "cached":
        need = svl.svl_kv4_workspace_bytes(att)
        _refused(_call(name, att, ws_bytes=need - 1), "SVL_E_WORKSPACE", str(need))


@pytest.mark.parametrize("name", ["window", "backward"])
def test_keys_are_refused(name):
    att = svl.make_attention(8, 2, 128)
    _refused(_call(name, att, cu_k=(0, 2, 9)), "SVL_E_VALUE", "sample 0 has 3 queries for 2 keys")
    _refused(_call(name, att, cu_k=(0, 9, 8)), "SVL_E_VALUE", "cu_k decreases")
    _refused(_call(name, att, cu_k=(0, 9, (1 << 30) + 1)), "SVL_E_SHAPE", "too many")
    if name == "backward":
        need = svl.svl_window_workspace_bytes(att, [0, 3, 5], [0, 9, 12])
        _refused(_call(name, att, ws_bytes=need - 1), "SVL_E_WORKSPACE", str(need))
        with pytest.raises(svl.SvlError, match="2 keys"):
            svl.svl_window_workspace_bytes(att, [0, 3], [0, 2])


@pytest.mark.parametrize("name", CALLS)
def test_nothing_to_do(name):
    """Samples without rows: done, and no launch (there is no GPU here)."""
    att = svl.make_attention(8, 2, 128)
    assert _call(name, att, cu=(0, 0, 0), cu_k=(0, 0, 0), null="q") == 0


def test_backward_workspace_follows_the_lengths():
    """Log-sum sized rows, and the partial blocks of a bounded number of pieces."""
    block = 2 * 128 * 128 * 4
    for heads, lengths, window, sinks in (((8, 2), [100], 0, 0), ((32, 32), [640, 577], 0, 0),
                                          ((32, 8), [32768], 64, 4), ((40, 40), [1] * 200, 0, 0),
                                          ((32, 32), [20000] * 3, 1, 300)):
        att = svl.make_attention(*heads, 128, window=window, sinks=sinks)
        cu = np.concatenate([[0], np.cumsum(lengths)])
        n = svl.svl_window_workspace_bytes(att, cu)
        assert n >= 2 * 4 * int(cu[-1]) * heads[0]
        assert n <= 2 * 4 * int(cu[-1]) * heads[0] + 2048 + 4 * 512 * block


# ------------------------------------------------------------------ the binding
def _rows(n, heads, d, dtype=torch.float16):
    return torch.zeros(n, heads, d, dtype=dtype)


def test_binding_refuses_arrays_that_do_not_fit():
    att = svl.make_attention(8, 2, 64)
    cache = torch.zeros(svl.svl_kv4_cache_bytes(att, 1, 32), dtype=torch.uint8)
    k, v, q = _rows(5, 2, 64), _rows(5, 2, 64), _rows(5, 8, 64)
    app = lambda **kw: svl.svl_kv4_append(att, **{**dict(cu_rows=[0, 5], pos=[0], k=k, v=v, cache=cache, max_len=32), **kw})
    for kw, words in ((dict(k=k.bfloat16()), "dtype"), (dict(v=_rows(4, 2, 64)), "4 rows"),
                      (dict(k=_rows(5, 3, 64)), "shape"), (dict(k=_rows(5, 2, 128)), "shape"), (dict(v=k[0]), "shape"),
                      (dict(k=_rows(5, 64, 2).transpose(1, 2)), "contiguous"), (dict(v=_rows(5, 4, 64)[:, ::2]), "contiguous"),
                      (dict(k=torch.zeros(5, 2 * 64 + 4, dtype=torch.float16)[:, :128].unflatten(1, (2, 64))), "row stride"),
                      (dict(v=k[:1].expand(5, 2, 64)), "row stride"), (dict(k=None), "torch tensor"),
                      (dict(cache=cache[:-1]), "cache"), (dict(cache=cache.to(torch.int8)), "dtype"),
                      (dict(pos=[0, 1]), "pos"), (dict(cu_rows=[5]), "cu_rows"), (dict(cu_rows=[[0, 5]]), "cu_rows"),
                      ({}, "must be a GPU tensor")):
        with pytest.raises(ValueError, match=words):
            app(**kw)
    win = lambda **kw: svl.svl_window_attention(att, **{**dict(cu_q=[0, 5], cu_k=None, q=q, k=k, v=v, out=q.clone()), **kw})
    for kw, words in ((dict(out=k), "shape"), (dict(cu_k=[0, 3, 5]), "entries"), (dict(cu_k=[0, 6]), "5 rows"),
                      (dict(q=q.float()), "dtype"), ({}, "must be a GPU tensor")):
        with pytest.raises(ValueError, match=words):
            win(**kw)
    # checks that do not come to a device pointer first
    with pytest.raises(ValueError, match="float32"):
        binding._log_sums(torch.zeros(5, 8, dtype=torch.float64), att, 5)
    with pytest.raises(ValueError, match="shape"):
        binding._log_sums(torch.zeros(8, 8).reshape(16, 4), att, 5)
    with pytest.raises(ValueError, match="needs at least 5"):
        binding._mask(torch.ones(4, dtype=torch.bool), 5)
    with pytest.raises(ValueError, match="dtype"):
        binding._mask(torch.ones(5), 5)
    with pytest.raises(ValueError, match="lse is required"):
        svl.svl_window_attention_backward(att, [0, 5], None, q, k, v, q, None, q, q, k, v, cache)
