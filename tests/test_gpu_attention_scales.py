"""Windowed attention, its gradient and the cached attention where scores or the cache's
scales span many powers of two."""
import pytest
import torch

import paper_2607_20357_amd as svl
from attention_helpers import check_window, draw, offsets, run_window

pytestmark = pytest.mark.gpu
COMPUTES = ["f16", "bf16"]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ------------------------------------------------------------------ query gradient
@pytest.mark.parametrize("compute", COMPUTES)
@pytest.mark.parametrize("heads,n,window,sinks", [((1, 1, 128), [577], 0, 0), ((4, 2, 64), [300, 161, 700], 0, 0),
                                                  ((2, 1, 128), [429, 170], 400, 5)])
def test_gradients_under_large_scores(heads, n, window, sinks, compute):
    """Scores of deviation 9: a sample's first row scores later keys, which it does not
    see, far above its log-sum.  Lengths end inside a wave's 32 rows."""
    A, H, d = heads
    att = svl.make_attention(*heads, window=window, sinks=sinks, compute=compute)
    for seed in range(3):
        gen, cu = _gen(seed), offsets(n)
        q, k = (draw(gen, (int(cu[-1]), h, d), compute, 3.0) for h in (A, H))
        v, grad = (draw(gen, (int(cu[-1]), h, d), compute) for h in (H, A))
        got = run_window(att, cu, cu, q, k, v, None, grad)
        check_window(att, compute, cu, cu, q, k, v, got, None, grad)


# ------------------------------------------------------------------ cached attention
@pytest.mark.parametrize("compute", COMPUTES)
def test_what_the_window_hides_may_hold_anything(compute):
    """Positions before the window that were never appended: the bytes under them, read as
    scales, are zeros or near the type's largest value."""
    A, H, d, max_len = 4, 2, 128, 700
    for window, sinks, rows, pos in ((20, 0, 1, 600), (20, 3, 1, 661), (50, 0, 5, 450), (9, 2, 30, 641)):
        att = svl.make_attention(A, H, d, window=window, sinks=sinks, compute=compute)
        gen, first = _gen(window), pos - window + 1
        m = pos + rows - first
        k, v = (draw(gen, (m, H, d), compute, 0.01) for _ in range(2))
        q = draw(gen, (rows, A, d), compute, 100.0)
        outs = []
        for byte in (0x00, 0x7b):
            cache = svl.alloc_kv4_cache(att, 1, max_len)
            cache.fill_(byte)
            svl.svl_kv4_append(att, [0, m], [first], k, v, cache, max_len)
            if sinks:
                svl.svl_kv4_append(att, [0, sinks], [0], k[:sinks], v[:sinks], cache, max_len)
            out = torch.full_like(q, float("nan"))
            svl.svl_kv4_attention(att, [0, rows], [pos], q, cache, max_len, out, svl.alloc_kv4_workspace(att))
            outs.append(out)
        assert torch.isfinite(outs[0]).all()
        assert torch.equal(outs[0], outs[1]), (window, sinks, rows)
