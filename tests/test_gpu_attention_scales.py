"""Windowed attention and its gradient where scores span many powers of two, against
the float64 oracle."""
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
