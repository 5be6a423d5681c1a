"""Optimizer steps over kept lists of tensors: 8-bit states without a seed of the
caller's own, and tensors that moved behind a list's back."""
import pytest
import torch

import paper_2607_20357_amd as svl

pytestmark = pytest.mark.gpu


def _zeros(n, bits=32):
    z = lambda m, dtype=torch.float32: torch.zeros(m, dtype=dtype, device="cuda")
    t = dict(param=z(n), grad=z(n))
    if bits == 32:
        return dict(t, m=z(n), v=z(n))
    return dict(t, m=z(n, torch.uint8), v=z(n, torch.uint8), m_scale=z(-(-n // 256)), v_scale=z(-(-n // 256)))


def test_small_changes_are_not_lost_without_a_seed():
    """Each step rounds by other bits by itself: a second moment that only decays follows its decay on average."""
    n = 1 << 16
    t = _zeros(n, 8)
    t["v"].fill_(240)
    t["v_scale"].fill_(1.0)
    table = svl.AdamwTensors([t])
    adam = svl.make_adamw(0.0, 0.9, 0.99, state_bits=8)
    for step in range(1, 201):
        svl.svl_adamw_step(adam, table, step=step)
    v = torch.empty(n, device="cuda")
    svl.svl_adamw_read_state("v", t["v"], t["v_scale"], v)
    # the root's mean after 200 steps is 0.99^100; a value's deviation is under 1/8 of it a step, sqrt(200) steps
    # over 65536 values: under 0.7 percent
    assert abs(v.double().sqrt().mean().item() / 0.99 ** 100 - 1) < 0.01


def test_the_seed_of_a_step_is_its_number():
    """Without a seed the bits are those of seed = step; a seed of the caller's counts, 0 too."""
    def run(**kw):
        gen = torch.Generator(device="cuda").manual_seed(3)
        t = _zeros(5000, 8)
        t["grad"].normal_(generator=gen)
        svl.svl_adamw_step(svl.make_adamw(1e-3, state_bits=8), [t], step=(1 << 32) + 7, **kw)
        return t
    free, seven, zero = run(), run(seed=7), run(seed=0)
    assert torch.equal(free["m"], seven["m"]) and torch.equal(free["v"], seven["v"])
    assert not torch.equal(free["m"], zero["m"])


@pytest.mark.parametrize("bits, name", [(32, "param"), (32, "grad"), (32, "m"), (32, "master"), (8, "v"),
                                        (8, "m_scale")])
def test_tensors_that_moved_are_refused(bits, name):
    t = _zeros(1000, bits)
    if name == "master":
        t["master"] = torch.zeros(1000, device="cuda")
    adam, table = svl.make_adamw(1e-3, state_bits=bits), svl.AdamwTensors([_zeros(10, bits), t])
    svl.svl_adamw_step(adam, table, step=1)
    kept = t[name].data
    t[name].data = t[name].data.clone()
    with pytest.raises(ValueError, match=f"{name} of tensor 1 .*moved"):
        svl.svl_adamw_step(adam, table, step=2)
    t[name].data = kept
    svl.svl_adamw_step(adam, table, step=2)
    assert torch.isfinite(t["param"]).all()
