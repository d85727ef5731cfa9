"""Moments without a gradient: what thousands of steps leave of them.

An fp32 moment takes one fp32 rounding a step.  The largest entry of a block of 8-bit moments
takes three, of the decay, of its scale and of its value, each at most 2^-24 of the value and to
either side; over T steps they add up like independent numbers, six standard deviations of
which are 6 sqrt(3 T) 2^-24 / sqrt(3).  Its scale's factor, the float 1 / 1.875, is too large by D
of itself, which adds T D.  An entry whose quotient is rounded to just below its own code drops
to the next where its 16 random bits are zero: in 2000 steps that happens in at most
2000 / 65536 = 3% of the blocks, so nine in ten are held to the bound."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("state", ["f32", "block8"])
def test_largest_entries_decay_with_the_stated_drift(state):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as M
    blocks, steps = 512, 2000
    b1, b2 = float(np.float32(0.99)), float(np.float32(0.999))
    n = blocks * 256
    rng = np.random.default_rng(1)
    g = torch.tensor(rng.standard_normal(n) * np.repeat(10.0 ** rng.uniform(-3, 3, blocks), 256), dtype=torch.float32).cuda()
    opt = M.AdamWGroup(0.99, 0.999, 1e-8, seed=5)
    opt.add(torch.zeros(n, device="cuda"), state=state)
    opt.step([g], 1, 0.0)
    first = [x[0].double().view(blocks, 256) for x in opt.moments()]
    zero = torch.zeros(n, device="cuda")
    for t in range(2, steps + 2):
        opt.step([zero], t, 0.0)
    last = [x[0].double().view(blocks, 256) for x in opt.moments()]
    bound = 6 * np.sqrt(3 * steps) * 2.0 ** -24 / np.sqrt(3)
    drift = steps * (float(np.float32(1 / 1.875)) * 1.875 - 1) if state == "block8" else 0.0
    for x, y, b in zip(first, last, (b1, b2)):
        at = x.abs().argmax(1, keepdim=True)
        ratio = y.gather(1, at) / x.gather(1, at) / b ** steps
        assert ((ratio - 1 - drift).abs() <= bound).double().mean().item() >= (0.9 if state == "block8" else 1.0)
    opt.close()
