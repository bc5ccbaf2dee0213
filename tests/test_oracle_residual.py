"""The 64-bit forms of dropout and layer norm: the generator's known answers, gradients against differences, the mask's statistics."""
import os

import numpy as np
import torch

import residual_oracle as R


def test_philox_known_answers():
    path = os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.txt")
    rows = [[int(x, 16) for x in line.split()[-10:]] for line in open(path) if line.strip() and not line.startswith("#")]
    assert rows
    for v in rows:
        assert [int(x) for x in R.philox(v[:4], v[4:6])] == v[6:]


def test_the_mask_keeps_the_share_and_differs_by_plan():
    f = R.factors(2000, 64, 0.3, 77)
    share = (f == 0).double().mean().item()
    assert abs(share - R.cut(0.3) / 65536) < 5 * (0.21 / f.numel()) ** 0.5
    assert abs(f.mean().item() - 1) < 5 * (0.3 / 0.7 / f.numel()) ** 0.5
    for other in (dict(seed=78), dict(seed=77 + (1 << 32)), dict(place=1), dict(step=1)):
        g = R.factors(2000, 64, 0.3, **{**dict(seed=77), **other})
        both = ((f == 0) & (g == 0)).double().mean().item()
        assert abs(both - share * share) < 0.01
    assert torch.equal(R.factors(50, 36, 0.3, 77), f[:50, :36])          # an element's mask goes by its place alone
    assert (R.factors(9, 16, 0.0, 1) == 1).all() and R.cut(0.9999999) == 65535


def test_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x, r, dy, dz, gain, shift = rnd(5, 12), rnd(5, 12), rnd(5, 12), rnd(5, 12), 1 + 0.3 * rnd(12), rnd(12)
    f = R.factors(5, 12, 0.4, 9)

    def loss(x, r, gain, shift):
        res = R.norm(x, r, f, gain, shift, 1e-5, torch.float32)
        return (res["y"][0] * dy).sum() + (res["z"][0] * dz).sum()

    got = R.norm(x, r, f, gain, shift, 1e-5, torch.float32, dy, dz)
    args = [x, r, gain, shift]
    for i, name in enumerate(("dx", "dr", "dgain", "dshift")):
        grad = torch.zeros_like(args[i])
        for at in np.ndindex(*args[i].shape):
            ends = []
            for step in (1e-6, -1e-6):
                moved = [a.clone() for a in args]
                moved[i][at] += step
                ends.append(loss(*moved))
            grad[at] = (ends[0] - ends[1]) / 2e-6
        assert (got[name][0] - grad).abs().max() < 1e-6, name


def test_bounds_are_not_wide():
    """What a bound allows is some hundreds of roundings of 32 bits, and in 16 bits little more than the last one."""
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(64, 256, generator=gen, dtype=torch.float64)
    for dtype in (torch.float32, torch.bfloat16):
        res = R.norm(x, None, torch.ones_like(x), None, None, 1e-5, dtype, x.flip(0))
        for name in ("y", "dx", "dgain"):
            value, bound = res[name]
            steps = (bound.median() / value.square().mean().sqrt()).item()
            assert steps < (2 * R.HALF[dtype] if dtype == torch.bfloat16 and name != "dgain" else 2000 * R.E), (name, dtype, steps)
