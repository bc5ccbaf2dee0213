"""The 64-bit implementation of the attention-based fusion that the GPU tests compare with: identities and differences (CPU)."""
import math

import torch

import fusion_oracle as F


def _rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed + sum(shape)), dtype=torch.float64)


def test_rotation_keeps_lengths_and_relative_positions():
    f = F.frequencies(12)
    for inter in (False, True):
        x, y = _rand(1, 32), _rand(1, 32, seed=1)
        px, py = torch.tensor([1_000_003]), torch.tensor([1_000_010])
        a = F.rotate(x, 2, f, px, interleaved=inter), F.rotate(y, 2, f, py, interleaved=inter)
        b = F.rotate(x, 2, f, px - 1_000_003, interleaved=inter), F.rotate(y, 2, f, py - 1_000_003, interleaved=inter)
        assert torch.allclose((a[0] * a[1]).sum(), (b[0] * b[1]).sum(), atol=1e-8)
        assert torch.allclose(F.rotate(a[0], 2, f, px, interleaved=inter, inverse=True), x, atol=1e-12)
    assert torch.equal(F.frequencies(64, factor=8.0, trained=0.0, low=1.0, high=32.0), F.frequencies(64) / 8)
    scaled = F.frequencies(64, factor=8.0, trained=4096.0)
    assert scaled[0] == 1.0 and torch.isclose(scaled[-1], F.frequencies(64)[-1] / 8)


def test_norm_gradient_against_differences():
    x, w, dy, pos, f = _rand(3, 24), _rand(12), _rand(3, 24, seed=2), torch.tensor([0, 5, -9]), F.frequencies(8)
    loss = lambda x, w: (F.rotate(F.norm(x, 2, w, 1e-3), 2, f, pos, 1.25, True) * dy).sum()
    dx, dw, _, _ = F.norm_rotary_backward(dy, x, 2, w, 1e-3, f, pos, 1.25, True)
    d = 1e-6
    for t, g in ((x, dx), (w, dw)):
        for i in range(t.numel()):
            up, down = t.clone().flatten(), t.clone().flatten()
            up[i] += d
            down[i] -= d
            args = (lambda v: (v.view_as(x), w)) if t is x else (lambda v: (x, v))
            assert abs((loss(*args(up)) - loss(*args(down))) / (2 * d) - g.flatten()[i]) < 1e-7


def test_attention_gradient_against_differences_and_a_dense_form():
    qp, kp = [0, 2, 2, 5, 6], [0, 3, 4, 9, 9]
    mask = torch.tensor([1, 0, 1, 1, 1, 1, 0, 1, 1])
    q, k, v, do = _rand(6, 4 * 8), _rand(9, 2 * 8), _rand(9, 2 * 8, seed=3), _rand(6, 4 * 8, seed=4)
    res = F.attention(q, k, v, qp, kp, 4, 2, 0.3, mask, do)
    assert not res["out"][0][5].any() and res["lse"][0][5].tolist() == [-math.inf] * 4 and not res["dk"][0][1].any()
    assert not res["dk"][0][3].any()                        # a sequence without queries
    sc = (q[2:5].view(3, 4, 8)[:, 3] @ k[4:9].view(5, 2, 8)[:, 1].T * 0.3).masked_fill(mask[4:9] == 0, -math.inf)
    assert torch.allclose(res["out"][0][2:5].view(3, 4, 8)[:, 3], sc.softmax(-1) @ v[4:9].view(5, 2, 8)[:, 1])
    loss = lambda q, k, v: (F.attention(q, k, v, qp, kp, 4, 2, 0.3, mask)["out"][0] * do).sum()
    d = 1e-6
    for n, t in enumerate((q, k, v)):
        g = res[("dq", "dk", "dv")[n]][0].flatten()
        for i in range(0, t.numel(), 3):
            sides = []
            for sign in (1, -1):
                m = t.clone().flatten()
                m[i] += sign * d
                args = [q, k, v]
                args[n] = m.view_as(t)
                sides.append(loss(*args))
            assert abs((sides[0] - sides[1]) / (2 * d) - g[i]) < 1e-7, (n, i)
