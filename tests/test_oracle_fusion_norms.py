"""The limits that the bf16 attention's errors are held to in the mean see the mistakes that they are there for: planted in the 64-bit form."""
import pytest
import torch

import fusion_oracle as F

BF16 = torch.bfloat16
U = F.HALF[BF16] / 3 ** 0.5


def rounded(x):
    return x.to(torch.float32).to(BF16).double()


def gradients(q, k, v, g, scale, factor=1.0, stored=False, fitted=False, operand=False):
    """dQ, dK of one head.  factor: all dS times it; stored: D from outputs rounded to bf16; fitted: and what it lacks taken out of dQ; operand:
    dS rounded to bf16."""
    p = torch.softmax(q @ k.T * scale, -1)
    out = p @ v
    d = (g * (rounded(out) if stored else out)).sum(-1, keepdim=True)
    ds = factor * p * (g @ v.T - d)
    dq = (rounded(ds) if operand else ds) @ k
    if fitted:
        dq = dq - ds.sum(-1, keepdim=True) * (p @ k)
    return rounded(dq * scale), rounded((rounded(ds) if operand else ds).T @ q * scale)


def off(got, want):
    return ((got - want).norm() / want.norm()).item()


def test_three_percent_of_ds():
    gen = torch.Generator().manual_seed(1)
    make = lambda n, w: rounded(torch.randn(n, w, generator=gen))
    q, k, v, g = make(300, 64), make(700, 64), make(700, 64), make(300, 64)
    want = gradients(q, k, v, g, 0.125)
    for a, b, steps in zip(gradients(q, k, v, g, 0.125, factor=0.97), want, (2, 3)):
        assert off(a, b) > 1.05 * steps * U


@pytest.mark.parametrize("k_len,hd", [(90, 32), (3001, 64), (5000, 96)])
def test_stored_outputs(k_len, hd):
    gen = torch.Generator().manual_seed(k_len)
    make = lambda n: rounded(torch.randn(n, hd, generator=gen))
    q, g, v, k = make(40), make(40), make(k_len), rounded(1 + 0.125 * torch.randn(k_len, hd, generator=gen))
    p = torch.softmax(q @ k.T * hd ** -0.5, -1)
    ds = p * (g @ v.T - (g * (p @ v)).sum(-1, keepdim=True))
    want = ds @ k * hd ** -0.5
    assert off(gradients(q, k, v, g, hd ** -0.5, stored=True, fitted=True)[0], want) <= 1.05 * U
    assert off(gradients(q, k, v, g, hd ** -0.5, stored=True)[0], want) > 3 * U


@pytest.mark.parametrize("k_len,hd", [(256, 64), (128, 96), (1024, 40)])
def test_one_operand(k_len, hd):
    gen = torch.Generator().manual_seed(hd)
    q, g = torch.zeros(60, hd, dtype=torch.float64), rounded(torch.randn(60, hd, generator=gen))
    v = torch.randint(-1, 2, (k_len, hd), generator=gen).double()
    k = rounded(1 + 0.125 * torch.randn(k_len, hd, generator=gen))
    p = torch.full((60, k_len), 1 / k_len, dtype=torch.float64)
    ds = p * (g @ v.T - (g * (p @ v)).sum(-1, keepdim=True))
    assert off(gradients(q, k, v, g, 1.0)[0], ds @ k) <= 1.05 * U
    assert off(gradients(q, k, v, g, 1.0, operand=True)[0], ds @ k) > 3 * U
