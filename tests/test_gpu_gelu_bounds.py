"""GELU and its derivative over dense fp32 arguments: the bounds that the interface states."""
import math

import pytest
import torch

import paper_1909_05840_b200 as qb

pytestmark = pytest.mark.gpu


def phi(z):
    """Phi with its relative precision in the lower tail (64 bits)."""
    return 0.5 * torch.special.erfc(z * -math.sqrt(0.5))


@pytest.mark.parametrize("width", [1.0, 6.0, 12.0])
def test_stated_bounds(width):
    M, K = 4096, 1024
    g = torch.Generator(device="cuda").manual_seed(int(width))
    saved = (torch.randint(-127, 128, (M, K), device="cuda", generator=g, dtype=torch.int8), torch.rand(M, K // 64, device="cuda", generator=g) * width / 127)
    p = qb.restore(saved, torch.float32).double()
    off = (qb.restore(saved, torch.float32, activation="gelu").double() - p * phi(p)).abs()
    value = (p * phi(p)).abs()
    assert (off <= 4e-7 + 2.0**-23 * value).all()
    lower = (p < 0) & (p >= -5.75)
    assert (off[lower] <= 2.0**-10 * value[lower]).all()
    far = (p < -5.75) & (p > -12)
    assert (off[far] <= 0.03 * value[far]).all() and (value[far] < 3e-8).all()
    slope = phi(p) + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    ones = torch.ones(M, K, device="cuda")
    assert ((qb.gelu_backward(ones, p.float()).double() - slope).abs() <= 4e-7).all()
    assert torch.equal(qb.gelu_backward(ones, saved), qb.gelu_backward(ones, p.float()))
