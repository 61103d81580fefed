"""Rows whose mean is far above their deviations: constant ones, and ones a few units of the last place apart."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_checkpoint import half, least

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0**-24
WIDTHS = [1, 7, 56, 664, 768, 1000, 1024, 1025, 2056, 4104, 8192, 9001]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("D", WIDTHS)
def test_constant_rows(D, kind):
    """Every deviation is 0: y is beta to the bit, the mean the value, rstd 1 / sqrt(eps) up to the roundings of eps, of a root and of a quotient;
    and in the backward pass xhat is 0, so that grad_x is rstd (g - mean g) and grad_gamma is 0."""
    t = TYPES[kind]
    values = [127.0, 100.0, 1.984375, -127.0, -1.984375, 0.0, 1e-3, 60000.0, -3e-5, 0.1, 1.0 / 3]
    x = torch.tensor(values, device="cuda").to(t)[:, None].repeat(1, D).contiguous()
    gamma, beta = 1 + torch.rand(D, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = qb.layer_norm(x, gamma, beta, 1e-12, want_stats=True)
    assert torch.equal(y, beta.to(t).expand_as(y)) and torch.equal(mean, x[:, 0].float())
    assert ((rstd.double() - 1e6).abs() <= 1e6 * 4 * U).all()
    assert torch.equal(qb.layer_norm(x, None, None, 1e-12), torch.zeros_like(x))
    z = x.clone()
    assert torch.equal(qb.layer_norm(z, gamma, beta, 1e-12, y=z), y)
    dy = (torch.randn(len(values), D, device="cuda") * 1e-6).to(t)
    ws = torch.zeros(qb.layer_norm_workspace_bytes(*x.shape), dtype=torch.uint8, device="cuda")
    dx, dgamma, dbeta = qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws)
    g = dy.double() * gamma.double()
    want = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    n = (32 if D <= 8192 else D / 256 + 1) + 13
    tol = rstd.double()[:, None] * U * (4 * g.abs() + (n + 5) * g.abs().mean(1, keepdim=True)) * 1.01 + want.abs() * half(t) * 1.01 + least(t)
    assert ((dx.double() - want).abs() <= tol).all() and (dgamma == 0).all() and dbeta.isfinite().all()


@pytest.mark.parametrize("offset", [1.0, -1000.0, 1e5])
@pytest.mark.parametrize("D", WIDTHS[1:])
def test_rows_a_few_units_apart(D, offset):
    """fp32 values some units of the last place around the offset.  Deviations d from the rounded mean are exact, and so is the rest of the
    mean, delta, up to n roundings of the mean |d| (n: the additions of a chain); the mean of squares has n + 2 of itself, and the variance is
    it less delta^2."""
    M, eps = 9, 1e-12
    g = torch.Generator(device="cuda").manual_seed(D)
    steps = torch.randint(-3, 4, (M, D), device="cuda", generator=g, dtype=torch.int32)
    x = (torch.full((M, D), offset, device="cuda").view(torch.int32) + steps).view(torch.float32)
    beta = torch.randn(D, device="cuda", generator=g)
    y, mean, rstd = qb.layer_norm(x, None, beta, eps, want_stats=True)
    x64 = x.double()
    m64 = x64.mean(1, keepdim=True)
    var = (x64 - m64).square().mean(1, keepdim=True)
    r64 = 1 / (var + eps).sqrt()
    xhat = (x64 - m64) * r64
    n = (32 if D <= 8192 else D / 256 + 1) + 13
    m0 = m64.float().double()
    m0 = torch.maximum((m0 - m64).abs(), (torch.nextafter(m64.float(), torch.full_like(m64.float(), float("inf"))).double() - m64).abs())  # either neighbour
    d = (x64 - m64).abs() + m0
    e_delta = (n + 2) * U * d.mean(1, keepdim=True)
    e_var = (n + 4) * U * (d.square().mean(1, keepdim=True) + m0.square()) + 2 * m0 * e_delta
    e_rstd = 0.5 * e_var / (var + eps) + 4 * U
    e_rstd = e_rstd * (1 + 4 * e_rstd)
    tol = r64 * (e_delta + 2 * U * d) + xhat.abs() * (e_rstd + 3 * U) + U * (xhat + beta.double()).abs() + U * beta.abs()
    assert ((y.double() - xhat - beta.double()).abs() <= 1.01 * tol).all()
    assert ((mean.double() - m64[:, 0]).abs() <= (U * m64.abs() + e_delta)[:, 0] * 1.01).all()
    assert ((rstd.double() / r64[:, 0] - 1).abs() <= 1.01 * e_rstd[:, 0]).all()


@pytest.mark.parametrize("D", [8, 768, 3000, 9000])
def test_first_element_far_out(D):
    """What is taken off before the first sum may be any of the row's elements, its largest too: the deviations have the last word."""
    x = torch.randn(6, D, device="cuda")
    x[:, 0] = torch.tensor([1e4, -1e4, 3e6, 1e-3, -50.0, 7.0], device="cuda")
    y, mean, rstd = qb.layer_norm(x, None, None, 1e-12, want_stats=True)
    x64 = x.double()
    m64 = x64.mean(1, keepdim=True)
    r64 = 1 / ((x64 - m64).square().mean(1, keepdim=True) + 1e-12).sqrt()
    n = (32 if D <= 8192 else D / 256 + 1) + 13
    e_mean = (n + 3) * U * ((x64 - m64).abs().mean(1, keepdim=True) + m64.abs())
    e_rstd = (n + 6) * U + (e_mean * r64) ** 2
    xhat = (x64 - m64) * r64
    assert ((y.double() - xhat).abs() <= 1.01 * (r64 * e_mean + xhat.abs() * (e_rstd + 4 * U))).all()
    assert ((mean.double() - m64[:, 0]).abs() <= 1.01 * e_mean[:, 0]).all()
    assert ((rstd.double() / r64[:, 0] - 1).abs() <= 1.01 * e_rstd[:, 0]).all()
