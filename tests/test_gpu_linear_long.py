"""Linears over long contractions with 16-bit outputs: sums in several runs, whatever the workspace has room for and whatever is saved."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_checkpoint import half, slope64, values64

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
LONG = {"bf16": 65536 + 72, "fp16": 16384 + 72}  # just beyond one run
# without room for parts these meet every form: tiles of 128 x 64, 128 x 128, 256 x 128 and 256 x 256, and halves
SIZES = [(1, 8), (33, 72), (40, 1032), (100, 17928), (1100, 1160), (2600, 2056)]


@pytest.fixture(scope="module")
def ws():
    return torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")  # (rows of 1,100 elements are copied)


def whole(seed, *shapes, t):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(-2, 3, s, device="cuda", generator=g).to(t) for s in shapes]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("room", ["parts", "none"])
@pytest.mark.parametrize("M,N", SIZES)
def test_whole_numbers(M, N, room, kind, ws):
    """Small whole numbers, whose sums (below 2^24) are exact in any order: equal to the bit in every form, and what is saved too (codes: half a
    step, and what the 32-bit quotient is off by, 127 * 2^-22 of a step)."""
    t, K = TYPES[kind], LONG[kind]
    ws = ws if room == "parts" else ws[:1024]
    x, w = whole(M + N, (M, K), (N, K), t=t)
    r = torch.randint(-9, 10, (M, N), device="cuda").to(t)
    bias = torch.randint(-3, 4, (N,), device="cuda").float()
    product = x.float() @ w.float().t()
    z = product.double() + bias.double()
    assert torch.equal(qb.linear(x, w, None, ws, out_dtype=torch.float32), product)
    assert torch.equal(qb.linear(x, w, bias, ws), z.to(t))
    assert torch.equal(qb.linear(x, w, bias, ws, residual=r), (z + r.double()).to(t))
    y, pre = qb.linear(x, w, bias, ws, residual=r, save="pre")
    assert torch.equal(y, (z + r.double()).to(t)) and torch.equal(pre, z.to(t))
    y, saved = qb.linear(x, w, bias, ws, residual=r, save="codes")
    step = saved[1].double().repeat_interleave(64, 1)[:, :N]
    assert torch.equal(y, (z + r.double()).to(t)) and ((values64(*saved) - z).abs() <= step * (0.5 + 2.0**-14)).all()
    g = qb.linear(x, w, bias, ws, activation="gelu")
    want = z * torch.special.ndtr(z)
    assert ((g.double() - want).abs() <= 5e-7 + want.abs() * (half(t) + 2.0**-23)).all()
    # the same sums as a gradient of an input, and as one of weights
    wt = w.t().contiguous()  # [K][N]: a linear of N inputs and K outputs
    assert torch.equal(qb.linear_grad_x(x, wt, ws), product.to(t))
    p = torch.randn(M, N, device="cuda").to(t)
    slope = slope64(p.double()) * product.double()
    assert ((qb.linear_grad_x(x, wt, ws, through=p).double() - slope).abs() <= product.double().abs() * 5e-7 + slope.abs() * (half(t) + 2.0**-23) + 2.0**-25).all()
    xt = x.t().contiguous()
    if M % 8 == 0 or room == "parts":
        dw, _ = qb.linear_grad_w(xt, wt, ws, out_dtype=t, needs=(True, False))
        assert torch.equal(dw, product.to(t))
    assert qb.read_status(ws) == qb.QB_OK


def test_forms_that_are_covered():
    forms = [qb.linear_form(M, N, K, 1024) for M, N in SIZES for K in LONG.values()]
    assert {f[:2] for f in forms} == {(128, 64), (128, 128), (256, 128), (256, 256)} and any(f[2] > 0 for f in forms) and all(f[3] == 1 for f in forms)
    assert qb.linear_form(33, 72, LONG["bf16"], 1 << 28)[3] > 1


@pytest.mark.parametrize("save", [None, "pre", "codes"])
@pytest.mark.parametrize("room", ["parts", "none"])
@pytest.mark.parametrize("kind,K", [("fp16", 1 << 20), ("bf16", 1 << 22)])
def test_sums_of_many_products(kind, K, room, save, ws):
    """Products of random signs.  A run is of 8,192 products at most, 512 additions that cut 2^-23 of the accumulator off: 2^-14 of the result's
    norm; the type's rounding is eps / 2 of a value at most.  (One chain of K / 16 additions would be off by K 2^-28 or more: 4e-3 and 1.6e-2.)"""
    t = TYPES[kind]
    ws = ws if room == "parts" else ws[:1024]
    g = torch.Generator(device="cuda").manual_seed(K)
    x, w = (torch.randn(n, K, device="cuda", generator=g).to(t) * 2.0**-10 for n in (40, 64))
    z = torch.zeros(40, 64, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 17):
        z += x[:, k:k + (1 << 17)].double() @ w[:, k:k + (1 << 17)].double().t()
    bound = half(t) + 2.0**-13

    def off(y):
        return float((y.double() - z).norm() / z.norm())
    out = qb.linear(x, w, None, ws, save=save)
    assert off(out if save is None else out[0]) <= bound
    if save == "pre":
        assert off(out[1]) <= bound
    if save == "codes":  # half a step of each value, and the sums' error
        step = out[1][1].double().repeat_interleave(64, 1)[:, :64]
        assert ((values64(*out[1]) - z).norm() - (step * 0.5).norm()) / z.norm() <= 2.0**-13
    if save is None:
        assert off(qb.linear_grad_x(x, w.t().contiguous(), ws)) <= bound
        assert off(qb.linear_grad_w(x.t().contiguous(), w.t().contiguous(), ws, out_dtype=t, needs=(True, False))[0]) <= bound
