"""Activations in 8 bits: codes against 64 bits value for value, what is restored from them, GELU and its gradient."""
import math

import pytest
import torch

import paper_1909_05840_b200 as qb

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# GELU and its derivative by themselves: an absolute part (the fit's 1.7e-7 and the roundings of its terms, which are below 2), a
# relative one where the value itself is rounded, and what is far out (below -5.75 the value is less than 3e-8)
GELU_ABS, SLOPE_ABS = 5e-7, 5e-7


def half(t):
    return torch.finfo(t).eps / 2


def least(t):
    return 2.0**-25 if t == torch.float16 else 2.0**-133 if t == torch.bfloat16 else 2.0**-149


def codes64(x):
    """Codes and scales (64 bits) by the definition."""
    M, K = x.shape
    blocks = (K + 63) // 64
    v = torch.zeros(M, blocks * 64, dtype=torch.float64, device="cuda")
    v[:, :K] = x.double()
    v = v.view(M, blocks, 64)
    top = v.abs().amax(2, keepdim=True)
    some = top >= 2.0**-100
    codes = torch.where(some, torch.round(v * 127 / torch.where(some, top, 1.0)), 0.0)
    return codes.view(M, -1)[:, :K].to(torch.int8), torch.where(some, top / 127, 1.0)[:, :, 0]


def values64(codes, scales):
    return codes.double() * scales.double().repeat_interleave(64, 1)[:, :codes.shape[1]]


def gelu64(z):
    return z * torch.special.ndtr(z)


def slope64(z):
    return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def data(M, K, t, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, device="cuda", generator=g) * torch.exp(2 * torch.randn(M, 1, device="cuda", generator=g))
    x[:, K // 3] *= 20
    return x.to(t)


SIZES = [(1, 1), (2, 7), (3, 8), (1, 63), (5, 64), (4, 65), (7, 72), (33, 100), (1, 768), (77, 768), (129, 1023), (613, 1024), (50, 4097), (3001, 130)]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,K", SIZES)
def test_codes_and_values(M, K, kind):
    t = TYPES[kind]
    x = data(M, K, t, M + K)
    room = torch.full((M * K + 64,), 99, dtype=torch.int8, device="cuda")
    codes, scales = qb.checkpoint(x, codes=room[:M * K].view(M, K))
    want, s64 = codes64(x)
    assert torch.equal(codes, want) and (room[M * K:] == 99).all()
    assert ((scales.double() - s64).abs() <= 2.0**-24 * s64).all()
    p = values64(codes, scales)
    for out in TYPES.values():
        room = torch.full((M * K + 64,), 7.0, dtype=out, device="cuda")
        y = qb.restore((codes, scales), out, y=room[:M * K].view(M, K))
        assert ((y.double() - p).abs() <= p.abs() * (2.0**-24 + half(out)) * 1.01 + least(out)).all() and (room[M * K:] == 7.0).all()
        y = qb.restore((codes, scales), out, activation="gelu").double()
        w = gelu64(p)
        assert ((y - w).abs() <= GELU_ABS + p.abs() * 2.0**-23 + w.abs() * half(out) * 1.01 + least(out)).all()
    # a value restores within half a step, and a little of the scale's rounding
    assert ((p - x.double()).abs() <= (0.5 + 127 * 2.0**-24) * scales.double().repeat_interleave(64, 1)[:, :K]).all()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,K", SIZES)
def test_gelu_backward(M, K, kind):
    t = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(K)
    p, dy = (2 * torch.randn(M, K, device="cuda", generator=g)).to(t), torch.randn(M, K, device="cuda", generator=g).to(t)

    def check(dx, q):
        want = dy.double() * slope64(q)
        # the restored value's rounding moves the slope by 0.8 of it at most
        tol = dy.double().abs() * (SLOPE_ABS + 2.0**-24 * q.abs()) + want.abs() * (2.0**-24 + half(t)) * 1.01 + least(t)
        assert ((dx.double() - want).abs() <= tol).all()
    dx = qb.gelu_backward(dy, p)
    check(dx, p.double())
    saved = qb.checkpoint(p)
    check(qb.gelu_backward(dy, saved), values64(*saved))
    z = dy.clone()
    assert qb.gelu_backward(z, p, grad_x=z) is z and torch.equal(z, dx)
    z = p.clone()
    assert torch.equal(qb.gelu_backward(dy, z, grad_x=z), dx)


def test_gelu_over_the_line():
    """All bfloat16 numbers, in fp32: the bounds of the fit over the whole line, limits and NaN."""
    x = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    dy = torch.ones_like(x)
    slope = qb.gelu_backward(dy[None], x[None])[0]
    assert slope[x.isnan()].isnan().all()
    real = ~x.isnan()
    xr, s = x[real].double(), slope[real].double()
    want = torch.where(xr.isinf(), (xr > 0).double(), slope64(xr.clamp(-1e4, 1e4)))
    assert ((s - want).abs() <= SLOPE_ABS).all()


@pytest.mark.parametrize("K", [64, 100, 768, 1025])
def test_borders_of_codes(K):
    """Values on and next to the border of two codes, where 32 bits cannot tell: (2 k + 1) a / 254 and its neighbours."""
    g = torch.Generator(device="cuda").manual_seed(K)
    M = 512
    top = torch.rand(M, 1, device="cuda", generator=g, dtype=torch.float64).float() + 0.5
    top[:64] = 127.0 / 128  # here the borders are numbers themselves
    k = torch.randint(0, 127, (M, K), device="cuda", generator=g)
    x = ((2 * k + 1).double() * top.double() / 254).float()
    step = torch.randint(-1, 2, (M, K), device="cuda", generator=g, dtype=torch.int32)
    x = (x.view(torch.int32) + step).view(torch.float32) * (1 - 2 * torch.randint(0, 2, (M, K), device="cuda", generator=g))
    x = torch.minimum(torch.maximum(x, -top), top)
    x[:, ::64] = top
    codes, scales = qb.checkpoint(x)
    want, _ = codes64(x)
    assert torch.equal(codes, want)


def test_zeros_tiny_and_not_finite():
    x = torch.randn(8, 200, device="cuda")
    x[0] = 0.0
    x[1] = 2.0**-101 * torch.sign(x[1])
    x[2] *= 2.0**-90
    x[3, 70] = float("inf")
    x[4, 199] = float("nan")
    x[5, 3] = -float("inf")
    x[6] *= 1e37
    codes, scales = qb.checkpoint(x)
    assert (codes[:2] == 0).all() and (scales[:2] == 1).all()
    y = qb.restore((codes, scales), torch.float32)
    assert (y[:2] == 0).all()
    for row, block in ((3, 1), (4, 3), (5, 0)):
        here = torch.arange(200, device="cuda") // 64 == block
        assert y[row, here].isnan().all() and y[row, ~here].isfinite().all()
        dx = qb.gelu_backward(torch.ones(8, 200, device="cuda"), (codes, scales))
        assert dx[row, here].isnan().all() and dx[row, ~here].isfinite().all()
    fine = torch.tensor([2, 6, 7], device="cuda")
    want, _ = codes64(x[fine])
    assert torch.equal(codes[fine], want) and y[fine].isfinite().all()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("K", [64, 100, 1023])
def test_whole_range_of_a_type(K, kind):
    """Blocks at every size that the type has, from its least normal number (fp32, bfloat16: from 2^-99) to its largest, with exact halves."""
    t, M = TYPES[kind], 300
    f = torch.finfo(t)
    low = max(f.smallest_normal, 2.0**-99)
    g = torch.Generator(device="cuda").manual_seed(K)
    size = torch.exp2(torch.linspace(torch.log2(torch.tensor(low)).item() + 1, torch.log2(torch.tensor(f.max)).item(), M, dtype=torch.float64)).cuda()[:, None]
    x = (torch.rand(M, K, device="cuda", generator=g, dtype=torch.float64) * 2 - 1) * size
    x[:, ::64] = size
    x[:, 1::5] = size.to(t).double() / 2
    x = x.clamp(-f.max, f.max).to(t)
    codes, scales = qb.checkpoint(x)
    want, _ = codes64(x)
    assert torch.equal(codes, want)
    assert qb.restore((codes, scales), torch.float32).isfinite().all()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("shift", [1, 3])
def test_any_alignment(kind, shift):
    t, M, K = TYPES[kind], 37, 192
    x = data(M, K, t, 5)
    dy = torch.randn(M, K, device="cuda").to(t)

    def moved(v):
        b = torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")
        b[shift:shift + v.numel()] = v.reshape(-1)
        return b[shift:shift + v.numel()].view(v.shape)
    codes, scales = qb.checkpoint(x)
    c2, s2 = qb.checkpoint(moved(x), scales=moved(scales))
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    assert torch.equal(qb.restore((codes, s2), t, y=moved(x)), qb.restore((codes, scales), t))
    assert torch.equal(qb.gelu_backward(moved(dy), moved(x), grad_x=moved(x)), qb.gelu_backward(dy, x))
    assert torch.equal(qb.gelu_backward(moved(dy), (codes, s2), grad_x=moved(x)), qb.gelu_backward(dy, (codes, scales)))


def test_offsets_beyond_32_bits():
    """More than 2^32 values, rows that are no whole blocks: the end is as the beginning."""
    K = 136
    M = (1 << 32) // K + 100
    rows = torch.randn(100, K, device="cuda").bfloat16()
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[:100], x[-100:] = rows, rows
    codes, scales = qb.checkpoint(x)
    want, s64 = codes64(rows)
    assert torch.equal(codes[:100], want) and torch.equal(codes[-100:], want) and torch.equal(scales[:100], scales[-100:])
    assert (codes[100:200] == 0).all() and (scales[100:200] == 1).all() and (codes[-200:-100] == 0).all()
    qb.restore((codes, scales), torch.bfloat16, y=x)
    assert torch.equal(x[:100], x[-100:]) and torch.equal(x[:100], qb.restore((codes[:100].clone(), scales[:100].clone()), torch.bfloat16))


def test_refusals():
    x = torch.randn(8, 100, device="cuda")
    codes, scales = qb.checkpoint(x)
    for call in (lambda: qb.checkpoint(x.t()), lambda: qb.checkpoint(x.double()), lambda: qb.checkpoint(x[0]), lambda: qb.checkpoint(x, codes=codes.t()),
                 lambda: qb.checkpoint(x, scales=scales[:, :1].contiguous()), lambda: qb.restore((codes.float(), scales)), lambda: qb.restore((codes, scales[:4])),
                 lambda: qb.restore((codes, scales), torch.float32, y=x.half()), lambda: qb.gelu_backward(x, x.half()), lambda: qb.gelu_backward(x, x[:4]),
                 lambda: qb.gelu_backward(x, (codes[:4], scales)), lambda: qb.gelu_backward(x, (codes, scales[:, :1].contiguous()))):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: qb.gelu_backward(x, None), lambda: qb.gelu_backward(x, (codes, None)), lambda: qb.checkpoint(x[:0])):
        with pytest.raises(qb.QbertError) as e:
            call()
        assert e.value.status == qb.QB_ERR_INVALID
    with pytest.raises(qb.QbertError) as e:
        qb.restore((torch.zeros(801, dtype=torch.int8, device="cuda")[1:].view(8, 100), scales))
    assert e.value.status == qb.QB_ERR_ALIGN
