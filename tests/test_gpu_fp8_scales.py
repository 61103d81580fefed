"""qb_gemm_fp8 over the whole range of the scale bytes: either side as small as 2^-127, both together below fp32's normal numbers, and
beyond its largest."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_fp8 import E4M3, check_product, up, values

pytestmark = pytest.mark.gpu
SHAPES = [(70, 100, 640), (2048, 1280, 512), (2200, 2300, 1152)]  # 64 and 128 columns, pairs
LEAST = 2.0**-126


def codes(R, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(R, K, device="cuda", generator=g).clamp(-3, 3).to(E4M3)


def scales(bytes_):
    """The scale tensor of bytes [R][blocks]."""
    R, blocks = bytes_.shape
    s = torch.full((up(R) // 128, (blocks + 3) // 4, 32, 4, 4), 127, dtype=torch.uint8, device="cuda")
    r, j = torch.arange(R, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None, :]
    at = ((r // 128) * s.shape[1] + j // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + j % 4
    s.view(-1)[at.reshape(-1)] = bytes_.reshape(-1).to(torch.uint8)
    return s


def spread(R, level, g):
    """Bytes [R][blocks] within 5 of each block's level."""
    return (level[None, :] + torch.randint(-5, 6, (R, level.numel()), device="cuda", generator=g)).clamp(0, 254)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("swap", [False, True])
def test_one_side_small(M, N, K, swap):
    """Blocks of a from 2^-127 up against blocks of b that make up for it: sums of ordinary size, to the usual bound."""
    ws = qb.workspace()
    g = torch.Generator(device="cuda").manual_seed(M + swap)
    level = torch.randint(0, 127, (K // 128,), device="cuda", generator=g)
    level[0], level[-1] = 0, 126
    low, high = (N, M) if swap else (M, N)
    small, large = scales(spread(low, level, g)), scales(spread(high, 254 - level, g))
    a, b = codes(M, K, 1), codes(N, K, 2)
    sa, sb = (large, small) if swap else (small, large)
    check_product(qb.gemm_fp8(a, sa, b, sb, None, ws, torch.float32), a, sa, b, sb, None, torch.float32)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("total", [-100, -118, -127, -134, -150, -254])
def test_both_small(M, N, K, total):
    """Scales whose product is about 2^total.  Beside the usual bound, a term or a sum below 2^-126 may become 0: up to K / 32 + 32
    times on the way to an output (its accumulations, and the additions inside one), 2^-126 each."""
    ws = qb.workspace()
    g = torch.Generator(device="cuda").manual_seed(M - total)
    la = torch.randint(max(0, 254 + total - 127), min(127, 254 + total) + 1, (K // 128,), device="cuda", generator=g)
    a, b = codes(M, K, 1), codes(N, K, 2)
    sa, sb = scales(spread(M, la, g)), scales(spread(N, 254 + total - la, g))
    y = qb.gemm_fp8(a, sa, b, sb, None, ws, torch.float32)
    va, vb = values(a, sa), values(b, sb)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    off, tol = (y.double() - want).abs(), (size * 2.0**-23 + LEAST) * (K / 32 + 32)
    assert (off <= tol).all(), f"worst {float((off / tol).max()):.3g} of the bound"
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_beyond_the_largest(M, N, K):
    """Sums that fp32 does not hold are infinite: terms of one sign, each beyond it; rows of ordinary size beside them stay.

    Here the first blocks may be 2^10 times the others, so that the accumulator is large when the small terms come.  An instruction adds
    32 products to the accumulator; each of the 33 addends is aligned to the largest of them and cut off there, and loses less than
    one unit of fp32's last place of the largest, 2^-23 of it at most.  All terms are positive: the largest is at most the
    final sum, so that K / 32 instructions lose less than 33 * K / 32 * 2^-23 of it.  (The usual bound takes an instruction's products to
    be cut at their own size.)"""
    ws = qb.workspace()
    g = torch.Generator(device="cuda").manual_seed(N)
    a, b = codes(M, K, 1).float().abs().clamp(min=0.5).to(E4M3), codes(N, K, 2).float().abs().clamp(min=0.5).to(E4M3)
    level = torch.full((K // 128,), 127, device="cuda")
    byte_a = spread(M, level, g)
    byte_a[::3] = 254
    byte_b = spread(N, level + 6, g)
    sa, sb = scales(byte_a), scales(byte_b)
    y = qb.gemm_fp8(a, sa, b, sb, None, ws, torch.float32)
    assert (y[::3] == float("inf")).all()
    keep = torch.arange(M, device="cuda") % 3 != 0
    va, vb = values(a, sa)[keep], values(b, sb)
    want = va @ vb.t()
    assert ((y[keep].double() - want).abs() <= want * (33 * K / 32) * 2.0**-23).all()
    assert qb.read_status(ws) == qb.QB_OK
