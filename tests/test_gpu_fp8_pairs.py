"""qb_gemm_fp8 by pairs of CTAs (256 columns, two accumulators that share 32), whole tiles and tiles cut to half the width.  The form is
asked of the library, so that a shape which another choice serves differently fails here and is replaced."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_fewer_sms import in_part, part  # noqa: F401 (a fixture)
from test_gpu_fp8 import E4M3, E5M2, check_product, rows_of, unpack, up

# (M, N, K), whether some tiles are halves: ragged last rows and columns, several tiles a pair, words of scales that are not full
PAIRS = [((2200, 2300, 1152), True), ((5003, 2304, 768), True), ((4096, 5000, 1024), True), ((6144, 1024, 1152), True),
         ((2561, 2313, 1152), True),  # odd rows of y; the last tile's second half is wholly behind the last column
         ((5003, 2311, 768), False), ((4100, 4099, 1024), False), ((6101, 4099, 640), False)]


@pytest.fixture(scope="module")
def ws():
    return qb.workspace()


def operands(M, N, K):
    return (*qb.quantize_fp8(rows_of(M, K, 1), qb.workspace(), E5M2 if N % 2 else E4M3),
            *qb.quantize_fp8(rows_of(N, K, 2), qb.workspace(), E4M3 if M % 3 else E5M2))


@pytest.mark.parametrize("columns,form", [((1, 1, 128), (64, 0, 1)), ((2048, 1280, 512), (128, 0, 1)), ((256, 300, 24576), (64, 0, 12)), ((24576, 1024, 4096), (256, 28, 1))])
def test_the_form_of_a_shape(columns, form):
    assert qb.gemm_fp8_form(*columns, 1 << 28) == form
    assert qb.gemm_fp8_form(*columns[:2], 130) == (0, 0, 0) and qb.gemm_fp8_form(0, 1, 128) == (0, 0, 0)
    assert qb.lib().qb_gemm_fp8_tile_columns(*columns, 1 << 28, None, None) == form[0]


@pytest.mark.parametrize("shape,halves", PAIRS)
def test_shapes_are_served_by_pairs(shape, halves):
    columns, half_tiles, splits = qb.gemm_fp8_form(*shape, qb.workspace_bytes(groups=4096))
    assert columns == 256 and (half_tiles > 0) == halves and splits == 1


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,halves", PAIRS)
def test_product(ws, shape, halves, out):
    M, N, K = shape
    assert qb.gemm_fp8_form(M, N, K, ws.numel())[0] == 256
    a, sa, b, sb = operands(M, N, K)
    bias = torch.randn(N, device="cuda", generator=torch.Generator(device="cuda").manual_seed(N)) if M % 2 == 0 else None
    for shift in (0, 1, 3):  # y from an address of 16 bytes, and not
        buffer = torch.full((M * N + 264,), 3.0, dtype=out, device="cuda")
        y = qb.gemm_fp8(a, sa, b, sb, bias, ws, out, y=buffer[shift:shift + M * N].view(M, N))
        check_product(y, a, sa, b, sb, bias, out)
        assert (buffer[:shift] == 3.0).all() and (buffer[shift + M * N:] == 3.0).all()
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("shape,halves", PAIRS[:1] + PAIRS[4:6])
def test_scale_bytes_that_do_not_exist(ws, shape, halves):
    """0xFF (NaN, as a scale) for every row and block that the codes do not have changes nothing."""
    M, N, K = shape
    a, sa, b, sb = operands(M, N, K)
    want = qb.gemm_fp8(a, sa, b, sb, None, ws, torch.float32)

    def filled(s, R):
        e = (unpack(s, R, K // 128) + 127).to(torch.uint8)
        r, j = torch.arange(R, device="cuda")[:, None], torch.arange(K // 128, device="cuda")[None, :]
        at = ((r // 128) * s.shape[1] + j // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + j % 4
        t = torch.full_like(s, 0xFF)
        t.view(-1)[at.reshape(-1)] = e.view(-1)
        assert (t == 0xFF).sum() >= t.numel() - up(R) * (K // 128)
        return t
    assert torch.equal(qb.gemm_fp8(a, filled(sa, M), b, filled(sb, N), None, ws, torch.float32), want)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
def test_on_a_part_of_the_device(ws, part):  # noqa: F811
    got, want = [], []
    for shape, _ in PAIRS[:2]:
        args = operands(*shape)
        want.append(qb.gemm_fp8(*args, None, ws))
        torch.cuda.synchronize()
        in_part(part, lambda: got.append(qb.gemm_fp8(*args, None, ws)))
    assert len(got) == 2 and all(torch.equal(a, b) for a, b in zip(got, want))
    assert qb.read_status(ws) == qb.QB_OK
