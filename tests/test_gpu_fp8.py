"""8-bit floating point linears: codes and scales exactly, products against 64 bits."""
import pytest
import torch

import paper_1909_05840_b200 as qb

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
TOP = {E4M3: 448.0, E5M2: 57344.0}
BITS = {E4M3: (3, -6), E5M2: (2, -14)}


@pytest.fixture(scope="module")
def ws():
    return qb.workspace()


def up(n, m=128):
    return (n + m - 1) // m * m


def unpack(scales, R, blocks):
    """Exponents [R][blocks] from the bytes, by their documented address."""
    r, j = torch.arange(R, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None, :]
    words = scales.shape[1]
    at = ((r // 128) * words + j // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + j % 4
    return scales.reshape(-1)[at.reshape(-1)].view(R, blocks).to(torch.int32) - 127


def reference(x, dtype, rows):
    """Values (fp64 [R][Kp]) and exponents [R][Kp / 128] in blocks of `rows` x 128, from the definition."""
    R, K = x.shape
    pad = torch.zeros(up(R, rows), up(K), dtype=torch.float64, device="cuda")
    pad[:R, :K] = x.double()
    b = pad.view(-1, rows, up(K) // 128, 128)
    amax = b.abs().amax(dim=(1, 3))
    # the least e with amax / top <= 2^e, from the quotient's own exponent (its logarithm rounds at powers of two)
    m, e = torch.frexp(torch.where(amax > 0, amax, TOP[dtype]) / TOP[dtype])
    e = (e - (m == 0.5).to(e.dtype)).clamp(min=-127).double()
    bits, least = BITS[dtype]
    v = b * torch.ldexp(torch.ones_like(e), -e.int())[:, None, :, None]
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp(min=2.0**least))[1] - 1 - bits)
    q = (v / step).round() * step
    return q.view(pad.shape)[:R], e.to(torch.int32).repeat_interleave(rows, dim=0)[:R]


def check_codes(codes, scales, x, dtype, rows):
    q, e = reference(x, dtype, rows)
    assert codes.dtype == dtype and codes.shape == q.shape
    assert torch.equal(unpack(scales, *e.shape), e)
    assert torch.equal(codes.double(), q)


def values(codes, scales):
    R, Kp = codes.shape
    e = unpack(scales, R, Kp // 128)
    return (codes.double().view(R, -1, 128) * torch.ldexp(torch.ones_like(e, dtype=torch.float64), e)[:, :, None]).view(R, Kp)


def rows_of(M, K, seed, kind=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, device="cuda", generator=g) * torch.exp(2 * torch.randn(M, 1, device="cuda", generator=g))
    return x.to(kind)


def poisoned(shape, dtype=torch.uint8):
    return torch.full(shape, 0xFF, dtype=torch.uint8, device="cuda").view(dtype)


SHAPES = [(1, 1), (1, 128), (3, 130), (127, 384), (128, 512), (129, 516), (200, 1000), (33, 1541), (513, 768), (130, 127), (67, 513), (40, 1022), (3, 6), (260, 2047)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [E4M3, E5M2])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K", SHAPES)
def test_quantize(ws, M, K, kind, dtype):
    x = rows_of(M, K, M * 1000 + K, kind)
    q, s = qb.quantize_fp8(x, ws, dtype)
    check_codes(q, s, x, dtype, 1)
    # both ways at once: the rows' codes are the same, the columns' are those of the transposed matrix
    outs = (poisoned((M, up(K)), dtype), poisoned((qb.fp8_scale_bytes(M, K),)), poisoned((K, up(M)), dtype), poisoned((qb.fp8_scale_bytes(K, M),)))
    both = qb.quantize_fp8(x, ws, dtype, True, *outs)
    assert all(a is b for a, b in zip(both, outs))
    check_codes(both[0], both[1].view(s.shape), x, dtype, 1)
    check_codes(both[2], both[3].view(up(K) // 128, -1, 32, 4, 4), x.t().contiguous(), dtype, 1)
    w = qb.quantize_fp8_weights(x, ws, dtype, transposed=True)
    check_codes(w[0], w[1], x, dtype, 128)
    check_codes(w[2], w[3], x.t().contiguous(), dtype, 128)
    assert torch.equal(qb.quantize_fp8_weights(x, ws, dtype)[0].view(torch.uint8), w[0].view(torch.uint8))
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K", [(2690, 2690), (2561, 2817)])
def test_many_tiles(ws, M, K, kind):
    """More tiles than fit the device at once; rows that are aligned to four values and that are not; the columns' sums."""
    x = rows_of(M, K, M + K, kind)
    q = qb.quantize_fp8(x, torch.zeros(qb.fp8_sums_workspace_bytes(M, K), dtype=torch.uint8, device="cuda"), E4M3, True, want_sums=True)
    check_codes(q[0], q[1], x, E4M3, 1)
    check_codes(q[2], q[3], x.t().contiguous(), E4M3, 1)
    # each of the M - 1 additions rounds by half a step of a partial sum, which is at most the sum of magnitudes
    bound = x.double().abs().sum(dim=0) * (M * 2.0**-24)
    assert ((q[4].double() - x.double().sum(dim=0)).abs() <= bound).all()
    w = qb.quantize_fp8_weights(x, ws, E5M2, transposed=True)
    check_codes(w[0], w[1], x, E5M2, 128)
    check_codes(w[2], w[3], x.t().contiguous(), E5M2, 128)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [E4M3, E5M2])
def test_borders(ws, dtype):
    """Maxima at and beside the format's largest value, the ends of fp32, zeros, ties."""
    x = torch.zeros(12, 256, device="cuda")
    top = TOP[dtype]
    x[0, 5], x[1, 5] = top, torch.nextafter(torch.tensor(top), torch.tensor(1e9))
    x[2, 7], x[3, 9] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).tiny
    x[4, 3] = 2.0**-149
    x[5, :128] = torch.arange(128, device="cuda") * 0.0625 + 1.0  # ties between codes
    x[5, 0] = top
    x[6] = -x[5]
    x[7, 128:] = 2.0**-119
    x[8, 0], x[8, 1] = top, 2.0**-9 * 0.5  # half of the least code of e4m3
    x[9, 0], x[9, 1] = top, 2.0**-9 * 1.5
    x[10, 200] = -top * 2.0**100
    for t in (False, True):
        q = qb.quantize_fp8(x, ws, dtype, transposed=t)
        check_codes(q[0], q[1], x, dtype, 1)
        if t:
            check_codes(q[2], q[3], x.t().contiguous(), dtype, 1)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_quantize_any_alignment(ws, kind, shift):
    flat = rows_of(1, 40 * 384 + 8, 5, kind).view(-1)
    x = flat[shift:shift + 40 * 384].view(40, 384)
    a, b = qb.quantize_fp8(x, ws, E4M3, True), qb.quantize_fp8(x.clone(), ws, E4M3, True)
    for i in (0, 2):
        assert torch.equal(a[i].view(torch.uint8), b[i].view(torch.uint8))
    assert torch.equal(unpack(a[1], 40, 3), unpack(b[1], 40, 3)) and torch.equal(unpack(a[3], 384, 1), unpack(b[3], 384, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("form", ["rows", "both", "weights"])
def test_not_finite(form, bad):
    ws = qb.workspace()
    x = rows_of(130, 300, 1)
    x[129, 260] = bad
    call = qb.quantize_fp8_weights if form == "weights" else qb.quantize_fp8
    q = call(x, ws, E4M3, transposed=form != "rows")
    assert qb.read_status(ws) == qb.QB_ERR_NONFINITE
    assert torch.isnan(q[0][129, 260].float()) and torch.isnan(q[0].float()).sum() == 1
    w, wsc = qb.quantize_fp8_weights(rows_of(9, 300, 2), ws)
    y = qb.gemm_fp8(q[0], q[1], w, wsc, None, ws, torch.float32)
    assert torch.isnan(y[129]).all() and torch.isfinite(y[:128]).all()
    if form != "rows":
        assert torch.isnan(q[2][260, 129].float()) and torch.isnan(q[2].float()).sum() == 1


def check_product(y, a, sa, b, sb, bias, out):
    """Against 64 bits.  The products of codes are exact; fp32 accumulation loses at most 2^-23 (its last bit, cut off) of the terms'
    absolute sum for each of the K / 32 accumulations and of the additions inside one of 32 terms; then the bias's addition
    and the output's rounding, half a step each."""
    va, vb = values(a, sa), values(b, sb)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    K = a.shape[1]
    tol = size * (K / 32 + 32) * 2.0**-23
    if bias is not None:
        want = want + bias.double()
        tol = tol + want.abs() * 2.0**-24
    tol = tol * 1.01 + want.abs() * (torch.finfo(out).eps / 2 if out == torch.bfloat16 else 0.0) + 1e-300
    assert y.dtype == out
    off = (y.double() - want).abs()
    assert (off <= tol).all(), f"{int((off > tol).sum())} of {off.numel()} off, worst {float((off / tol).max()):.3g} of the bound"


# (M, N, K): one value, odd sizes, every tile form (64 and 128 columns, pairs), several tiles a CTA, partial last tiles
PRODUCTS = [(1, 1, 128), (1, 9, 768), (5, 64, 256), (77, 130, 640), (128, 128, 128), (300, 520, 1152), (2000, 900, 384), (2048, 1280, 512),
            (2561, 2600, 768), (4100, 4099, 256), (4096, 5000, 128),
            (6144, 1024, 640), (5003, 2304, 256)]


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(ws, M, N, K, out):
    g = torch.Generator(device="cuda").manual_seed(N)
    a, sa = qb.quantize_fp8(rows_of(M, K, 1), ws, E5M2 if N % 2 else E4M3)
    b, sb = qb.quantize_fp8(rows_of(N, K, 2), ws, E4M3 if M % 3 else E5M2)
    bias = torch.randn(N, device="cuda", generator=g) if M % 2 == 0 else None
    buffer = torch.full((M * N + 256,), 3.0, dtype=out, device="cuda")
    y = qb.gemm_fp8(a, sa, b, sb, bias, ws, out, y=buffer[:M * N].view(M, N))
    assert qb.read_status(ws) == qb.QB_OK
    check_product(y, a, sa, b, sb, bias, out)
    assert (buffer[M * N:] == 3.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K", [(1, 1), (130, 9), (613, 768), (1024, 131), (5003, 260)])
def test_column_sums(M, K, kind):
    """A bias's gradient beside the codes.  fp32 additions: 16 rows, 8 warps, an eighth of the tiles and 8 warps in a chain, 2^-24 of the
    terms' absolute sum each."""
    x = rows_of(M, K, M + K, kind)
    ws = torch.zeros(qb.fp8_sums_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    plain = qb.quantize_fp8(x, ws, E5M2, transposed=True)
    sums = torch.full((K + 3,), 7.0, device="cuda")
    both = qb.quantize_fp8(x, ws, E5M2, transposed=True, want_sums=True, sums=sums[:K])
    assert len(both) == 5 and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(plain[::2], both[::2]))
    want, size = x.double().sum(0), x.double().abs().sum(0)
    assert ((sums[:K].double() - want).abs() <= size * (16 + 8 + M / 1024 + 1 + 8) * 2.0**-24).all() and (sums[K:] == 7.0).all()
    assert torch.equal(sums[:K], qb.quantize_fp8(x, ws, E5M2, transposed=True, want_sums=True)[4])
    for bad in (dict(sums=sums), dict(sums=sums[:K].half()), dict(sums=sums[:K].cpu())):
        with pytest.raises(AssertionError):
            qb.quantize_fp8(x, ws, E5M2, transposed=True, want_sums=True, **bad)
    with pytest.raises(qb.QbertError):
        qb.quantize_fp8(x, ws, want_sums=True)
    with pytest.raises(qb.QbertError):
        qb.quantize_fp8(x, ws[:-4], E5M2, transposed=True, want_sums=True)


# few tiles over a long contraction: summed in parts side by side where the workspace has room, in one piece where not
@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(9, 7, 8192), (256, 300, 24576), (129, 770, 65536), (768, 768, 4224), (70, 40, 131200)])
def test_long_contractions(M, N, K, out):
    a, sa = qb.quantize_fp8(rows_of(M, K, 1), qb.workspace())
    b, sb = qb.quantize_fp8(rows_of(N, K, 2), qb.workspace())
    bias = torch.randn(N, device="cuda")
    if K > 65536:  # the contraction of a weight gradient over more tokens than the integer linears take features
        assert a.shape[1] == K
    for nbytes in (256, 1024 + 3 * M * N * 4, 1024 + 100 * M * N * 4):
        ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
        y = qb.gemm_fp8(a, sa, b, sb, bias, ws, out)
        check_product(y, a, sa, b, sb, bias, out)
        assert torch.equal(y, qb.gemm_fp8(a, sa, b, sb, bias, ws, out))
        shifted = torch.empty(M * N + 1, dtype=out, device="cuda")[1:].view(M, N)
        assert torch.equal(y, qb.gemm_fp8(a, sa, b, sb, bias, ws, out, y=shifted))
        assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(3, 40, 512), (2100, 2100, 384)])
def test_product_output_alignment(ws, M, N, K):
    a, sa = qb.quantize_fp8(rows_of(M, K, 1), ws)
    b, sb = qb.quantize_fp8(rows_of(N, K, 2), ws)
    for out in (torch.float32, torch.bfloat16):
        want = qb.gemm_fp8(a, sa, b, sb, None, ws, out)
        for shift in (1, 3):
            buffer = torch.full((M * N + 8,), 3.0, dtype=out, device="cuda")
            got = qb.gemm_fp8(a, sa, b, sb, None, ws, out, y=buffer[shift:shift + M * N].view(M, N))
            assert torch.equal(got, want)
            assert (buffer[:shift] == 3.0).all() and (buffer[shift + M * N:] == 3.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(70, 100, 640), (2200, 2300, 640)])
def test_scales_of_every_block(ws, M, N, K):
    """Every row and block with a scale of its own, over the whole range of the bytes that keeps the sums finite; bytes of rows and
    blocks that do not exist hold 0xFF."""
    g = torch.Generator(device="cuda").manual_seed(3)
    a = torch.randn(M, K, device="cuda", generator=g).clamp(-3, 3).to(E4M3)
    b = torch.randn(N, K, device="cuda", generator=g).clamp(-3, 3).to(E4M3)

    def scales(R):
        s = torch.full((up(R) // 128, (K + 511) // 512, 32, 4, 4), 0xFF, dtype=torch.uint8, device="cuda")
        r, j = torch.arange(R, device="cuda")[:, None], torch.arange(K // 128, device="cuda")[None, :]
        at = ((r // 128) * s.shape[1] + j // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + j % 4
        s.view(-1)[at.reshape(-1)] = torch.randint(100, 150, (at.numel(),), device="cuda", generator=g).to(torch.uint8)
        return s
    sa, sb = scales(M), scales(N)
    check_product(qb.gemm_fp8(a, sa, b, sb, None, ws, torch.float32), a, sa, b, sb, None, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 9, 130), (613, 9, 768), (700, 520, 392), (3000, 1100, 1024)])
def test_three_products_of_a_linear(ws, M, N, K):
    """A linear and its gradients, from tensors to tensors.  A code is off by at most half its step, 2^-4 (e4m3) or 2^-3 (e5m2) of
    the value, and 2^-10 * 2^-8 of its block's maximum below the least normal code; each product by the sum over its terms."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn(M, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g) * 0.02
    dy = torch.randn(M, N, device="cuda", generator=g) * 1e-4
    xq, xs, xqt, xst = qb.quantize_fp8(x, ws, transposed=True)
    wq, wsc, wqt, wst = qb.quantize_fp8_weights(w, ws, transposed=True)
    gq, gs, gqt, gst = qb.quantize_fp8(dy.bfloat16(), ws, E5M2, transposed=True)
    y = qb.gemm_fp8(xq, xs, wq, wsc, None, ws, torch.float32)
    dx = qb.gemm_fp8(gq, gs, wqt, wst, None, ws, torch.float32)
    dw = qb.gemm_fp8(gqt, gst, xqt, xst, None, ws, torch.float32)
    assert (y.shape, dx.shape, dw.shape) == ((M, N), (M, K), (N, K))
    for got, args in ((y, (xq, xs, wq, wsc)), (dx, (gq, gs, wqt, wst)), (dw, (gqt, gst, xqt, xst))):
        check_product(got, *args, None, torch.float32)
    xd, wd, gd = x.double(), w.double(), dy.bfloat16().double()
    ex, ew, eg = 2.0**-4, 2.0**-4, 2.0**-3

    def close(got, a, b, ea, eb):
        size = a.abs() @ b.abs()
        floor = 2.0**-17 * (a.abs().amax() * b.abs().sum(0)[None, :] + a.abs().sum(1)[:, None] * b.abs().amax())
        assert ((got.double() - a @ b).abs() <= size * (ea + eb + ea * eb) * 1.01 + floor).all()
    close(y, xd, wd.t(), ex, ew)
    close(dx, gd, wd, eg, ew)
    close(dw, gd.t(), xd, eg, ex)


@pytest.mark.gpu
def test_captured_and_on_another_stream(ws):
    x, w = rows_of(600, 768, 1), rows_of(520, 768, 2)
    bias = torch.randn(520, device="cuda")
    wq, wsc = qb.quantize_fp8_weights(w, ws)
    xq, xs = qb.quantize_fp8(x, ws)
    y = qb.gemm_fp8(xq, xs, wq, wsc, bias, ws)

    def call():
        qb.quantize_fp8(x, ws, codes=xq, scales=xs)
        qb.gemm_fp8(xq, xs, wq, wsc, bias, ws, y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    s, ws2 = torch.cuda.Stream(), qb.workspace()
    for seed in (5, 6):
        x.copy_(rows_of(600, 768, seed))
        s.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(s):  # at the same time, with a workspace of its own
            other = qb.gemm_fp8(*qb.quantize_fp8(x, ws2), wq, wsc, bias, ws2)
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(other, y)
        check_product(y, xq, xs, wq, wsc, bias, torch.bfloat16)


@pytest.mark.gpu
def test_outputs_are_ordinary_tensors(ws):
    """Codes and scales share an allocation: they outlive each other, and views, copies and in-place calls work on them."""
    x, w = rows_of(200, 300, 1), rows_of(40, 300, 2)
    q, s, qt, st = qb.quantize_fp8(x, ws, transposed=True)
    want = [t.clone() for t in (q, s, qt, st)]
    y = qb.gemm_fp8(q, s, *qb.quantize_fp8_weights(w, ws), None, ws)
    del q, qt
    for _ in range(20):
        torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(s, want[1]) and torch.equal(st, want[3])
    assert torch.equal(y, qb.gemm_fp8(want[0], s, *qb.quantize_fp8_weights(w, ws), None, ws))
    assert s.is_contiguous() and s.view(-1).numel() == qb.fp8_scale_bytes(200, 300) and not s.requires_grad
    s.fill_(127)
    assert torch.equal(want[0].cpu().float(), want[0].float().cpu()) and (s == 127).all()
    assert torch.equal(want[2].float()[:, :200], want[2][:, :200].float())


@pytest.mark.gpu
def test_python_refusals(ws):
    x = rows_of(8, 256, 1)
    q, s = qb.quantize_fp8(x, ws)
    w, t = qb.quantize_fp8(rows_of(5, 256, 2), ws)
    for call in (lambda: qb.quantize_fp8(x.double(), ws), lambda: qb.quantize_fp8(x.t(), ws), lambda: qb.quantize_fp8(x.cpu(), ws),
                 lambda: qb.quantize_fp8(x.view(-1), ws), lambda: qb.quantize_fp8(x, ws.float()), lambda: qb.quantize_fp8(x, ws.cpu()),
                 lambda: qb.quantize_fp8(x, ws, codes=q[:4]), lambda: qb.quantize_fp8(x, ws, E5M2, codes=q),
                 lambda: qb.quantize_fp8(x, ws, scales=s.view(-1)[:256]),
                 lambda: qb.gemm_fp8(q, s, w[:, :128].contiguous(), t, None, ws), lambda: qb.gemm_fp8(q.view(torch.uint8), s, w, t, None, ws),
                 lambda: qb.gemm_fp8(q, s.view(-1)[:256], w, t, None, ws), lambda: qb.gemm_fp8(q, s, w, t, x.view(-1)[:4], ws),
                 lambda: qb.gemm_fp8(q, s, w, t, None, ws, y=torch.empty(8, 5, device="cuda")),
                 lambda: qb.gemm_fp8(q, s, w, t, None, ws, torch.float32, y=torch.empty(8, 4, device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: qb.quantize_fp8(x, ws, torch.int8), lambda: qb.gemm_fp8(q, s, w, t, None, ws, torch.float16),
                 lambda: qb.quantize_fp8(x, ws[:128]), lambda: qb.gemm_fp8(q, s, w, t, None, ws[:128]), lambda: qb.quantize_fp8(x[:0], ws)):
        with pytest.raises(qb.QbertError):
            call()


@pytest.mark.gpu
def test_outputs_of_another_shape(ws):
    """As many elements in another shape are refused: rows and columns exchanged, a flat buffer."""
    x, w = rows_of(256, 128, 1), rows_of(384, 128, 2)
    q, s, qt, st = qb.quantize_fp8(x, ws, transposed=True)
    v, t = qb.quantize_fp8(w, ws)
    y = torch.empty(384, 256, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: qb.gemm_fp8(q, s, v, t, None, ws, y=y), lambda: qb.gemm_fp8(q, s, v, t, None, ws, y=y.view(-1)),
                 lambda: qb.quantize_fp8(x, ws, codes=qt), lambda: qb.quantize_fp8(x, ws, codes=q.view(-1)),
                 lambda: qb.quantize_fp8(x, ws, transposed=True, codes_t=q), lambda: qb.quantize_fp8_weights(x, ws, transposed=True, codes_t=q)):
        with pytest.raises(AssertionError):
            call()
    y = y.view(256, 384)
    assert qb.gemm_fp8(q, s, v, t, None, ws, y=y) is y and qb.quantize_fp8(x, ws, codes=q, scales=s)[0] is q
