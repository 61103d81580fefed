"""Linears in 16 bits with what follows them, and their gradients, against 64 bits."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_checkpoint import GELU_ABS, SLOPE_ABS, codes64, gelu64, half, least, slope64, values64

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0**-24


@pytest.fixture(scope="module")
def ws():
    return torch.zeros(1 << 27, dtype=torch.uint8, device="cuda")


def product(a, b, K):
    """a b^T in 64 bits and the bound of its error in fp32: an addition of 16 products cuts the accumulator and each product off at the
    last place of the largest of them (2^-23 of the sum of magnitudes for each of the 17 at most, in all 2^-19); partial sums of
    parts are added once more."""
    want, magnitude = a @ b.t(), a.abs() @ b.abs().t()
    return want, magnitude * (K / 16 + 1) * 2.0**-22 + magnitude * 2.0**-19


def within(got, want, tol):
    tol = tol * 1.01 + want.abs() * half(got.dtype) * 1.01 + least(got.dtype)
    far = (got.double() - want).abs() - tol
    assert got.shape == want.shape and (far <= 0).all(), (float(far.max()), int((far > 0).sum()))


def data(seed, *shapes, t):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, device="cuda", generator=g).to(t) for s in shapes]


# one token, less than a tile, every remainder of 8 and 64, more tiles than SMs, widths that are no multiple of 8
SIZES = [(1, 1, 1), (1, 8, 8), (1, 768, 768), (2, 3, 5), (5, 9, 17), (33, 64, 128), (64, 72, 96), (127, 129, 64), (128, 128, 64), (130, 257, 65), (200, 200, 200), (256, 256, 192),
         (300, 520, 1000), (613, 9, 768), (1000, 776, 768), (2500, 1030, 513), (2049, 2304, 768), (4100, 1024, 328), (9000, 520, 136), (77, 3000, 2056), (1, 4099, 4097), (5003, 768, 776), (5003, 2304, 328), (4099, 4096, 264), (5003, 328, 2304), (328, 5008, 2304), (264, 4099, 4096)]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_whole_numbers(M, N, K, kind, ws):
    """Small whole numbers, whose sums are exact in any order: the three products equal to the bit, at every size."""
    t = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    x, w, dy = (torch.randint(-2, 3, s, device="cuda", generator=g).to(t) for s in ((M, K), (N, K), (M, N)))
    bias = torch.randint(-3, 4, (N,), device="cuda", generator=g).float()
    z = x.double() @ w.double().t() + bias.double()
    room = torch.full((M * N + 64,), 7.0, device="cuda")
    assert torch.equal(qb.linear(x, w, bias, ws, out_dtype=torch.float32, y=room[:M * N].view(M, N)).double(), z) and (room[M * N:] == 7.0).all()
    room = torch.full((M * N + 64,), 7.0, dtype=t, device="cuda")
    assert torch.equal(qb.linear(x, w, bias, ws, y=room[:M * N].view(M, N)), z.to(t)) and (room[M * N:] == 7.0).all()
    room = torch.full((M * K + 64,), 7.0, dtype=t, device="cuda")
    assert torch.equal(qb.linear_grad_x(dy, w, ws, grad_x=room[:M * K].view(M, K)), (dy.double() @ w.double()).to(t)) and (room[M * K:] == 7.0).all()
    room = torch.full((N * K + 64,), 7.0, device="cuda")
    dw, db = qb.linear_grad_w(dy, x, ws, grad_w=room[:N * K].view(N, K))
    assert torch.equal(dw.double(), dy.double().t() @ x.double()) and (room[N * K:] == 7.0).all()
    assert torch.equal(db.double(), dy.double().sum(0))
    dw, db = qb.linear_grad_w(dy, x, ws, out_dtype=t, needs=(True, False))
    assert db is None and torch.equal(dw, (dy.double().t() @ x.double()).to(t))
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("activation", [None, "gelu"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("out", ["same", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 768, 768), (5, 9, 17), (130, 257, 72), (300, 520, 1000), (613, 776, 64), (2500, 1030, 136), (4100, 1024, 328), (77, 136, 4096)])
def test_forward(M, N, K, out, residual, activation, kind, ws):
    t = TYPES[kind]
    x, w, bias, r = data(M + N + K, (M, K), (N, K), (N,), (M, N), t=t)
    w, bias = w * 0.05, bias.float()
    o = t if out == "same" else torch.float32
    r = r.to(o) if residual else None
    z, tol = product(x.double(), w.double(), K)
    z, tol = z + bias.double(), tol + U * (z.abs() + bias.double().abs())
    y, tol_y = (gelu64(z), 1.13 * tol + GELU_ABS + U * 2 * z.abs()) if activation else (z, tol)
    if residual:
        y, tol_y = y + r.double(), tol_y + U * (y.abs() + r.double().abs())
    got = qb.linear(x, w, bias, ws, activation=activation, residual=r, out_dtype=o)
    within(got, y, tol_y)
    # with a workspace that leaves no room for parts, and in place of the residual
    small = ws if K % 8 or N % 8 else ws[:1024]
    if residual:
        kept = r.clone()
        again = qb.linear(x, w, bias, small, activation=activation, residual=kept, out_dtype=o, y=kept)
        assert again is kept
    else:
        again = qb.linear(x, w, bias, small, activation=activation, out_dtype=o)
    within(again, y, tol_y)
    if out == "same":
        got2, pre = qb.linear(x, w, bias, ws, activation=activation, residual=r, save="pre")
        assert torch.equal(got2, got)
        within(pre, z, tol)
        got3, saved = qb.linear(x, w, bias, ws, activation=activation, residual=r, save="codes")
        within(got3, y, tol_y)
        # a code is that of a value that lies within the product's error of z: half a step and that error off at most
        s = saved[1].double().repeat_interleave(64, 1)[:, :N]
        assert ((values64(*saved) - z).abs() <= s * (0.5 + 2.0**-16) + tol).all()
        _, s64 = codes64(z)
        block_tol = torch.nn.functional.pad(tol, (0, -N % 64)).view(M, -1, 64).amax(2)
        assert ((saved[1].double() - s64).abs() <= block_tol / 127 + 2 * U * s64).all()
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,N,K", [(1, 768, 768), (5, 9, 17), (130, 257, 72), (300, 520, 1000), (613, 9, 776), (2500, 136, 1030), (4100, 328, 1024), (77, 4096, 136)])
def test_grad_x(M, N, K, kind, ws):
    t = TYPES[kind]
    dy, w, p, r = data(M * N, (M, N), (N, K), (M, K), (M, K), t=t)
    w, p = w * 0.05, p * 2
    g, tol = product(dy.double(), w.double().t(), N)
    within(qb.linear_grad_x(dy, w, ws), g, tol)
    within(qb.linear_grad_x(dy, w, ws, residual=r), g + r.double(), tol + U * (g.abs() + r.double().abs()))
    kept = r.clone()
    within(qb.linear_grad_x(dy, w, ws, residual=kept, grad_x=kept), g + r.double(), tol + U * (g.abs() + r.double().abs()))
    s = slope64(p.double())
    within(qb.linear_grad_x(dy, w, ws, through=p), g * s, 1.13 * tol + g.abs() * SLOPE_ABS + U * (g * s).abs())
    saved = qb.checkpoint(p)
    q = values64(*saved)
    s = slope64(q)
    tol_q = 1.13 * tol + g.abs() * (SLOPE_ABS + U * q.abs()) + U * (g * s).abs()
    within(qb.linear_grad_x(dy, w, ws, through=saved), g * s, tol_q)
    small = ws if K % 8 or N % 8 else ws[:1024]
    within(qb.linear_grad_x(dy, w, small, through=saved), g * s, tol_q)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("out", ["same", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 768, 768), (2, 9, 17), (130, 257, 72), (300, 520, 1000), (613, 9, 768), (5003, 768, 136), (24576, 64, 1024), (20001, 9, 133)])
def test_grad_w(M, N, K, out, kind, ws):
    t = TYPES[kind]
    o = t if out == "same" else torch.float32
    dy, x = data(M + K, (M, N), (M, K), t=t)
    want, tol = product(dy.double().t(), x.double().t(), M)
    dw, db = qb.linear_grad_w(dy, x, ws, out_dtype=o)
    within(dw, want, tol)
    # the chain of a column: rows of a warp's run, the warps, the runs
    db_tol = 1.01 * U * (M / 100 + 1300) * dy.double().abs().sum(0)
    assert ((db.double() - dy.double().sum(0)).abs() <= db_tol).all()
    again, db2 = qb.linear_grad_w(dy, x, ws, out_dtype=o)
    assert torch.equal(again, dw) and torch.equal(db2, db)
    only, none = qb.linear_grad_w(dy, x, ws, out_dtype=o, needs=(True, False))
    assert none is None
    within(only, want, tol)
    none, db3 = qb.linear_grad_w(dy, x, ws, needs=(False, True))
    assert none is None and ((db3.double() - dy.double().sum(0)).abs() <= db_tol).all()  # (another order of the same sums)


@pytest.mark.parametrize("M,N,K", [(24576, 256, 1024), (1024, 768, 768), (6144, 1030, 520), (613, 2000, 1000)])
def test_fp32_sums(M, N, K, ws):
    """fp32 outputs are nearer to 64 bits than one chain of additions that are cut off would be (24,576 of them: 2.8e-5): at most 512 products,
    32 additions, go into one accumulator, each cut by 2^-23 of it at most, 2^-18 of a run's sum; what the runs' sums are off by adds up
    as they do."""
    g = torch.Generator(device="cuda").manual_seed(3)
    dy, x = torch.randn(M, N, device="cuda", generator=g).bfloat16(), torch.randn(M, K, device="cuda", generator=g).bfloat16()
    want = dy.double().t() @ x.double()
    for room in (ws, ws[:1 << 20]):
        if N % 8 == 0 or room is ws:
            dw, _ = qb.linear_grad_w(dy, x, room)
            assert float((dw.double() - want).norm() / want.norm()) <= 2.0**-18
    w = torch.randn(N, M, device="cuda", generator=g).bfloat16()
    y = qb.linear(x.t().contiguous(), w, None, ws, out_dtype=torch.float32)
    z = x.double().t() @ w.double().t()
    assert float((y.double() - z).norm() / z.norm()) <= 2.0**-18


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("M,N,K", [(70, 100, 96), (600, 1000, 520)])
def test_not_finite(bad, M, N, K, ws):
    """What is not finite reaches its own row or column and no other."""
    x, w = data(1, (M, K), (N, K), t=torch.bfloat16)
    clean = qb.linear(x, w, None, ws, activation="gelu")
    xb = x.clone()
    xb[3, K - 1] = bad
    y, saved = qb.linear(xb, w, None, ws, activation="gelu", save="codes")
    keep = torch.arange(M, device="cuda") != 3
    z = xb[3].double() @ w.double().t()
    limit = torch.where(z.isnan(), z, torch.where(z > 0, z, -torch.zeros_like(z)))  # gelu(-inf) is the limit 0
    assert torch.equal(y[3].isnan(), limit.isnan()) and torch.equal(y[3].isinf(), limit.isinf()) and torch.equal(y[keep], clean[keep])
    restored = qb.restore(saved, torch.float32)
    assert restored[3].isnan().all() and restored[keep].isfinite().all()
    wb = w.clone()
    wb[5, 0] = bad
    dx = qb.linear_grad_x(clean, wb, ws)
    assert not dx[:, 0].isfinite().any() and dx[:, 1:].isfinite().all()


def test_forms_that_are_covered(ws):
    """The sizes above meet every form in every product: tiles of 128 x 64, 128 x 128, 256 x 128 and 256 x 256, halves, parts."""
    forms = [qb.linear_form(*s, ws.numel()) for M, N, K in SIZES for s in ((M, N, K), (M, K, N), (N, K, M))]
    assert {f[:2] for f in forms} == {(128, 64), (128, 128), (256, 128), (256, 256)}
    assert any(f[2] > 0 for f in forms) and any(f[3] > 1 for f in forms)


def test_codes_of_any_alignment(ws):
    M, N, K = 70, 128, 64
    x, w, dy = data(2, (M, K), (N, K), (M, K), t=torch.bfloat16)
    y, (codes, scales) = qb.linear(x, w, None, ws, save="codes")
    moved = torch.empty(M * N + 16, dtype=torch.int8, device="cuda")[3:3 + M * N].view(M, N)
    y2, (c2, s2) = qb.linear(x, w, None, ws, save="codes", saved=(moved, torch.empty_like(scales)))
    assert c2 is moved and torch.equal(c2, codes) and torch.equal(s2, scales) and torch.equal(y2, y)
    g = qb.linear_grad_x(dy, w.t().contiguous(), ws, through=(codes, scales))
    assert torch.equal(qb.linear_grad_x(dy, w.t().contiguous(), ws, through=(moved, scales)), g)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("shift", [1, 3, 8])
@pytest.mark.parametrize("M,N,K", [(70, 136, 64), (600, 1016, 520), (2500, 1024, 136)])
def test_any_alignment(M, N, K, shift, kind, ws):
    """Outputs, residuals and pre-activations that begin at any element: the same values as aligned ones, and nothing beside them."""
    t = TYPES[kind]
    x, w, r, dy, p = data(3, (M, K), (N, K), (M, N), (M, N), (M, K), t=t)

    def moved(v):
        b = torch.full((v.numel() + 16,), 7.0, dtype=v.dtype, device="cuda")
        b[shift:shift + v.numel()] = v.reshape(-1)
        return b, b[shift:shift + v.numel()].view(v.shape)

    def clean(b, v):
        return bool((b[:shift] == 7).all() and (b[shift + v.numel():] == 7).all())
    for o in (t, torch.float32):
        want = qb.linear(x, w, None, ws, residual=r.to(o), out_dtype=o)
        (b, y), (_, rm) = moved(torch.empty_like(want)), moved(r.to(o))
        assert torch.equal(qb.linear(x, w, None, ws, residual=rm, out_dtype=o, y=y), want) and clean(b, y)
    want, pre = qb.linear(x, w, None, ws, activation="gelu", save="pre")
    (b, y), (c, z) = moved(torch.empty_like(want)), moved(torch.empty_like(pre))
    qb.linear(x, w, None, ws, activation="gelu", save="pre", y=y, pre=z)
    assert torch.equal(y, want) and torch.equal(z, pre) and clean(b, y) and clean(c, z)
    want = qb.linear_grad_x(dy, w, ws, through=p)
    (b, g), (_, pm) = moved(torch.empty_like(want)), moved(p)
    assert torch.equal(qb.linear_grad_x(dy, w, ws, through=pm, grad_x=g), want) and clean(b, g)
    want, _ = qb.linear_grad_w(dy, x, ws)
    b, g = moved(torch.empty_like(want))
    assert torch.equal(qb.linear_grad_w(dy, x, ws, grad_w=g)[0], want) and clean(b, g)


def test_offsets_beyond_32_bits(ws):
    """More than 2^32 bytes of every output: the last rows are as they are alone."""
    N, K = 4096, 64
    M = (1 << 31) // N + 300
    part = torch.randn(512, K, device="cuda").bfloat16()
    x = part.repeat((M + 511) // 512, 1)[:M].contiguous()
    w, bias = torch.randn(N, K, device="cuda").bfloat16(), torch.randn(N, device="cuda")
    r = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    y, saved = qb.linear(x, w, bias, ws, activation="gelu", residual=r, save="codes")
    tail = x[-300:].contiguous()
    y0, saved0 = qb.linear(tail, w, bias, ws, activation="gelu", residual=r[:300], save="codes")
    assert torch.equal(y[-300:], y0) and torch.equal(saved[0][-300:], saved0[0]) and torch.equal(saved[1][-300:], saved0[1])
    assert torch.equal(y[:512], y[512 * 100:512 * 101])
    back = torch.randn(K, N, device="cuda").bfloat16()  # grad_x [M][N] of a linear of N inputs and K outputs
    g = qb.linear_grad_x(x, back, ws, through=saved, grad_x=r)
    assert torch.equal(g[-300:], qb.linear_grad_x(tail, back, ws, through=(saved0[0], saved0[1])))
    dw, db = qb.linear_grad_w(y, x, ws)
    assert dw.isfinite().all() and db.isfinite().all()


def test_refusals(ws):
    x, w, dy, wide = data(2, (64, 96), (40, 96), (64, 40), (64, 264), t=torch.bfloat16)
    bias = torch.zeros(40, device="cuda")
    for call in (lambda: qb.linear(x.t(), w, bias, ws), lambda: qb.linear(x, w.half(), bias, ws), lambda: qb.linear(x, w[:, :88], bias, ws), lambda: qb.linear(x.float(), w.float(), bias, ws),
                 lambda: qb.linear(x, w, bias.bfloat16(), ws), lambda: qb.linear(x, w, bias[:8], ws), lambda: qb.linear(x, w, bias, ws, residual=x),
                 lambda: qb.linear(x, w, bias, ws, residual=dy, out_dtype=torch.float32), lambda: qb.linear(x, w, bias, ws, y=x), lambda: qb.linear(x, w, bias, ws.cpu()),
                 lambda: qb.linear_grad_x(dy, w.t().contiguous(), ws), lambda: qb.linear_grad_x(dy, w, ws, through=dy), lambda: qb.linear_grad_x(dy, w, ws, residual=dy),
                 lambda: qb.linear_grad_w(dy, x[:8], ws), lambda: qb.linear_grad_w(dy, x.half(), ws), lambda: qb.linear_grad_w(dy, x, ws, grad_w=w),
                 lambda: qb.linear_grad_w(dy, x, ws, grad_bias=bias[:3])):
        with pytest.raises(AssertionError):
            call()
    for call, status in ((lambda: qb.linear(x, w, bias, ws, save="pre", out_dtype=torch.float32), qb.QB_ERR_INVALID),
                         (lambda: qb.linear_grad_x(dy, w, ws, through=x, residual=x), qb.QB_ERR_INVALID),
                         (lambda: qb.linear_grad_w(dy, x, ws, needs=(False, False)), qb.QB_ERR_INVALID),
                         (lambda: qb.linear(x[:, :33].contiguous(), w[:, :33].contiguous(), bias, ws[:1024]), qb.QB_ERR_WORKSPACE),
                         (lambda: qb.linear_grad_w(wide, x, ws[:1024]), qb.QB_ERR_WORKSPACE)):
        with pytest.raises(qb.QbertError) as e:
            call()
        assert e.value.status == status
