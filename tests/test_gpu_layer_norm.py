"""Layer norm, forward and backward, against 64 bits and against differences."""
import pytest
import torch

import paper_1909_05840_b200 as qb

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-12


@pytest.fixture(scope="module")
def ws():
    return qb.linear_workspace(4096, 4096, 4096)


def half(t):
    return torch.finfo(t).eps / 2


def least(t):
    """Half a step of the type's subnormals."""
    return 2.0**-25 if t == torch.float16 else 2.0**-133 if t == torch.bfloat16 else 2.0**-149


def forward64(x, gamma, beta, eps=EPS):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    xhat = (x - mean) * rstd
    g = 1.0 if gamma is None else gamma.double()
    return xhat * g + (0.0 if beta is None else beta.double()), mean, rstd, xhat


def check_forward(y, x, gamma, beta, mean, rstd, eps=EPS):
    """A lane adds up to 32 elements, or, in rows beyond 8,192, D / 256, the lanes and warps another 13 in a tree: the mean is off by at most
    n = 32 (D / 256) + 13 roundings of the row's mean magnitude a, so is the sum of squares by n + 2 of itself, twice the mean's error
    of a deviation each.  rstd: half of that, and three roundings more.  y: the deviation's error (the mean's and a rounding of x - mean),
    rstd's and four roundings of the terms, and the type's own."""
    want, m64, r64, xhat = forward64(x, gamma, beta, eps)
    D, u = x.shape[1], 2.0**-24
    n = (32 if D <= 8192 else D / 256 + 1) + 13
    a = x.double().abs().mean(1, keepdim=True)
    e_mean = n * u * a + u * m64.abs()
    e_rstd = r64 * ((n + 6) * u + e_mean * r64)
    g = torch.ones(D, device="cuda", dtype=torch.float64) if gamma is None else gamma.double().abs()
    b = 0.0 if beta is None else beta.double().abs()
    e_y = g * (r64 * e_mean + xhat.abs() * (e_rstd / r64 + 4 * u)) + u * (want.abs() + b)
    e_y = e_y * 1.01 + want.abs() * half(y.dtype) * 1.01 + least(y.dtype)
    assert ((y.double() - want).abs() <= e_y).all()
    if mean is not None:
        assert ((mean.double() - m64[:, 0]).abs() <= 1.01 * e_mean[:, 0]).all()
        assert ((rstd.double() - r64[:, 0]).abs() <= 1.01 * e_rstd[:, 0]).all()


def data(M, D, t, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(M, D, device="cuda", generator=g) * 2 + torch.randn(1, D, device="cuda", generator=g)).to(t)
    gamma = 1 + 0.3 * torch.randn(D, device="cuda", generator=g)
    beta = 0.2 * torch.randn(D, device="cuda", generator=g)
    dy = torch.randn(M, D, device="cuda", generator=g).to(t)
    return x, gamma, beta, dy


def check_backward(got, dy, x, gamma, mean, rstd):
    """From the statistics as they were given.  The two means of a row: n roundings of the mean magnitudes of their terms, and three of
    each term; grad_x three more and the type's.  The columns' sums: a chain of at most (rows of a block) + 8 + (blocks / 8) + 8
    additions of terms with three roundings."""
    dx, dgamma, dbeta = got
    M, D, u = *x.shape, 2.0**-24
    g64, m, r = dy.double(), mean.double()[:, None], rstd.double()[:, None]
    xhat = (x.double() - m) * r
    e_xhat = 3 * u * xhat.abs()
    gw = g64 if gamma is None else g64 * gamma.double()
    s, sx = gw.mean(1, keepdim=True), (gw * xhat).mean(1, keepdim=True)
    want = r * (gw - s - xhat * sx)
    n = (32 if D <= 8192 else D / 256 + 1) + 13
    a, ax = gw.abs().mean(1, keepdim=True), (gw * xhat).abs().mean(1, keepdim=True)
    e = r * ((n + 3) * u * a + xhat.abs() * (n + 6) * u * ax + 4 * u * (gw.abs() + s.abs() + (xhat * sx).abs()) + e_xhat * sx.abs())
    e = 1.01 * e + want.abs() * half(dx.dtype) * 1.01 + least(dx.dtype)
    assert ((dx.double() - want).abs() <= e).all()
    chain = M / 100 + 120  # rows of a block over 148 blocks of one row at a time, and the joins
    if dgamma is not None:
        assert ((dgamma.double() - (g64 * xhat).sum(0)).abs() <= 1.01 * u * (chain + 4) * (g64 * xhat).abs().sum(0) + 1e-40).all()
    if dbeta is not None:
        assert ((dbeta.double() - g64.sum(0)).abs() <= 1.01 * u * chain * g64.abs().sum(0) + 1e-40).all()


SIZES = [(1, 1), (3, 2), (2, 7), (7, 8), (1, 768), (37, 100), (9, 768), (33, 1023), (40, 1024), (5, 1025), (6, 1032), (17, 2047), (19, 2048), (4, 2056), (3, 4095),
         (21, 4096), (5, 4104), (2, 8191), (3, 8192), (2, 8193), (3, 8200), (2, 20001), (2, 65536), (2500, 64), (5003, 768)]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,D", SIZES)
def test_both_passes(M, D, kind, ws):
    x, gamma, beta, dy = data(M, D, TYPES[kind], seed=M + D)
    buffer = torch.full((M * D + 64,), 7.0, dtype=x.dtype, device="cuda")
    y, mean, rstd = qb.layer_norm(x, gamma, beta, 1e-5, want_stats=True, y=buffer[:M * D].view(M, D))
    assert (buffer[M * D:] == 7.0).all()
    check_forward(y, x, gamma, beta, mean, rstd, 1e-5)
    assert torch.equal(qb.layer_norm(x, gamma, beta, 1e-5), y)
    buffer.fill_(7.0)
    got = qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws, grad_x=buffer[:M * D].view(M, D))
    assert (buffer[M * D:] == 7.0).all()
    check_backward(got, dy, x, gamma, mean, rstd)
    again = qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("D", [96, 768, 2049])
def test_without_weights_and_in_place(D, kind, ws):
    M = 41
    x, gamma, beta, dy = data(M, D, TYPES[kind])
    y, mean, rstd = qb.layer_norm(x, None, None, EPS, want_stats=True)
    check_forward(y, x, None, None, mean, rstd)
    check_forward(qb.layer_norm(x, gamma, None, EPS), x, gamma, None, None, None)
    check_forward(qb.layer_norm(x, None, beta, EPS), x, None, beta, None, None)
    z = x.clone()
    assert qb.layer_norm(z, None, None, EPS, y=z) is z and torch.equal(z, y)
    got = qb.layer_norm_backward(dy, x, None, mean, rstd, ws)
    check_backward(got, dy, x, None, mean, rstd)
    only = qb.layer_norm_backward(dy, x, None, mean, rstd, ws[:256], need_weights=False)
    assert only[1] is None and only[2] is None and torch.equal(only[0], got[0])
    for alias in (dy.clone(), x.clone()):
        a, b = (alias, x) if torch.equal(alias, dy) else (dy, alias)
        assert torch.equal(qb.layer_norm_backward(a, b, None, mean, rstd, ws, grad_x=alias)[0], got[0])


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_any_alignment(kind, shift, ws):
    """Arrays that begin anywhere: the bounds of aligned ones."""
    M, D = 13, 768
    x, gamma, beta, dy = data(M, D, TYPES[kind])

    def moved(t):
        b = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
        b[shift:shift + t.numel()] = t.reshape(-1)
        return b[shift:shift + t.numel()].view(t.shape)
    xs, gs, bs = moved(x), moved(gamma), moved(beta)
    y, mean, rstd = qb.layer_norm(xs, gs, bs, EPS, want_stats=True, y=moved(x))
    check_forward(y, x, gamma, beta, mean, rstd)
    got = qb.layer_norm_backward(moved(dy), xs, gs, mean, rstd, ws, grad_x=moved(x), grad_gamma=moved(gamma), grad_beta=moved(beta))
    check_backward(got, dy, x, gamma, mean, rstd)
    y = qb.layer_norm(x, gs, beta, EPS)  # rows aligned, weights not
    check_forward(y, x, gamma, beta, None, None)


@pytest.mark.parametrize("offset", [0.0, 1000.0])
def test_far_mean_and_constant_rows(offset, ws):
    """The variance is of the deviations: a mean a thousand deviations away costs what its rounding does; a row of one value gives beta."""
    M, D = 11, 768
    x = torch.randn(M, D, device="cuda") + offset
    x[3] = 5.0
    gamma, beta = torch.full((D,), 1.5, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = qb.layer_norm(x, gamma, beta, 1e-3, want_stats=True)
    check_forward(y, x, gamma, beta, mean, rstd, 1e-3)
    assert torch.equal(y[3], beta)


@pytest.mark.parametrize("D", [768, 3000, 9000])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_not_finite(bad, D, ws):
    """Such a row is NaN; the others, and grad_beta, are as they were."""
    x, gamma, beta, dy = data(6, D, torch.float32)
    clean = qb.layer_norm(x, gamma, beta, EPS)
    x[2, D // 2] = bad
    y, mean, rstd = qb.layer_norm(x, gamma, beta, EPS, want_stats=True)
    keep = torch.arange(6, device="cuda") != 2
    assert y[2].isnan().all() and torch.equal(y[keep], clean[keep])
    dx, dgamma, dbeta = qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws)
    assert dx[2].isnan().all() and dx[keep].isfinite().all() and dgamma.isnan().all() and dbeta.isfinite().all()


def test_gradients_against_differences(ws):
    """Central differences of the 64-bit forward pass in random directions; h = 2^-10 leaves an error of h^2 times the third derivative,
    which rows of variance 4 keep below 2^-20 of the terms' magnitudes (bounded by their sum); the passes' own 2^-20 comes on top."""
    M, D = 5, 96
    x, gamma, beta, dy = data(M, D, torch.float32)
    _, mean, rstd = qb.layer_norm(x, gamma, beta, EPS, want_stats=True)
    dx, dgamma, dbeta = qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws)
    h = 2.0**-10

    def loss(x, gamma, beta):
        return (forward64(x, gamma, beta)[0] * dy.double()).sum()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for i, (leaf, grad) in enumerate(((x, dx), (gamma, dgamma), (beta, dbeta))):
            v = torch.randn(leaf.shape, device="cuda", generator=g, dtype=torch.float64)
            args = [[x.double(), gamma.double(), beta.double()] for _ in range(2)]
            args[0][i] = args[0][i] + h * v
            args[1][i] = args[1][i] - h * v
            quotient = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert (quotient - (grad.double() * v).sum()).abs() <= 2.0**-18 * (dy.double().abs().sum() + (grad.double() * v).abs().sum())


def test_offsets_beyond_32_bits(ws):
    """More than 2^32 bytes of rows; the last and the first rows are right and the rows between were written."""
    M, D = (1 << 31) // 1024 + 77, 1024
    x = torch.randn(1024, D, device="cuda").half().repeat((M + 1023) // 1024, 1)[:M].contiguous()
    gamma, beta = torch.rand(D, device="cuda"), torch.rand(D, device="cuda")
    y, mean, rstd = qb.layer_norm(x, gamma, beta, EPS, want_stats=True)
    for part in (slice(0, 1024), slice(M - 77, M)):
        check_forward(y[part], x[part], gamma, beta, mean[part], rstd[part])
    assert torch.equal(y[:1024], y[1024 * 1000:1024 * 1001]) and torch.equal(y[:77], y[-77:])
    dx, dgamma, dbeta = qb.layer_norm_backward(y, x, gamma, mean, rstd, ws)
    dx0, _, _ = qb.layer_norm_backward(y[:77], x[:77], gamma, mean[:77], rstd[:77], ws)
    assert torch.equal(dx[:77], dx0) and torch.equal(dx[-77:], dx0) and dgamma.isfinite().all()


def test_refusals(ws):
    x, gamma, beta, dy = data(8, 768, torch.bfloat16)
    _, mean, rstd = qb.layer_norm(x, gamma, beta, want_stats=True)
    for call in (lambda: qb.layer_norm(x.t(), gamma, beta), lambda: qb.layer_norm(x, gamma.bfloat16(), beta), lambda: qb.layer_norm(x, gamma[:-1], beta),
                 lambda: qb.layer_norm(x.double(), gamma, beta), lambda: qb.layer_norm(x[None], gamma, beta), lambda: qb.layer_norm(x.cpu(), gamma, beta),
                 lambda: qb.layer_norm(x, gamma, beta, y=x[:4]), lambda: qb.layer_norm(x, gamma, beta, y=torch.empty(8, 768, device="cuda")),
                 lambda: qb.layer_norm_backward(dy, x.float(), gamma, mean, rstd, ws), lambda: qb.layer_norm_backward(dy, x[:4], gamma, mean, rstd, ws),
                 lambda: qb.layer_norm_backward(dy, x, gamma, mean[:4], rstd, ws), lambda: qb.layer_norm_backward(dy, x, gamma, mean, None, ws)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(qb.QbertError) as e:
        qb.layer_norm_backward(dy, x, gamma, mean, rstd, ws[:1024])
    assert e.value.status == qb.QB_ERR_WORKSPACE
    with pytest.raises(qb.QbertError) as e:
        qb.layer_norm(x, gamma, beta, -1.0)
    assert e.value.status == qb.QB_ERR_INVALID
