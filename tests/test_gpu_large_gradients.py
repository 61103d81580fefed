"""Gradients of weights and biases over more than 2^32 bytes of rows: whole numbers, whose sums are exact, so that every row counts."""
import pytest
import torch

import paper_1909_05840_b200 as qb

pytestmark = pytest.mark.gpu
PART = 1 << 16


def whole(seed, M, N, low, high, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(M, N, dtype=dtype, device="cuda")
    for m in range(0, M, PART):
        rows = min(PART, M - m)
        out[m:m + rows] = torch.randint(low, high + 1, (rows, N), device="cuda", generator=g, dtype=torch.int8).to(dtype)
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,K", [(4096, 64), (4099, 24)])
def test_linear(N, K, dtype):
    M = (1 << 31) // N + 300
    ws = torch.zeros(qb.linear_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    dy, x = whole(1, M, N, -1, 1, dtype), whole(2, M, K, -1, 1, dtype)
    want, bias = torch.zeros(N, K, device="cuda"), torch.zeros(N, device="cuda")
    for m in range(0, M, PART):
        want += dy[m:m + PART].float().t() @ x[m:m + PART].float()
        bias += dy[m:m + PART].float().sum(0)
    dw, db = qb.linear_grad_w(dy, x, ws)
    assert torch.equal(dw, want) and torch.equal(db, bias)
    w = whole(3, N, K, -1, 1, dtype)
    dx = qb.linear_grad_x(dy, w, ws)
    for m in (0, M // 2, M - 300):
        assert torch.equal(dx[m:m + 300], (dy[m:m + 300].float() @ w.float()).to(dtype))
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("D", [1024, 1023, 9000])
def test_layer_norm(D):
    """With mean 0 and rstd 1 given, xhat is x."""
    M = (1 << 31) // D + 77
    dy, x = whole(4, M, D, -1, 1, torch.float16), whole(5, M, D, -2, 2, torch.float16)
    ws = torch.zeros(qb.layer_norm_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    gamma, beta = torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
    for m in range(0, M, PART):
        gamma += (dy[m:m + PART].float() * x[m:m + PART].float()).sum(0)
        beta += dy[m:m + PART].float().sum(0)
    _, dgamma, dbeta = qb.layer_norm_backward(dy, x, None, torch.zeros(M, device="cuda"), torch.ones(M, device="cuda"), ws)
    assert torch.equal(dgamma, gamma) and torch.equal(dbeta, beta)
