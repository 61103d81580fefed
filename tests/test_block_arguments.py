"""What the calls of an encoder block in fine-tuning refuse on the host, before anything is launched (fake addresses, no GPU)."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from paper_1909_05840_b200 import build as qb_build

A = 0x1000


@pytest.fixture(scope="module")
def lib():
    qb_build.build()
    return qb.lib()


def test_layer_norm(lib):
    ok = dict(x=A, type=0, gamma=A, beta=A, eps=1e-12, M=8, D=100, y=A, mean=A, rstd=A)

    def call(**kw):
        return lib.qb_layer_norm(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(M=0), dict(D=0), dict(M=(1 << 24) + 1), dict(D=65537), dict(type=3), dict(type=-1),
                dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert call(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(x=A + 2), dict(y=A + 1), dict(type=2, x=A + 1), dict(gamma=A + 2), dict(beta=A + 2), dict(mean=A + 2), dict(rstd=A + 1)):
        assert call(**bad) == qb.QB_ERR_ALIGN, bad
    assert b"qb_layer_norm" in lib.qb_last_error()
    need = qb.layer_norm_workspace_bytes(1000, 100)
    assert need >= 1024 + 320 * 800 and qb.layer_norm_workspace_bytes(3, 100) >= 1024 + 3 * 800 and qb.layer_norm_workspace_bytes(3, 9000) >= 1024 + 3 * 72000
    assert qb.layer_norm_workspace_bytes(0, 8) == 0 and qb.layer_norm_workspace_bytes(8, 65537) == 0
    ok = dict(gy=A, x=A, type=1, gamma=None, mean=A, rstd=A, M=1000, D=100, gx=A, gg=A, gb=A, ws=A, ws_bytes=need)

    def back(**kw):
        return lib.qb_layer_norm_backward(*{**ok, **kw}.values(), None)
    for bad in (dict(gy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(gx=None), dict(M=0), dict(D=-1), dict(type=3)):
        assert back(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(gy=A + 1), dict(x=A + 1), dict(gx=A + 1), dict(type=0, x=A + 2), dict(gamma=A + 1), dict(mean=A + 2), dict(rstd=A + 2), dict(gg=A + 2), dict(gb=A + 2)):
        assert back(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=A + 8), dict(ws_bytes=need - 1)):
        assert back(**bad) == qb.QB_ERR_WORKSPACE, bad


def test_checkpoint(lib):
    ok = dict(x=A, type=0, M=8, K=100, codes=A, scales=A)

    def save(**kw):
        return lib.qb_checkpoint(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(M=0), dict(K=0), dict(type=3), dict(M=(1 << 34) + 1, K=1), dict(M=1 << 34, K=65),
                dict(M=1, K=(1 << 40) + 1), dict(M=1 << 62, K=1 << 62)):
        assert save(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(x=A + 2), dict(type=1, x=A + 1), dict(codes=A + 8), dict(scales=A + 2)):
        assert save(**bad) == qb.QB_ERR_ALIGN, bad
    ok2 = dict(codes=A, scales=A, M=8, K=100, activation=1, type=0, y=A)

    def restore(**kw):
        return lib.qb_restore(*{**ok2, **kw}.values(), None)
    for bad in (dict(codes=None), dict(scales=None), dict(y=None), dict(M=0), dict(activation=2), dict(activation=-1), dict(type=3)):
        assert restore(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(codes=A + 1), dict(scales=A + 2), dict(y=A + 2)):
        assert restore(**bad) == qb.QB_ERR_ALIGN, bad
    ok3 = dict(gy=A, type=1, pre=None, codes=A, scales=A, M=8, K=100, gx=A)

    def back(**kw):
        return lib.qb_gelu_backward(*{**ok3, **kw}.values(), None)
    for bad in (dict(gy=None), dict(gx=None), dict(codes=None), dict(scales=None), dict(pre=A), dict(pre=A, codes=None), dict(pre=A, scales=None), dict(codes=None, scales=None),
                dict(M=-1), dict(type=-1)):
        assert back(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(gy=A + 1), dict(gx=A + 1), dict(codes=A + 4), dict(scales=A + 1), dict(pre=A + 1, codes=None, scales=None)):
        assert back(**bad) == qb.QB_ERR_ALIGN, bad


def test_linear(lib):
    need = qb.linear_workspace_bytes(100, 90, 33)
    # rows of 33 and of 90 elements are copied to rows of 40 and 96
    assert need >= 1024 + 100 * 80 + 90 * 80 + 100 * 192 + 4 * 90
    assert qb.linear_workspace_bytes(0, 8, 8) == 0 and qb.linear_workspace_bytes(8, (1 << 24) + 1, 8) == 0
    assert qb.linear_form(0, 8, 8) == (0, 0, 0, 0) and qb.linear_form(1 << 24, 1 << 24, 8)[1] == 0
    ok = dict(x=A, w=A, type=1, bias=A, act=1, residual=A, M=8, N=16, K=32, out=1, y=A, pre=A, codes=None, scales=None, ws=A, ws_bytes=1 << 20)

    def call(**kw):
        return lib.qb_linear(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(type=0), dict(type=3), dict(out=2), dict(out=3), dict(out=0), dict(act=2), dict(act=-1), dict(M=0), dict(N=0),
                dict(K=0), dict(M=(1 << 24) + 1), dict(M=1 << 24, N=1 << 24), dict(codes=A, scales=A), dict(pre=None, codes=A), dict(pre=None, scales=A),
                dict(pre=None, codes=A, scales=A, out=0)):
        assert call(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(x=A + 8), dict(w=A + 2), dict(bias=A + 2), dict(residual=A + 1), dict(y=A + 1), dict(pre=A + 1), dict(pre=None, out=0, y=A + 2),
                dict(pre=None, out=0, residual=A + 2), dict(pre=None, codes=A, scales=A + 2)):
        assert call(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=A + 8), dict(ws_bytes=255)):
        assert call(**bad) == qb.QB_ERR_WORKSPACE, bad
    assert b"qb_linear" in lib.qb_last_error()
    okx = dict(gy=A, w=A, type=2, pre=A, codes=None, scales=None, residual=None, M=8, N=16, K=32, gx=A, ws=A, ws_bytes=1 << 20)

    def grad_x(**kw):
        return lib.qb_linear_grad_x(*{**okx, **kw}.values(), None)
    for bad in (dict(gy=None), dict(w=None), dict(gx=None), dict(type=0), dict(M=0), dict(N=-1), dict(K=0), dict(codes=A, scales=A), dict(pre=None, codes=A), dict(residual=A),
                dict(pre=None, codes=A, scales=A, residual=A)):
        assert grad_x(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(gy=A + 8), dict(w=A + 8), dict(pre=A + 1), dict(gx=A + 1), dict(pre=None, residual=A + 1), dict(pre=None, codes=A, scales=A + 2)):
        assert grad_x(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=A + 4), dict(ws_bytes=8)):
        assert grad_x(**bad) == qb.QB_ERR_WORKSPACE, bad
    okw = dict(gy=A, x=A, type=1, M=8, N=16, K=32, out=0, gw=A, gb=A, ws=A, ws_bytes=1 << 20)

    def grad_w(**kw):
        return lib.qb_linear_grad_w(*{**okw, **kw}.values(), None)
    for bad in (dict(gy=None), dict(x=None), dict(gw=None, gb=None), dict(type=0), dict(out=2), dict(M=0), dict(N=0), dict(K=0)):
        assert grad_w(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(gy=A + 8), dict(x=A + 8), dict(gw=A + 2), dict(out=1, gw=A + 1), dict(gb=A + 2)):
        assert grad_w(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=A + 4), dict(ws_bytes=8)):
        assert grad_w(**bad) == qb.QB_ERR_WORKSPACE, bad


def test_forms(lib):
    """Every form serves some shape, with 148 SMs: the GPU tests' shapes are among these."""
    ws = 1 << 28
    forms = [qb.linear_form(*s, ws) for s in ((32, 768, 768), (613, 2304, 768), (5003, 768, 768), (24576, 4096, 1024), (5003, 2304, 768))]
    assert {f[:2] for f in forms} == {(128, 64), (128, 128), (256, 128), (256, 256)} and any(f[2] > 0 for f in forms)
    assert qb.linear_form(1024, 1024, 24576, ws)[3] > 1 and qb.linear_form(1024, 1024, 24576, 0)[3] == 1


def test_names_and_buffers_that_are_refused():
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    calls = (lambda: qb.linear(x, x, None, None, activation="relu"), lambda: qb.linear(x, x, None, None, save="all"), lambda: qb.linear(x, x, None, None, pre=x),
             lambda: qb.linear(x, x, None, None, save="pre", saved=(x, x)), lambda: qb.linear(x, x, None, None, out_dtype=torch.float16),
             lambda: qb.linear_grad_w(x, x, None, out_dtype=torch.float16), lambda: qb.linear_grad_w(x, x, None, needs=(False, True), grad_w=x),
             lambda: qb.linear_grad_w(x, x, None, needs=(True, False), grad_bias=x), lambda: qb.restore((x, x), torch.float64), lambda: qb.restore((x, x), activation="tanh"),
             lambda: qb.layer_norm(x, None, None, mean=x), lambda: qb.layer_norm_backward(x, x, None, x, x, x, grad_gamma=x, need_weights=False))
    for call in calls:
        with pytest.raises(qb.QbertError) as e:
            call()
        assert e.value.status == qb.QB_ERR_INVALID


def test_no_cpu_fallback(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    assert lib.qb_layer_norm(A, 0, None, None, 0.0, 8, 8, A, None, None, None) == qb.QB_ERR_CUDA
    assert lib.qb_checkpoint(A, 0, 8, 8, A, A, None) == qb.QB_ERR_CUDA
    assert lib.qb_linear(A, A, 1, None, 0, None, 8, 8, 8, 1, A, None, None, None, A, 1024, None) == qb.QB_ERR_CUDA
