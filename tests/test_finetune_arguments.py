"""What the calls of a fine-tuning step refuse on the host, before anything is launched (fake addresses, no GPU)."""
import pytest

import paper_1909_05840_b200 as qb
from paper_1909_05840_b200 import build as qb_build

A = 0x1000


@pytest.fixture(scope="module")
def lib():
    qb_build.build()
    return qb.lib()


def test_dropout(lib):
    ok = dict(x=A, type=0, n=64, p=0.1, rng=A, call=0, residual=None, y=A)

    def call(**kw):
        return lib.qb_dropout(*{**ok, **kw}.values(), None)
    for bad in (dict(x=None), dict(y=None), dict(rng=None), dict(n=0), dict(n=-1), dict(n=(1 << 40) + 1), dict(type=3), dict(type=-1), dict(p=1.0),
                dict(p=-1e-9), dict(p=float("nan"))):
        assert call(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(x=A + 2), dict(y=A + 1), dict(residual=A + 2), dict(type=1, x=A + 1), dict(rng=A + 4)):
        assert call(**bad) == qb.QB_ERR_ALIGN, bad
    assert b"qb_dropout" in lib.qb_last_error()


def test_fp8(lib):
    assert qb.fp8_scale_bytes(1, 1) == 512 and qb.fp8_scale_bytes(129, 513) == 4 * 512 and qb.fp8_scale_bytes(128, 512) == 512
    assert qb.fp8_scale_bytes(0, 128) == 0 and qb.fp8_scale_bytes(128, -1) == 0 and qb.fp8_scale_bytes((1 << 24) + 1, 1) == 0
    assert qb.fp8_sums_workspace_bytes(129, 10) == 1024 + 2 * 10 * 4 and qb.fp8_sums_workspace_bytes(0, 1) == 0
    for f in (lib.qb_quantize_fp8, lib.qb_quantize_fp8_weights):
        ok = dict(x=A, type=0, M=8, K=100, format=0, q=A, s=A, qt=A, st=A)
        if f is lib.qb_quantize_fp8:
            ok["sums"] = None
        ok.update(ws=A, ws_bytes=256)

        def call(**kw):
            return f(*{**ok, **kw}.values(), None)
        if f is lib.qb_quantize_fp8:
            assert call(sums=A, qt=None, st=None) == qb.QB_ERR_INVALID
            assert call(sums=A + 2, ws_bytes=4096) == qb.QB_ERR_ALIGN
            assert call(sums=A, ws_bytes=1024 + 399) == qb.QB_ERR_WORKSPACE
        for bad in (dict(x=None), dict(q=None), dict(s=None), dict(qt=None), dict(st=None), dict(M=0), dict(K=0), dict(M=(1 << 24) + 1),
                    dict(K=(1 << 24) + 1), dict(M=1 << 24, K=1 << 24), dict(M=1 << 24, K=1 << 16, qt=None, st=None), dict(type=3), dict(format=2), dict(format=-1)):
            assert call(**bad) == qb.QB_ERR_INVALID, bad
        for bad in (dict(x=A + 2), dict(type=1, x=A + 1), dict(q=A + 8), dict(s=A + 4), dict(qt=A + 1), dict(st=A + 2)):
            assert call(**bad) == qb.QB_ERR_ALIGN, bad
        for bad in (dict(ws=None), dict(ws_bytes=255), dict(ws=A + 2)):
            assert call(**bad) == qb.QB_ERR_WORKSPACE, bad
    ok = dict(a=A, sa=A, fa=0, b=A, sb=A, fb=1, bias=None, M=8, N=9, K=128, out=0, y=A, ws=A, ws_bytes=256)

    def gemm(**kw):
        return lib.qb_gemm_fp8(*{**ok, **kw}.values(), None)
    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(y=None), dict(M=0), dict(N=0), dict(K=0), dict(K=(1 << 24) + 128), dict(M=1 << 24, N=1 << 24), dict(M=1 << 24, K=1 << 24),
                dict(M=(1 << 24) + 1), dict(N=(1 << 24) + 1), dict(fa=2), dict(fb=-1), dict(out=2), dict(out=-1)):
        assert gemm(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(K=130), dict(a=A + 8), dict(b=A + 8), dict(sa=A + 8), dict(sb=A + 8), dict(y=A + 2), dict(out=1, y=A + 1), dict(bias=A + 2)):
        assert gemm(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws_bytes=255), dict(ws=A + 2)):
        assert gemm(**bad) == qb.QB_ERR_WORKSPACE, bad


def test_no_cpu_fallback(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    assert lib.qb_dropout(A, 0, 64, 0.1, A, 0, None, A, None) == qb.QB_ERR_CUDA
    assert lib.qb_quantize_fp8(A, 0, 8, 128, 0, A, A, None, None, None, A, 256, None) == qb.QB_ERR_CUDA
    assert lib.qb_gemm_fp8(A, A, 0, A, A, 0, None, 8, 8, 128, 0, A, A, 256, None) == qb.QB_ERR_CUDA


def test_vocab_loss(lib):
    need = qb.vocab_loss_workspace_bytes(100, 1000, 64)
    assert need > 0 and need % 256 == 0
    assert qb.vocab_loss_workspace_bytes(0, 10, 8) == 0 and qb.vocab_loss_workspace_bytes(1, 10, 8193) == 0
    W = 0x10000
    ok = dict(h=A, w=A, bias=None, targets=A, T=100, V=1000, D=64, loss=A, lse=A, ws=W, ws_bytes=need)

    def call(**kw):
        return lib.qb_vocab_loss(*{**ok, **kw}.values(), None)
    for bad in (dict(h=None), dict(w=None), dict(targets=None), dict(loss=None), dict(lse=None), dict(T=0), dict(V=0), dict(D=0), dict(T=(1 << 24) + 1),
                dict(V=(1 << 24) + 1), dict(D=8200), dict(T=1 << 24, V=1 << 24)):
        assert call(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(D=60), dict(h=A + 8), dict(w=A + 8), dict(bias=A + 2), dict(targets=A + 1), dict(loss=A + 2), dict(lse=A + 2)):
        assert call(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=W + 16), dict(ws_bytes=4096)):
        assert call(**bad) == qb.QB_ERR_WORKSPACE, bad
    ok = dict(h=A, w=A, bias=A, targets=A, lse=A, gl=A, T=100, V=1000, D=64, gh=A, gw=A, gb=A, ws=W, ws_bytes=need)

    def back(**kw):
        return lib.qb_vocab_loss_backward(*{**ok, **kw}.values(), None)
    for bad in (dict(h=None), dict(w=None), dict(targets=None), dict(lse=None), dict(gl=None), dict(gh=None, gw=None, gb=None), dict(T=0), dict(V=-1),
                dict(D=8200)):
        assert back(**bad) == qb.QB_ERR_INVALID, bad
    for bad in (dict(D=60), dict(h=A + 8), dict(w=A + 8), dict(gh=A + 8), dict(gw=A + 8), dict(gb=A + 2), dict(lse=A + 2), dict(gl=A + 2), dict(bias=A + 1),
                dict(targets=A + 2)):
        assert back(**bad) == qb.QB_ERR_ALIGN, bad
    for bad in (dict(ws=None), dict(ws=W + 16), dict(ws_bytes=4096)):
        assert back(**bad) == qb.QB_ERR_WORKSPACE, bad


def test_buffers_of_outputs_that_are_not_computed():
    """A buffer that the call would leave as it was is refused, before anything else is looked at."""
    for call in (lambda: qb.quantize_fp8(None, None, sums=1), lambda: qb.quantize_fp8(None, None, transposed=True, sums=1),
                 lambda: qb.quantize_fp8(None, None, codes_t=1), lambda: qb.quantize_fp8(None, None, scales_t=1),
                 lambda: qb.quantize_fp8_weights(None, None, codes_t=1), lambda: qb.quantize_fp8_weights(None, None, scales_t=1)):
        with pytest.raises(qb.QbertError) as e:
            call()
        assert e.value.status == qb.QB_ERR_INVALID
