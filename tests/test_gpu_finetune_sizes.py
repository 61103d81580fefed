"""The calls of a fine-tuning step at sizes whose offsets pass 32 bits, with many tokens, on a part of the device's SMs, and from several
threads."""
import threading

import pytest
import torch

import paper_1909_05840_b200 as qb
import test_gpu_vocab_loss as vl
from test_gpu_fewer_sms import in_part, part  # noqa: F401 (a fixture)
from test_gpu_fp8 import E4M3, check_product, rows_of, unpack, up

pytestmark = pytest.mark.gpu


def test_codes_and_product_beyond_32_bits():
    """More than 2^32 codes: the last rows' codes, and the product that reads them."""
    K, tail = 1024, 300
    M = (1 << 22) + tail + 5
    ws = qb.workspace()
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[-tail:] = rows_of(tail, K, 3, torch.bfloat16)
    x[0] = 1.0
    q, s = qb.quantize_fp8(x, ws)
    del x
    e = unpack(s.view(up(M) // 128, -1, 32, 4, 4)[(M - tail) // 128:], M - (M - tail) // 128 * 128, K // 128)[-tail:]
    ref, ref_s = qb.quantize_fp8(rows_of(tail, K, 3, torch.bfloat16), ws)
    assert torch.equal(q[-tail:].view(torch.uint8), ref.view(torch.uint8)) and torch.equal(e, unpack(ref_s, tail, K // 128))
    b, sb = qb.quantize_fp8(rows_of(40, K, 4), ws)
    y = qb.gemm_fp8(q, s, b, sb, None, ws, torch.float32)
    assert torch.equal(y[-tail:], qb.gemm_fp8(ref, ref_s, b, sb, None, ws, torch.float32)) and (y[1:-tail] == 0).all()
    assert qb.read_status(ws) == qb.QB_OK


def test_output_beyond_32_bits():
    """More than 2^32 outputs: the last rows of a product with 70,000 columns."""
    M, N, K = 62000, 70000, 128
    ws = qb.workspace()
    a, sa = qb.quantize_fp8(rows_of(M, K, 1), ws)
    b, sb = qb.quantize_fp8(rows_of(N, K, 2), ws)
    y = qb.gemm_fp8(a, sa, b, sb, None, ws)
    rows = slice(M - 40, M)
    first = (M - 40) // 128 * 128
    part_s = sa.view(up(M) // 128, -1, 32, 4, 4)[first // 128:].contiguous()
    a_part = a[first:].contiguous()
    want = qb.gemm_fp8(a_part, part_s, b, sb, None, ws)
    assert torch.equal(y[rows], want[-40:])
    check_product(want, a_part, part_s, b, sb, None, torch.bfloat16)


def test_vocabulary_beyond_32_bits():
    """More than 2^32 values of w: loss, lse and the gradients of the first and last words, in 64 bits by chunks of the vocabulary."""
    T, V, D = 3, (1 << 22) + 300, 1024
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for i in range(0, V, 1 << 20):
        w[i:i + (1 << 20)] = torch.randn(min(1 << 20, V - i), D, device="cuda", generator=g).mul_(0.05).bfloat16()
    h = torch.randn(T, D, device="cuda", generator=g).bfloat16()
    targets = torch.tensor([V - 1, 5, V - 200], dtype=torch.int32, device="cuda")
    gl = torch.tensor([0.5, 0.25, 1.0], device="cuda")
    ws = qb.vocab_loss_workspace(T, V, D)
    loss, lse = qb.vocab_loss(h, w, None, targets, ws)
    gh, gw, _ = qb.vocab_loss_backward(h, w, None, targets, lse, gl, ws)
    z = torch.cat([h.double() @ w[i:i + (1 << 18)].double().t() for i in range(0, V, 1 << 18)], dim=1)
    ez = float((h.double().abs().sum(1) * 0.3).max()) * (D / 16 + 16) * 2.0**-23  # |w| < 0.3: six standard deviations
    want = torch.logsumexp(z, 1)
    assert ((lse.double() - want).abs() <= ez + 2.0**-17).all()
    at = targets.long()[:, None]
    assert ((loss.double() - (want - z.gather(1, at)[:, 0])).abs() <= 2 * ez + 2.0**-17).all()
    p = torch.softmax(z, 1)
    p.scatter_add_(1, at, -torch.ones(T, 1, dtype=torch.float64, device="cuda"))
    p *= gl.double()[:, None]
    del z
    for rows in (slice(0, 600), slice(V - 600, V)):
        a, b = gw[rows].double(), p[:, rows].t() @ h.double()
        bound = (p[:, rows].abs().t() @ h.double().abs()) * (2.0**-8 + 4 * ez + 2.0**-15) * 1.01 + b.abs() * 2.0**-8 + 2.0**-126
        assert ((a - b).abs() <= bound).all()
    dh, size = torch.zeros(T, D, dtype=torch.float64, device="cuda"), torch.zeros(T, D, dtype=torch.float64, device="cuda")
    for i in range(0, V, 1 << 18):
        wd = w[i:i + (1 << 18)].double()
        dh += p[:, i:i + (1 << 18)] @ wd
        size += p[:, i:i + (1 << 18)].abs() @ wd.abs()
    # accumulation: a split of at most a few thousand K blocks in a chain of V / 16 additions in all
    assert ((gh.double() - dh).abs() <= size * (2.0**-8 + 4 * ez + (V / 16 + 64) * 2.0**-23 + 2.0**-15) + dh.abs() * 2.0**-8 * 1.01).all()
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("T,V,D", [(70001, 300, 64), (9000, 2000, 8)])
def test_many_tokens(T, V, D):
    vl.check_all(*vl.inputs(T, V, D), qb.vocab_loss_workspace(T, V, D))


def test_on_a_part_of_the_device(part):  # noqa: F811
    ws = qb.vocab_loss_workspace(700, 5000, 256)
    x, w = rows_of(2100, 768, 1), rows_of(2300, 768, 2)
    args = vl.inputs(700, 5000, 256)
    few = vl.inputs(40, 5000, 256)
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda")

    def calls():
        xq, xs = qb.quantize_fp8(x, ws)
        wq, wsc = qb.quantize_fp8_weights(w, ws)
        out = [qb.dropout(x, 0.1, rng), qb.gemm_fp8(xq, xs, wq, wsc, None, ws)]
        for a in (args, few):
            loss, lse = qb.vocab_loss(*a[:4], ws)
            out += [loss, lse, *qb.vocab_loss_backward(*a[:4], lse, a[4], ws)]
        return out
    whole, got = calls(), []
    in_part(part, lambda: got.extend(calls()))
    assert len(got) == len(whole) and all(torch.equal(a, b) for a, b in zip(got, whole))
    assert qb.read_status(ws) == qb.QB_OK


def test_several_threads():
    """Four threads, each with a stream and a workspace of its own, over the same tensors."""
    x, w = rows_of(900, 640, 1), rows_of(520, 640, 2)
    args = vl.inputs(130, 1500, 128)
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda")

    def calls(ws):
        q = qb.quantize_fp8(x, ws, E4M3, True)
        v = qb.quantize_fp8_weights(w, ws)
        loss, lse = qb.vocab_loss(*args[:4], ws)
        return [qb.gemm_fp8(q[0], q[1], *v, None, ws), qb.dropout(x, 0.3, rng, 7), loss, *qb.vocab_loss_backward(*args[:4], lse, args[4], ws)]
    want = calls(qb.vocab_loss_workspace(130, 1500, 128))
    torch.cuda.synchronize()
    failed = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ws = qb.vocab_loss_workspace(130, 1500, 128)
            for _ in range(20):
                got = calls(ws)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)) or qb.read_status(ws) != qb.QB_OK:
                    failed.append(1)
    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
