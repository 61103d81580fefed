"""A fine-tuning step as its calls are used together: quantized embeddings, a linear in 8-bit floating point, dropout with the residual,
the vocabulary loss, and all of it backwards; eager, and captured in a graph with one workspace."""
import numpy as np
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_dropout import words
from test_gpu_fp8 import E4M3, E5M2, check_product, reference, values

pytestmark = pytest.mark.gpu
P_DROP = 0.1


class Step:
    """Two tables, one linear with a residual, a decoder; every buffer of the step is kept."""

    def __init__(self, T, V, D, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.V, self.D = T, V, D
        self.ws = qb.vocab_loss_workspace(T, V, D)
        self.words = qb.quantize_embedding(torch.randn(V, D, device="cuda", generator=g) * 0.05, 4, 16, self.ws)
        self.places = qb.quantize_embedding(torch.randn(512, D, device="cuda", generator=g) * 0.05, 8, 16, self.ws)
        self.w = torch.randn(D, D, device="cuda", generator=g) * 0.05
        self.bias = torch.randn(D, device="cuda", generator=g) * 0.1
        self.decoder = (torch.randn(V, D, device="cuda", generator=g) * 0.1).bfloat16()
        self.out_bias = torch.randn(V, device="cuda", generator=g) * 0.1
        self.ids = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
        self.at = torch.arange(T, device="cuda", dtype=torch.int32) % 512
        self.targets = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
        self.targets[::7] = -100
        self.grad_loss = torch.full((T,), 1.0 / T, device="cuda")
        self.rng = torch.tensor([seed, 40], dtype=torch.int64, device="cuda")

    def run(self):
        ws, D = self.ws, self.D
        x = qb.embedding_lookup(self.ids, *self.words, D, 4, 16, ws)
        qb.embedding_lookup(self.at, *self.places, D, 8, 16, ws, out=x, accumulate=True)
        xq, xs, xqt, xst = qb.quantize_fp8(x, ws, E4M3, transposed=True)
        wq, wsc, wqt, wst = qb.quantize_fp8_weights(self.w, ws, E4M3, transposed=True)
        y = qb.gemm_fp8(xq, xs, wq, wsc, self.bias, ws, torch.float32)
        h = qb.dropout(y, P_DROP, self.rng, 1, residual=x).bfloat16()
        loss, lse = qb.vocab_loss(h, self.decoder, self.out_bias, self.targets, ws)
        dh, dec, db = qb.vocab_loss_backward(h, self.decoder, self.out_bias, self.targets, lse, self.grad_loss, ws)
        dy = qb.dropout(dh, P_DROP, self.rng, 1)
        gq, gs, gqt, gst, dbias = qb.quantize_fp8(dy, ws, E5M2, transposed=True, want_sums=True)
        dx = qb.gemm_fp8(gq, gs, wqt, wst, None, ws, torch.float32)
        dx += dh  # the residual's part
        dw = qb.gemm_fp8(gqt, gst, xqt, xst, None, ws, torch.float32)
        self.rng[1] += 1
        return {"loss": loss, "decoder": dec, "out_bias": db, "x": dx, "w": dw, "bias": dbias}

    def reference(self, offset):
        """The same step in 64 bits, rounded to 8 and 16 bits where the step rounds."""
        def table(t, ids, bits):
            codes, delta, q0 = t
            bit = torch.arange(self.D, device="cuda") * bits
            row = codes[ids.long()].long() & 0xFFFFFFFF
            v = ((row[:, bit // 32] >> (bit % 32)) & (2**bits - 1)).double()  # 4 and 8 bits: no code straddles words
            group = torch.arange(self.D, device="cuda") * 16 // self.D
            return v * delta.double()[group] + q0.double()[group]

        def fp8(v, dtype, rows):
            q, e = reference(v, dtype, rows)
            return (q.view(v.shape[0], -1, 128) * torch.ldexp(torch.ones_like(e, dtype=torch.float64), e)[:, :, None]).view(q.shape)[:, :v.shape[1]]
        n = self.T * self.D
        seed = int(self.rng[0])
        keep = torch.from_numpy(words(np.arange(n), seed, offset + 1) >= np.uint64(round(P_DROP * 2**32))).cuda().view(self.T, self.D)
        x = table(self.words, self.ids, 4) + table(self.places, self.at, 8)
        y = fp8(x, E4M3, 1) @ fp8(self.w.double(), E4M3, 128).t() + self.bias.double()
        h = (keep * y / (1 - P_DROP) + x).bfloat16().double()
        z = h @ self.decoder.double().t() + self.out_bias.double()
        valid = self.targets >= 0
        lse = torch.logsumexp(z, 1)
        at = self.targets.clamp(min=0).long()[:, None]
        loss = torch.where(valid, lse - z.gather(1, at)[:, 0], 0.0)
        g = torch.softmax(z, 1) - torch.zeros_like(z).scatter_(1, at, 1.0)
        g = g * (self.grad_loss.double() * valid)[:, None]
        dh = (g @ self.decoder.double()).bfloat16().double()
        dy = (keep * dh / (1 - P_DROP)).bfloat16().double()
        dx = fp8(dy, E5M2, 1) @ fp8(self.w.double(), E4M3, 128) + dh
        dw = fp8(dy.t().contiguous(), E5M2, 1) @ fp8(x.t().contiguous(), E4M3, 1).t()
        return {"loss": loss, "decoder": g.t() @ h, "out_bias": g.sum(0), "x": dx, "w": dw, "bias": dy.sum(0)}


@pytest.mark.parametrize("T,V,D", [(70, 1000, 256), (300, 3001, 384)])
def test_step(T, V, D):
    """Relative to the norm of each result.  The step and its 64-bit form round to 8 and 16 bits at the same places; they differ by
    fp32 arithmetic (some 2^-20), by g in bfloat16 (2^-8 of each term at most, on the way to dh and the decoder's gradient), and
    where a value lies so near the border of two codes that these differences decide: then by a step, 2^-2 (e5m2) of the value at
    most.  With differences of 2^-8 that happens to one value in 2^-8 / 2^-2 = 2^-6 of the gradient's codes, 2^-3 * 2^-2 = 2^-5 of
    the norm; two such roundings and g's: 0.08 bounds them all; the loss and the output bias have no such rounding but h's in
    bfloat16 (one value in 2^-20 / 2^-8 = 2^-12 off by 2^-8: 2^-14 of the norm), which 2^-10 bounds."""
    step = Step(T, V, D, seed=3)
    got, want = step.run(), step.reference(40)
    assert qb.read_status(step.ws) == qb.QB_OK
    for name, bound in (("loss", 2.0**-10), ("out_bias", 2.0**-10), ("decoder", 0.08), ("x", 0.08), ("w", 0.08), ("bias", 0.08)):
        off = float((got[name].double() - want[name]).norm() / want[name].norm())
        assert off <= bound, (name, off)


def test_captured_step():
    """Replays read the buffers as they are then, draw a new mask each, and equal the eager step bit for bit."""
    step = Step(200, 2000, 256, seed=5)
    step.run()
    torch.cuda.synchronize()
    step.rng[1] = 40
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step.run()
    step.rng[1] = 40
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in range(3):
        step.ids.copy_(torch.randint(0, step.V, (step.T,), device="cuda", generator=g, dtype=torch.int32))
        step.w.mul_(1.01)
        graph.replay()
        assert int(step.rng[1]) == 41 + k
        kept = {n: t.clone() for n, t in captured.items()}
        step.rng[1] = 40 + k
        eager = step.run()
        for n in kept:
            assert torch.equal(kept[n], eager[n]), n
    assert qb.read_status(step.ws) == qb.QB_OK


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("clipped", [False, True])
def test_fake_quantized_linear(bits, clipped):
    """Quantization-aware training of one linear: Q(W) by the library's quantizer, its products in 8 bits, the gradient back through the
    straight-through estimator.  The forward product reads Q(W) rounded once more, to e4m3: by 2^-4 of a value at most, or, below the
    least normal code, by 2^-10 of a unit of 2^e, where 448 * 2^e is less than twice the block's maximum."""
    M, N, K, groups = 613, 264, 384, 11
    g = torch.Generator(device="cuda").manual_seed(bits)
    x, w = torch.randn(M, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g) * 0.05
    dy = (torch.randn(M, N, device="cuda", generator=g) * 1e-4).bfloat16()
    lo = hi = None
    if clipped:
        lo, hi = torch.full((groups,), -0.08, device="cuda"), torch.full((groups,), 0.09, device="cuda")
    ws = qb.workspace(groups=groups)
    wq, delta, _ = qb.fake_quantize_weights(w, bits, groups, ws, lo, hi)
    q, s, qt, st = qb.quantize_fp8_weights(wq, ws, E4M3, transposed=True)
    codes = values(q, s)[:, :K]
    top = wq.abs().max().double()
    assert ((codes - wq.double()).abs() <= wq.double().abs() * 2.0**-4 + 2.0**-10 * top / 224).all()
    xq, xs, xqt, xst = qb.quantize_fp8(x, ws, E4M3, transposed=True)
    y = qb.gemm_fp8(xq, xs, q, s, None, ws, torch.float32)
    check_product(y, xq, xs, q, s, None, torch.float32)
    gq, gs, gqt, gst = qb.quantize_fp8(dy, ws, E5M2, transposed=True)
    dx = qb.gemm_fp8(gq, gs, qt, st, None, ws, torch.float32)
    check_product(dx, gq, gs, qt, st, None, torch.float32)
    dwq = qb.gemm_fp8(gqt, gst, xqt, xst, None, ws, torch.float32)
    check_product(dwq, gqt, gst, xqt, xst, None, torch.float32)
    dw = qb.ste_backward(dwq, w, groups, lo, hi)
    inside = (w >= -0.08 if clipped else w == w) & (w <= 0.09 if clipped else w == w)
    assert torch.equal(dw, torch.where(inside, dwq, torch.zeros_like(dwq))) and bool(inside.all()) != clipped
    assert qb.read_status(ws) == qb.QB_OK
