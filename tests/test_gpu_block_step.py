"""The feed-forward half of an encoder layer in a training step, as its calls are used together: two linears with GELU between them and the
residual behind, dropout, a layer norm, and all of it backwards, with the pre-activation saved in 16 or in 8 bits; eager, captured,
on another stream and beside another step."""
import threading

import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_checkpoint import gelu64, slope64, values64
from test_gpu_fewer_sms import in_part, part  # noqa: F401 (a fixture)
from test_gpu_layer_norm import forward64

pytestmark = pytest.mark.gpu
EPS = 1e-12


class Block:
    def __init__(self, T, D, F, seed, dtype=torch.bfloat16, save="codes"):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, device="cuda", generator=g)
        self.save, self.dtype = save, dtype
        self.x = randn(T, D).to(dtype)
        self.w1, self.w2 = (randn(F, D) * 0.05).to(dtype), (randn(D, F) * 0.05).to(dtype)
        self.b1, self.b2 = randn(F) * 0.1, randn(D) * 0.1
        self.gamma, self.beta = 1 + 0.2 * randn(D), 0.1 * randn(D)
        self.dy = randn(T, D).to(dtype)
        self.ws = qb.linear_workspace(T, F, D)
        self.norm_ws = torch.zeros(qb.layer_norm_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")

    def run(self):
        ws = self.ws
        h, saved = qb.linear(self.x, self.w1, self.b1, ws, activation="gelu", save=self.save)
        s = qb.linear(h, self.w2, self.b2, ws, residual=self.x)
        y, mean, rstd = qb.layer_norm(s, self.gamma, self.beta, EPS, want_stats=True)
        ds, dgamma, dbeta = qb.layer_norm_backward(self.dy, s, self.gamma, mean, rstd, self.norm_ws)
        if self.save == "codes":
            h = qb.restore(saved, self.dtype, activation="gelu")  # formed anew: h need not be kept
        dw2, db2 = qb.linear_grad_w(ds, h, ws)
        dz = qb.linear_grad_x(ds, self.w2, ws, through=saved)
        dw1, db1 = qb.linear_grad_w(dz, self.x, ws)
        dx = qb.linear_grad_x(dz, self.w1, ws, residual=ds)
        return {"y": y, "dgamma": dgamma, "dbeta": dbeta, "w2": dw2, "b2": db2, "w1": dw1, "b1": db1, "x": dx}

    def reference(self, rounded=True):
        """The same in 64 bits, rounded where a tensor of the step is."""
        def t(v):
            return v.to(self.dtype).double() if rounded else v
        x, w1, w2 = self.x.double(), self.w1.double(), self.w2.double()
        z = x @ w1.t() + self.b1.double()
        h = t(gelu64(z))
        s = t(h @ w2.t() + self.b2.double() + x)
        y, _, rstd, xhat = forward64(s, self.gamma, self.beta)
        g = self.dy.double() * self.gamma.double()
        ds = t(rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)))
        p = t(z) if self.save == "pre" else values64(*qb.checkpoint(z.float()))
        hb = h if self.save == "pre" else t(gelu64(p))
        dz = t((ds @ w2) * slope64(p))
        return {"y": y, "dgamma": (self.dy.double() * xhat).sum(0), "dbeta": self.dy.double().sum(0), "w2": ds.t() @ hb, "b2": ds.sum(0),
                "w1": dz.t() @ x, "b1": dz.sum(0), "x": dz @ w1 + ds}


def off(got, want):
    return {k: float((got[k].double() - want[k]).norm() / want[k].norm()) for k in want}


@pytest.mark.parametrize("save", ["pre", "codes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,F", [(1, 64, 128), (70, 96, 264), (613, 768, 1030), (5003, 256, 1024)])
def test_step(T, D, F, dtype, save):
    """Relative to the norm of each result: both sides round at the same places, so that they differ by fp32 arithmetic (2^-20) and by a step
    of the type (eps, or 1 / 127 of a block's maximum, a fifth of its norm's share per value or so) where a value lies so near to a border
    that this decides: one in 2^-20 / eps (2^-12 for bfloat16) of the values at each of the four tensors between a result and its
    inputs, sqrt(2^-12) * eps of the norm each; 2^-2 of eps bounds them, and the result's own rounding is eps / 2 at most (dgamma's,
    dbeta's and the biases' is none)."""
    b = Block(T, D, F, T, dtype, save)
    eps = torch.finfo(dtype).eps
    far = off(b.run(), b.reference())
    assert all(v <= eps for v in far.values()), far
    assert qb.read_status(b.ws) == qb.QB_OK


@pytest.mark.parametrize("save", ["pre", "codes"])
def test_gradients_against_differences(save):
    """Central differences of the unrounded step in 64 bits in random directions.  The step's gradients are off by the roundings of what it
    keeps: of relative size eps / 2 a value (bfloat16: 2^-8) in six tensors, and with codes by half a step (1 / 254 of a block's maximum) in the
    slope and in h; the differences' own error is below 2^-16.  Directions are random: the errors add up like the norm of the gradient
    times these, which 2^-4 bounds."""
    b = Block(40, 64, 96, 5, torch.bfloat16, save)
    got = b.run()

    def loss(x, w1, w2, b1, b2, gamma, beta):
        s = gelu64(x @ w1.t() + b1) @ w2.t() + b2 + x
        return (forward64(s, gamma, beta)[0] * b.dy.double()).sum()
    leaves = [t.double() for t in (b.x, b.w1, b.w2, b.b1, b.b2, b.gamma, b.beta)]
    h = 2.0**-12
    for i, name in enumerate(("x", "w1", "w2", "b1", "b2", "dgamma", "dbeta")):
        for seed in range(2):
            v = torch.randn(leaves[i].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed), dtype=torch.float64)
            ends = []
            for sign in (1, -1):
                args = list(leaves)
                args[i] = args[i] + sign * h * v
                ends.append(loss(*args))
            quotient = (ends[0] - ends[1]) / (2 * h)
            assert abs(float(quotient - (got[name].double() * v).sum())) <= 2.0**-4 * float(got[name].double().norm()) * 4


@pytest.mark.parametrize("save", ["pre", "codes"])
def test_captured_step(save):
    """Replays read the buffers as they are then and equal the eager step bit for bit; two graphs over one workspace, replayed in turn, as well."""
    b, other = Block(613, 256, 520, 1, save=save), Block(300, 256, 520, 2, save=save)
    other.ws = b.ws
    other.norm_ws = b.norm_ws
    for block in (b, other):
        block.run()
    torch.cuda.synchronize()
    graphs = []
    for block in (b, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = block.run()
        graphs.append((block, graph, out))
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(3):
        for block, graph, out in graphs:
            block.x.copy_(torch.randn(block.x.shape, device="cuda", generator=g))
            block.w1.mul_(1.01)
            graph.replay()
            kept = {n: t.clone() for n, t in out.items()}
            eager = block.run()
            for n in kept:
                assert torch.equal(kept[n], eager[n]), n
    assert qb.read_status(b.ws) == qb.QB_OK


def test_streams_and_threads():
    """Steps on streams of their own, from threads of their own, with workspaces of their own: each as it is alone."""
    blocks = [Block(613, 256, 520, 3), Block(300, 520, 264, 4, torch.float16), Block(2100, 128, 1024, 5, save="pre")]
    alone = [b.run() for b in blocks]
    torch.cuda.synchronize()
    got = [None] * len(blocks)

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got[i] = blocks[i].run()
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(blocks))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(alone, got):
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_back_to_back():
    """Calls directly behind one another, each reading what the one before wrote, many times: no kernel begins on what is not there yet."""
    b = Block(2500, 768, 1024, 6)
    want = b.run()
    torch.cuda.synchronize()
    for _ in range(20):
        got = b.run()
    for n in want:
        assert torch.equal(got[n], want[n]), n
    # the bias's gradient runs under the product: of a tensor that the kernel before the call wrote, and that the one behind it overwrites
    dy = torch.randn(4000, 1024, device="cuda").bfloat16()
    x = torch.randn(4000, 1024, device="cuda").bfloat16()
    buffer = torch.empty_like(dy)
    dw0, db0 = qb.linear_grad_w(dy, x, b.ws)
    for _ in range(20):
        buffer.copy_(dy)
        dw, db = qb.linear_grad_w(buffer, x, b.ws)
        buffer.fill_(7.0)
        assert torch.equal(db, db0) and torch.equal(dw, dw0)


def test_beside_autograd():
    """Inputs that require gradients are read like others and outputs do not; a step captured while an eager torch graph of the same leaves
    lives leaves that graph as it was."""
    b = Block(64, 64, 128, 7)
    x, w = b.x.float().requires_grad_(), b.w1.float().requires_grad_()
    y = torch.nn.functional.gelu(x @ w.t())
    b.x.requires_grad_()
    b.w1.requires_grad_()
    b.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.run()
    graph.replay()
    assert not any(t.requires_grad for t in out.values())
    y.sum().backward()
    assert x.grad.isfinite().all() and w.grad.isfinite().all()
    assert torch.equal(out["x"], b.run()["x"])


def test_on_a_part_of_the_device(part):  # noqa: F811
    """On a stream that has sixteen SMs the grids, made for the whole device, take turns: the same results."""
    b = Block(2500, 768, 1024, 8)
    want, got = b.run(), {}
    in_part(part, lambda: got.update(b.run()))
    for n in want:
        assert torch.equal(got[n], want[n]), n
    assert qb.read_status(b.ws) == qb.QB_OK
