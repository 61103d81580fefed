"""The operators of an encoder block in fine-tuning that are not quantized, as cases for timing and for comparing results.

* ``layer_norm``    a layer norm of hidden states, forward, and where asked its backward pass with the gradients of its weights;
* ``linear``        serving: a linear in 16 bits with its bias, and where asked GELU and a residual behind it;
* ``train``         the same linear in a training step: forward, where asked with its pre-activation saved in 16 or in 8 bits, then
                    the gradients of its input, of its weights and of its bias; where the input is GELU of a saved
                    pre-activation, its gradient is taken on through that;
* ``checkpoint``    activations saved in 8 bits (one scale per row and block of 64), restored, and GELU's gradient taken from them.

``run`` computes them in elementary torch operations where ``own`` is false, else through the package.
"""
import math

import torch

own = False

WS_BYTES = 1 << 28  # the workspace that a program keeps for all of its calls
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 64    # values with one scale in an 8-bit checkpoint
EPS = 1e-12   # of BERT's layer norms


def listed():
    return [
        # Hidden states of the last token of 32 sequences: the smallest call, launch latency.
        {"name": "norm_32x768_fp32", "kind": "layer_norm", "M": 32, "D": 768, "type": "fp32", "backward": False},
        # A ragged batch of the large encoder, training.
        {"name": "norm_5003x1024_bf16", "kind": "layer_norm", "M": 5003, "D": 1024, "type": "bf16", "backward": True},
        # 64 x 384 tokens of the large encoder, training: throughput.
        {"name": "norm_24576x1024_fp16", "kind": "layer_norm", "M": 24576, "D": 1024, "type": "fp16", "backward": True},
        # The pooler of a small batch.
        {"name": "linear_m32", "kind": "linear", "M": 32, "N": 768, "K": 768, "type": "bf16", "out": "bf16", "bias": True, "gelu": False, "residual": False},
        # A ragged batch through the attention output with the residual.
        {"name": "linear_m5003_attention", "kind": "linear", "M": 5003, "N": 768, "K": 768, "type": "bf16", "out": "bf16", "bias": True, "gelu": False, "residual": True},
        # The first feed-forward linear of the large encoder at 64 x 384 tokens.
        {"name": "linear_m24576_ffn1", "kind": "linear", "M": 24576, "N": 4096, "K": 1024, "type": "bf16", "out": "bf16", "bias": True, "gelu": True, "residual": False},
        # The second one in half precision with the residual.
        {"name": "linear_m24576_ffn2", "kind": "linear", "M": 24576, "N": 1024, "K": 4096, "type": "fp16", "out": "fp16", "bias": True, "gelu": False, "residual": True},
        # A task head of nine labels in a training step: odd sizes in every product.
        {"name": "train_m613_head9", "kind": "train", "M": 613, "N": 9, "K": 768, "type": "fp16", "gelu": False, "residual": False, "save": "no", "through": "no"},
        # The first feed-forward linear of the large encoder over 16 x 384 tokens, its pre-activation saved in 8 bits.
        {"name": "train_m6144_ffn1", "kind": "train", "M": 6144, "N": 4096, "K": 1024, "type": "bf16", "gelu": True, "residual": False, "save": "codes", "through": "no"},
        # The second one over 64 x 384 tokens, its input's gradient taken on through GELU of what was saved in 8 bits.
        {"name": "train_m24576_ffn2", "kind": "train", "M": 24576, "N": 1024, "K": 4096, "type": "bf16", "gelu": False, "residual": True, "save": "no", "through": "codes"},
        # A pre-activation of 32 x 128 tokens of the base encoder, saved and used.
        {"name": "checkpoint_4096x768_fp32", "kind": "checkpoint", "M": 4096, "K": 768, "type": "fp32"},
        # The wide one of the large encoder at 64 x 384 tokens: throughput.
        {"name": "checkpoint_24576x4096_bf16", "kind": "checkpoint", "M": 24576, "K": 4096, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: tokens and widths over their logarithm, mostly odd sizes."""
    kind = rng.choice(["layer_norm", "layer_norm", "linear", "linear", "train", "train", "checkpoint"])
    if kind == "layer_norm":
        return {"kind": kind, "M": _log_int(rng, 1, 24576), "D": _log_int(rng, 64, 4096), "type": rng.choice(sorted(DTYPES)), "backward": rng.random() < 0.7}
    if kind == "checkpoint":
        return {"kind": kind, "M": _log_int(rng, 1, 24576), "K": _log_int(rng, 64, 4096), "type": rng.choice(sorted(DTYPES))}
    while True:
        c = {"kind": kind, "M": _log_int(rng, 1, 24576), "N": _log_int(rng, 8, 4096), "K": _log_int(rng, 64, 4096), "type": rng.choice(["bf16", "bf16", "fp16"])}
        if rng.random() < 0.7:  # a model's widths
            c["N"], c["K"] = max(8, c["N"] // 8 * 8), c["K"] // 8 * 8
        if c["M"] * c["N"] * c["K"] <= 24576 * 4096 * 1024:
            break
    c["gelu"] = rng.random() < 0.5
    c["residual"] = rng.random() < 0.5
    if kind == "linear":
        return dict(c, out=rng.choice([c["type"], c["type"], "fp32"]), bias=rng.random() < 0.7)
    return dict(c, save=rng.choice(["no", "pre", "codes"]), through=rng.choice(["no", "pre", "codes"]))


def _saved_bytes(how, n):
    return {"no": 0, "pre": 2 * n, "codes": n + 4 * n // BLOCK}[how]


def work(case):
    """Each input read once and each output written once; the products' multiplications and additions."""
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if case["kind"] == "layer_norm":
        n, M, D = case["M"] * case["D"] * size[case["type"]], case["M"], case["D"]
        forward = {"bytes": 2 * n + 8 * D + 8 * M, "flops": 8 * M * D}
        if not case["backward"]:
            return forward
        return {"bytes": forward["bytes"] + 3 * n + 8 * M + 12 * D, "flops": 24 * M * D}
    if case["kind"] == "checkpoint":
        n, e = case["M"] * case["K"], size[case["type"]]
        # saved; read and restored; read beside the gradient
        return {"bytes": 4 * n * e + 3 * _saved_bytes("codes", n), "flops": 60 * n}
    M, N, K = case["M"], case["N"], case["K"]
    x, w, y = 2 * M * K, 2 * N * K, M * N
    if case["kind"] == "linear":
        out = y * size[case["out"]]
        return {"bytes": x + w + 4 * N * case["bias"] + out * (2 if case["residual"] else 1), "flops": 2 * M * N * K}
    forward = x + w + 4 * N + 2 * y * (2 if case["residual"] else 1) + _saved_bytes(case["save"], y)
    grad_x = 2 * y + w + x + _saved_bytes(case["through"], M * K)
    return {"bytes": forward + grad_x + 2 * y + x + 4 * N * K + 4 * N, "flops": 6 * M * N * K}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _randn(seed, stream, *shape):
    return torch.randn(*shape, device="cuda", generator=_generator(seed, stream))


def _weights(seed, stream, N, K):
    """Normal weights, 1 % of them outliers five times as wide."""
    w = _randn(seed, stream, N, K) * 0.02
    w *= 1 + 4 * (torch.rand(N, K, device="cuda", generator=_generator(seed, stream + 50)) < 0.01)
    return w


def _activations(seed, stream, M, K):
    """Normal activations with two outlier channels."""
    x = _randn(seed, stream, M, K)
    x[:, torch.randint(0, K, (2,), device="cuda", generator=_generator(seed, stream + 50))] *= 20
    return x


def _gradients(seed, stream, M, N, type):
    """Small gradients whose size differs from token to token; in half precision of a loss that was scaled up."""
    return (_randn(seed, stream, M, N) * torch.exp(_randn(seed, stream + 50, M, 1)) * (0.1 if type == "fp16" else 1e-4)).to(DTYPES[type])


def prepare(case, seed):
    s = {"case": case, "ws": torch.zeros(WS_BYTES, dtype=torch.uint8, device="cuda")}
    t, M = case["type"], case["M"]
    if case["kind"] == "layer_norm":
        D = case["D"]
        s["x"] = (_activations(seed, 1, M, D) + 0.3 * _randn(seed, 2, 1, D)).to(DTYPES[t])
        s["gamma"], s["beta"] = 1 + 0.2 * _randn(seed, 3, D), 0.1 * _randn(seed, 4, D)
        if case["backward"]:
            s["dy"] = _gradients(seed, 5, M, D, t)
        return s
    if case["kind"] == "checkpoint":
        s["x"] = _activations(seed, 1, M, case["K"]).to(DTYPES[t])
        s["dy"] = _gradients(seed, 2, M, case["K"], t)
        return s
    N, K = case["N"], case["K"]
    s["w"] = _weights(seed, 1, N, K).to(DTYPES[t])
    s["bias"] = 0.1 * _randn(seed, 2, N) if case.get("bias", True) else None
    x = _activations(seed, 3, M, K)
    if case.get("through", "no") != "no":  # x is GELU of what the pass before saved
        if case["through"] == "codes":
            s["codes"], s["scales"] = _codes(x)
            x = _values(s["codes"], s["scales"])
        else:
            s["pre"] = x = x.to(DTYPES[t])
        x = _gelu(x.float())
    s["x"] = x.to(DTYPES[t])
    if case["residual"]:
        s["residual"] = _randn(seed, 4, M, N).to(DTYPES[case.get("out", t)])
    if case["kind"] == "train":
        s["dy"] = _gradients(seed, 5, M, N, t)
    return s


# ---- the package's calls -----------------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_1909_05840_b200 as qb
    c = s["case"]
    t = DTYPES[c["type"]]
    if c["kind"] == "layer_norm":
        if not c["backward"]:
            return [qb.layer_norm(s["x"], s["gamma"], s["beta"], EPS)]
        y, mean, rstd = qb.layer_norm(s["x"], s["gamma"], s["beta"], EPS, want_stats=True)
        return [y, mean, rstd, *qb.layer_norm_backward(s["dy"], s["x"], s["gamma"], mean, rstd, s["ws"])]
    if c["kind"] == "checkpoint":
        saved = qb.checkpoint(s["x"])
        return [qb.restore(saved, t), qb.gelu_backward(s["dy"], saved)]
    activation = "gelu" if c["gelu"] else None
    if c["kind"] == "linear":
        return [qb.linear(s["x"], s["w"], s["bias"], s["ws"], activation=activation, residual=s.get("residual"), out_dtype=DTYPES[c["out"]])]
    out = qb.linear(s["x"], s["w"], s["bias"], s["ws"], activation=activation, residual=s.get("residual"), save=None if c["save"] == "no" else c["save"])
    # what was saved in 8 bits is given as the values that it stands for
    outs = [out] if c["save"] == "no" else [out[0], qb.restore(out[1], t) if c["save"] == "codes" else out[1]]
    before = {"no": None, "pre": s.get("pre"), "codes": (s.get("codes"), s.get("scales"))}[c["through"]]
    dx = qb.linear_grad_x(s["dy"], s["w"], s["ws"], through=before)
    return [*outs, dx, *qb.linear_grad_w(s["dy"], s["x"], s["ws"])]


# ---- the plain forms -----------------------------------------------------------------------------------------------------------
ROOT_HALF = 0.5 ** 0.5


def _gelu(z):
    return z * (0.5 * torch.special.erfc(z * -ROOT_HALF))


def _gelu_slope(z):
    return 0.5 * torch.special.erfc(z * -ROOT_HALF) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2 * math.pi))


def _codes(x):
    """Codes (int8 [M][K]) and scales (fp32 [M][blocks]): scale = max|x| / 127 of a row's 64 values, code = x * 127 / max|x| rounded to
    nearest even.  The quotient is taken in 64 bits: in 32 it may be rounded onto the border of two codes."""
    M, K = x.shape
    blocks = (K + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - K)).view(M, blocks, BLOCK)
    top = v.abs().amax(dim=2, keepdim=True)
    some = top >= 2.0**-100
    q = torch.where(some, torch.round(v.double() * 127.0 / top.double()), 0.0).to(torch.int8)
    scales = torch.where(some, top / 127.0, torch.ones((), device=x.device))
    return q.view(M, blocks * BLOCK)[:, :K].contiguous(), scales.view(M, blocks)


def _values(codes, scales):
    return codes.float() * scales.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    t = DTYPES[c["type"]]
    if c["kind"] == "layer_norm":
        x = s["x"].float()
        mean = x.mean(dim=1)
        d = x - mean[:, None]
        rstd = torch.rsqrt((d * d).mean(dim=1) + EPS)
        xhat = d * rstd[:, None]
        y = (xhat * s["gamma"] + s["beta"]).to(t)
        if not c["backward"]:
            return [y]
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = rstd[:, None] * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
        return [y, mean, rstd, dx.to(t), (dy * xhat).sum(dim=0), dy.sum(dim=0)]
    if c["kind"] == "checkpoint":
        v = _values(*_codes(s["x"]))
        return [v.to(t), (s["dy"].float() * _gelu_slope(v)).to(t)]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"]
    y = _gelu(z) if c["gelu"] else z
    if c["residual"]:
        y = y + s["residual"].float()
    if c["kind"] == "linear":
        return [y.to(DTYPES[c["out"]])]
    outs = [y.to(t)]
    if c["save"] != "no":
        outs.append((_values(*_codes(z)) if c["save"] == "codes" else z).to(t))
    dy = s["dy"].float()
    dx = dy @ w
    if c["through"] != "no":
        dx = dx * _gelu_slope(s["pre"].float() if c["through"] == "pre" else _values(s["codes"], s["scales"]))
    return [*outs, dx.to(t), dy.t() @ x, dy.sum(dim=0)]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------
def _normal(z):
    """Distribution function and density of the normal distribution."""
    return torch.special.ndtr(z), torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)


def _exact_saved(z):
    """The values that fp64 [M][K] becomes when it is saved in 8 bits."""
    out = torch.empty_like(z)
    for k in range(0, z.shape[1], BLOCK):
        part = z[:, k:k + BLOCK]
        top = part.abs().amax(dim=1, keepdim=True)
        out[:, k:k + BLOCK] = torch.where(top > 0, torch.round(part * 127 / top) * top / 127, 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "layer_norm":
        x, D = s["x"].double(), case["D"]
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        xhat = torch.einsum("md,m->md", x - mean[:, None], rstd)
        y = torch.addcmul(s["beta"].double(), xhat, s["gamma"].double())
        if not case["backward"]:
            return [y]
        dy = s["dy"].double()
        g = dy * s["gamma"].double()
        along, mean_g = torch.einsum("md,md->m", g, xhat) / D, g.sum(dim=1) / D
        dx = (g - mean_g[:, None] - xhat * along[:, None]) * rstd[:, None]
        return [y, mean, rstd, dx, torch.einsum("md,md->d", dy, xhat), dy.sum(dim=0)]
    if case["kind"] == "checkpoint":
        v = _exact_saved(s["x"].double())
        cdf, density = _normal(v)
        return [v, s["dy"].double() * (cdf + v * density)]
    x, w = s["x"].double(), s["w"].double()
    z = torch.nn.functional.linear(x, w, None if s["bias"] is None else s["bias"].double())
    y = z * _normal(z)[0] if case["gelu"] else z
    if case["residual"]:
        y = y + s["residual"].double()
    if case["kind"] == "linear":
        return [y]
    outs = [y] + {"no": [], "pre": [z], "codes": [_exact_saved(z)] if case["save"] == "codes" else []}[case["save"]]
    dy = s["dy"].double()
    dx = torch.einsum("mn,nk->mk", dy, w)
    if case["through"] != "no":
        if case["through"] == "pre":
            p = s["pre"].double()
        else:
            column = torch.arange(case["K"], device="cuda")
            p = s["codes"].double() * s["scales"].double()[:, column // BLOCK]
        cdf, density = _normal(p)
        dx = dx * (cdf + p * density)
    return [*outs, dx, torch.einsum("mn,mk->nk", dy, x), dy.sum(dim=0)]
