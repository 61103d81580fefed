"""The operators of a fine-tuning step around the quantized linears, as cases for timing and for comparing results.

* ``dropout``       one dropout with the residual added behind it, forward, and where asked its backward pass;
* ``fp8_linear``    serving: a fresh activation tensor quantized to 8-bit floating point in blocks of 1 x 128 and
                    multiplied by weights that were quantized in blocks of 128 x 128 when the model was loaded;
* ``fp8_train``     a linear of a training step: x, w and dy quantized (both ways each is contracted), the three products;
* ``vocab_loss``    softmax cross entropy of masked words over the vocabulary, and where asked its gradients.

``run`` computes them in elementary torch operations where ``own`` is false, else through the package.
"""
import math

import numpy as np
import torch

own = False

WS_BYTES = 1 << 28  # the workspace that a program keeps for all of its calls
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FP8_TOP = {"e4m3": 448.0, "e5m2": 57344.0}


def listed():
    return [
        # Hidden states of the last token of 32 sequences: the smallest call, launch latency.
        {"name": "dropout_32x768_fp32", "kind": "dropout", "M": 32, "N": 768, "type": "fp32", "p": 0.1, "residual": False, "backward": False},
        # Behind the attention output of a ragged batch of the large encoder, with the residual, and its backward pass.
        {"name": "dropout_5003x1024_bf16", "kind": "dropout", "M": 5003, "N": 1024, "type": "bf16", "p": 0.1, "residual": True, "backward": True},
        # The wide activations of 64 x 384 tokens in 16 bits, and their backward pass: throughput.
        {"name": "dropout_24576x4096_fp16", "kind": "dropout", "M": 24576, "N": 4096, "type": "fp16", "p": 0.1, "residual": False, "backward": True},
        # The pooler of a small batch.
        {"name": "linear_m32", "kind": "fp8_linear", "M": 32, "N": 768, "K": 768, "type": "fp32", "out": "bf16", "format": "e4m3", "bias": True},
        # A ragged batch through the fused query, key and value projection.
        {"name": "linear_m5003_qkv", "kind": "fp8_linear", "M": 5003, "N": 2304, "K": 768, "type": "fp32", "out": "bf16", "format": "e4m3", "bias": True},
        # The second feed-forward linear of the large encoder at 64 x 384 tokens: throughput, fp32 handed on.
        {"name": "linear_m24576_ffn2", "kind": "fp8_linear", "M": 24576, "N": 1024, "K": 4096, "type": "bf16", "out": "fp32", "format": "e4m3", "bias": True},
        # A task head of nine labels in a training step: odd sizes in every product.
        {"name": "train_m613_head9", "kind": "fp8_train", "M": 613, "N": 9, "K": 768, "type": "fp32", "gradient": "e5m2"},
        # The first feed-forward linear of the large encoder in a training step over 16 x 384 tokens.
        {"name": "train_m6144_ffn1", "kind": "fp8_train", "M": 6144, "N": 4096, "K": 1024, "type": "bf16", "gradient": "e4m3"},
        # Scoring the masked words of four sequences.
        {"name": "loss_t77", "kind": "vocab_loss", "T": 77, "V": 30522, "D": 768, "bias": True, "backward": False},
        # The masked words (15 %) of 32 x 128 tokens, training.
        {"name": "loss_t613_train", "kind": "vocab_loss", "T": 613, "V": 30522, "D": 768, "bias": True, "backward": True},
        # Every token of 32 x 128 scored.
        {"name": "loss_t4096", "kind": "vocab_loss", "T": 4096, "V": 30522, "D": 768, "bias": True, "backward": False},
        # The masked words of 64 x 384 tokens, training the large encoder.
        {"name": "loss_t3686_train", "kind": "vocab_loss", "T": 3686, "V": 30522, "D": 1024, "bias": True, "backward": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: batches and vocabularies over their logarithm, mostly odd sizes."""
    kind = rng.choice(["dropout", "fp8_linear", "fp8_linear", "fp8_train", "vocab_loss", "vocab_loss"])
    if kind == "dropout":
        return {"kind": kind, "M": _log_int(rng, 1, 24576), "N": _log_int(rng, 8, 4096), "type": rng.choice(sorted(DTYPES)),
                "p": rng.choice([0.0, 0.1, 0.25, 0.5]), "residual": rng.random() < 0.5, "backward": rng.random() < 0.5}
    if kind == "vocab_loss":
        while True:
            c = {"kind": kind, "T": _log_int(rng, 1, 4096), "V": _log_int(rng, 500, 60000), "D": 8 * rng.randint(8, 128),
                 "bias": rng.random() < 0.7, "backward": rng.random() < 0.6}
            if c["T"] * c["V"] * c["D"] <= 3686 * 30522 * 1024:
                return c
    while True:
        c = {"kind": kind, "M": _log_int(rng, 1, 24576), "N": _log_int(rng, 8, 4096), "K": _log_int(rng, 64, 4096),
             "type": rng.choice(["fp32", "bf16"])}
        if kind == "fp8_linear":
            return dict(c, out=rng.choice(["bf16", "fp32"]), format=rng.choice(["e4m3", "e4m3", "e5m2"]), bias=rng.random() < 0.7)
        if c["M"] * c["N"] * c["K"] <= 6144 * 4096 * 1024:
            return dict(c, gradient=rng.choice(["e4m3", "e5m2"]))


def work(case):
    """Each input read once and each output written once; the products' multiplications and additions."""
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if case["kind"] == "dropout":
        n = case["M"] * case["N"]
        tensors = (3 if case["residual"] else 2) + (2 if case["backward"] else 0)
        return {"bytes": n * size[case["type"]] * tensors, "flops": 2 * n}
    if case["kind"] == "vocab_loss":
        T, V, D = case["T"], case["V"], case["D"]
        read = 2 * (T * D + V * D) + 4 * V * case["bias"] + 4 * T
        if not case["backward"]:
            return {"bytes": read + 8 * T, "flops": 2 * T * V * D}
        # the logits are not kept: the backward pass computes them again
        return {"bytes": 2 * read + 2 * (T * D + V * D) + 4 * V * case["bias"] + 16 * T, "flops": 8 * T * V * D}
    M, N, K, e = case["M"], case["N"], case["K"], size[case["type"]]
    if case["kind"] == "fp8_linear":
        return {"bytes": M * K * e + N * K + N * K // 128 + 4 * N * case["bias"] + M * N * size[case["out"]], "flops": 2 * M * N * K}
    return {"bytes": M * K * e + 4 * N * K + 2 * M * N + 2 * M * N + 2 * M * K + 4 * N * K, "flops": 6 * M * N * K}


# ---- 8-bit floating point with power-of-two scales -----------------------------------------------------------------------
def _up(n, m):
    return (n + m - 1) // m * m


def _pad(x, rows, cols):
    return torch.nn.functional.pad(x, (0, cols - x.shape[1], 0, rows - x.shape[0]))


def _exponent(amax, fmt):
    """The least e with amax * 2^-e <= the largest code value; 0 for a block of zeros."""
    mantissa, exponent = torch.frexp(amax)  # amax = mantissa * 2^exponent, 0.5 <= mantissa < 1
    e = exponent - (9 if fmt == "e4m3" else 16) + (mantissa > 0.875).to(torch.int32)
    return torch.where(amax > 0, e.clamp(min=-127), torch.zeros_like(e))


def _quantize(x, fmt, rows):
    """Codes [R][Kp] (as 8-bit floats) and exponents [R][Kp / 128] of fp32 [R][K]; blocks of `rows` x 128."""
    R, K = x.shape
    Rp, Kp = _up(R, rows), _up(K, 128)
    xp = _pad(x, Rp, Kp).view(Rp // rows, rows, Kp // 128, 128)
    e = _exponent(xp.abs().amax(dim=(1, 3)), fmt)
    q = torch.ldexp(xp, -e[:, None, :, None]).view(Rp, Kp)[:R].to(FP8[fmt])
    return q, e.repeat_interleave(rows, dim=0)[:R]


def _pack_scales(e):
    """Exponents [R][B] as the bytes e + 127 in the order in which the package keeps them: per 128 rows and 4 blocks 512 bytes,
    row r at 16 * (r % 32) + 4 * (r % 128 / 32), one byte per block."""
    R, B = e.shape
    full = torch.full((_up(R, 128), _up(B, 4)), 127, dtype=torch.uint8, device=e.device)
    full[:R, :B] = (e + 127).to(torch.uint8)
    return full.view(_up(R, 128) // 128, 4, 32, _up(B, 4) // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _unpack_scales(s, R, B):
    return (s.permute(0, 3, 2, 1, 4).reshape(s.shape[0] * 128, s.shape[1] * 4)[:R, :B].to(torch.int32)) - 127


def _values(q, e):
    R, Kp = q.shape
    return torch.ldexp(q.float().view(R, Kp // 128, 128), e[:, :, None]).view(R, Kp)


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


def _gradients(seed, stream, M, N):
    """Small gradients whose size differs from token to token."""
    return _randn(seed, stream, M, N) * torch.exp(_randn(seed, stream + 50, M, 1)) * 1e-4


def prepare(case, seed):
    s = {"case": case, "ws": torch.zeros(WS_BYTES, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "dropout":
        t = DTYPES[case["type"]]
        s["x"] = _activations(seed, 1, case["M"], case["N"]).to(t)
        if case["residual"]:
            s["residual"] = _randn(seed, 2, case["M"], case["N"]).to(t)
        if case["backward"]:
            s["dy"] = _gradients(seed, 3, case["M"], case["N"]).to(t)
        # seed and offset of the generator, on the device: a captured step advances the offset itself
        s["rng"] = torch.tensor([0x1234567 + 7919 * seed, 1000 + seed], dtype=torch.int64, device="cuda")
        return s
    if case["kind"] == "vocab_loss":
        T, V, D = case["T"], case["V"], case["D"]
        w = _weights(seed, 1, V, D)
        targets = torch.randint(0, V, (T,), device="cuda", generator=_generator(seed, 2))
        # a trained model: the right word stands out, by more or less
        sure = torch.rand(T, 1, device="cuda", generator=_generator(seed, 3))
        h = _randn(seed, 4, T, D) + sure * (w[targets] * 50)
        s["h"], s["w"] = h.bfloat16(), w.bfloat16()
        s["bias"] = _randn(seed, 5, V) * 0.02 if case["bias"] else None
        # every eighth word or so is no target (the batch was padded to a fixed number of masked words)
        s["targets"] = torch.where(torch.rand(T, device="cuda", generator=_generator(seed, 6)) < 0.12, -100, targets).to(torch.int32)
        if T == 1:
            s["targets"] = targets.to(torch.int32)
        s["grad_loss"] = torch.full((T,), 1.0 / T, device="cuda")
        return s
    M, N, K = case["M"], case["N"], case["K"]
    s["x"] = _activations(seed, 1, M, K).to(DTYPES[case["type"]])
    w = _weights(seed, 2, N, K)
    if case["kind"] == "fp8_linear":
        q, e = _quantize(w, case["format"], 128)
        s["wq"], s["wscale"] = q, _pack_scales(e)
        s["bias"] = _randn(seed, 3, N) * 0.02 if case["bias"] else None
    else:
        s["w"] = w
        s["dy"] = _gradients(seed, 4, M, N).bfloat16()
    return s


# ---- the package's calls -----------------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_1909_05840_b200 as qb
    c = s["case"]
    if c["kind"] == "dropout":
        y = qb.dropout(s["x"], c["p"], s["rng"], call=3, residual=s.get("residual"))
        return [y, qb.dropout(s["dy"], c["p"], s["rng"], call=3)] if c["backward"] else [y]
    if c["kind"] == "vocab_loss":
        loss, lse = qb.vocab_loss(s["h"], s["w"], s["bias"], s["targets"], s["ws"])
        if not c["backward"]:
            return [loss, lse]
        dh, dw, db = qb.vocab_loss_backward(s["h"], s["w"], s["bias"], s["targets"], lse, s["grad_loss"], s["ws"])
        return [loss, lse, dh, dw] + ([db] if c["bias"] else [])
    if c["kind"] == "fp8_linear":
        xq, xs = qb.quantize_fp8(s["x"], s["ws"], FP8[c["format"]])
        return [qb.gemm_fp8(xq, xs, s["wq"], s["wscale"], s["bias"], s["ws"], DTYPES[c["out"]])]
    e4m3, grad = FP8["e4m3"], FP8[c["gradient"]]
    xq, xs, xqt, xst = qb.quantize_fp8(s["x"], s["ws"], e4m3, transposed=True)
    wq, wsc, wqt, wst = qb.quantize_fp8_weights(s["w"], s["ws"], e4m3, transposed=True)
    y = qb.gemm_fp8(xq, xs, wq, wsc, None, s["ws"], torch.bfloat16)
    gq, gs, gqt, gst = qb.quantize_fp8(s["dy"], s["ws"], grad, transposed=True)
    dx = qb.gemm_fp8(gq, gs, wqt, wst, None, s["ws"], torch.bfloat16)
    dw = qb.gemm_fp8(gqt, gst, xqt, xst, None, s["ws"], torch.float32)
    return [y, dx, dw]


# ---- the plain forms -----------------------------------------------------------------------------------------------------------
def _mulhilo(a, b):
    """High and low 32 bits of the product of two 32-bit numbers held in int64."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _words(n, rng, call):
    """n 32-bit words of Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers, SC 2011)."""
    i = torch.arange((n + 3) // 4, device="cuda")
    sub = rng[1] + call
    c0, c1 = i & 0xFFFFFFFF, i >> 32
    c2, c3 = (sub & 0xFFFFFFFF).expand_as(i), ((sub >> 32) & 0xFFFFFFFF).expand_as(i)
    k0, k1 = rng[0] & 0xFFFFFFFF, (rng[0] >> 32) & 0xFFFFFFFF
    for _ in range(7):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.stack([c0, c1, c2, c3], dim=1).view(-1)[:n]


def _dropout(x, p, rng, call, residual=None):
    keep = _words(x.numel(), rng, call).view(x.shape) >= int(round(p * 2.0**32))
    y = torch.where(keep, x.float() * (1.0 / (1.0 - p)), torch.zeros((), device=x.device))
    if residual is not None:
        y = y + residual.float()
    return y.to(x.dtype)


def _product(a, b):
    return a @ b.t()


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    if c["kind"] == "dropout":
        y = _dropout(s["x"], c["p"], s["rng"], 3, s.get("residual"))
        return [y, _dropout(s["dy"], c["p"], s["rng"], 3)] if c["backward"] else [y]
    if c["kind"] == "vocab_loss":
        h, w = s["h"].float(), s["w"].float()
        z = h @ w.t()
        if s["bias"] is not None:
            z += s["bias"]
        top = z.amax(dim=1, keepdim=True)
        lse = (top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True)))
        valid = s["targets"] >= 0
        at = s["targets"].clamp(min=0).long()
        rows = torch.arange(c["T"], device="cuda")
        loss = torch.where(valid, lse[:, 0] - z[rows, at], torch.zeros((), device="cuda"))
        if not c["backward"]:
            return [loss, lse[:, 0]]
        g = torch.exp(z.sub_(lse))
        g[rows, at] -= 1.0
        g *= torch.where(valid, s["grad_loss"], torch.zeros((), device="cuda"))[:, None]
        return [loss, lse[:, 0], (g @ w).bfloat16(), (g.t() @ h).bfloat16()] + ([g.sum(dim=0)] if c["bias"] else [])
    if c["kind"] == "fp8_linear":
        xv = _values(*_quantize(s["x"].float(), c["format"], 1))
        wv = _values(s["wq"], _unpack_scales(s["wscale"], c["N"], s["wq"].shape[1] // 128))
        y = _product(xv, wv)
        if s["bias"] is not None:
            y += s["bias"]
        return [y.to(DTYPES[c["out"]])]
    x, w, dy, grad = s["x"].float(), s["w"], s["dy"].float(), c["gradient"]
    y = _product(_values(*_quantize(x, "e4m3", 1)), _values(*_quantize(w, "e4m3", 128)))
    dx = _product(_values(*_quantize(dy, grad, 1)), _values(*_quantize(w.t(), "e4m3", 128)))
    dw = _product(_values(*_quantize(dy.t(), grad, 1)), _values(*_quantize(x.t(), "e4m3", 1)))
    return [y.bfloat16(), dx.bfloat16(), dw]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------
def _exact_drop(x, p, seed, offset, residual):
    """Dropout with the generator in numpy's 64-bit whole numbers."""
    n, low = x.numel(), np.uint64(0xFFFFFFFF)
    c = [np.arange((n + 3) // 4, dtype=np.uint64), np.uint64(0), np.uint64(offset) & low, np.uint64(offset) >> np.uint64(32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack([np.broadcast_to(w, c[0].shape).astype(np.uint32) for w in c], axis=1).reshape(-1)[:n]
    dropped = torch.from_numpy(words < np.uint64(round(p * 2.0**32))).cuda().view(x.shape)
    y = x.double() / (1.0 - p)
    y[dropped] = 0.0
    return y if residual is None else y + residual.double()


def _exact_fp8(x, fmt, rows):
    """The values that fp64 [R][K] becomes in blocks of `rows` x 128, from the grid of the format."""
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], 128):
        for r, part in enumerate([x[:, k:k + 128]] if rows == 1 else torch.split(x[:, k:k + 128], rows)):
            amax = part.abs().amax(dim=1, keepdim=True) if rows == 1 else part.abs().amax()
            # from the numbers' own exponents: a logarithm may round at a power of two
            m, e = torch.frexp(amax / FP8_TOP[fmt])
            e = torch.where(amax > 0, (e - (m == 0.5).int()).clamp(min=-127), torch.zeros_like(e))
            v = torch.ldexp(part, -e)
            step = torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp(min=2.0**least))[1] - 1 - bits)
            q = torch.ldexp(torch.round(v / step) * step, e)
            out[r * rows if rows > 1 else 0:(r * rows if rows > 1 else 0) + part.shape[0], k:k + 128] = q
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        if case["M"] * case["N"] > 1 << 25:  # the generator alone takes too long
            return None
        key, offset = (int(v) for v in s["rng"].tolist())
        y = _exact_drop(s["x"], case["p"], key, offset + 3, s.get("residual"))
        return [y, _exact_drop(s["dy"], case["p"], key, offset + 3, None)] if case["backward"] else [y]
    if case["kind"] == "vocab_loss":
        h, w, valid = s["h"].double(), s["w"].double(), s["targets"] >= 0
        z = torch.nn.functional.linear(h, w, s["bias"].double() if case["bias"] else None)
        lse = torch.logsumexp(z, dim=1)
        hot = torch.zeros_like(z)
        hot[valid] = torch.nn.functional.one_hot(s["targets"][valid].long(), case["V"]).double()
        loss = torch.where(valid, lse, 0.0) - (z * hot).sum(dim=1)
        if not case["backward"]:
            return [loss, lse]
        g = (torch.softmax(z, dim=1) * valid[:, None] - hot) * s["grad_loss"].double()[:, None]
        return [loss, lse, g @ w, g.t() @ h] + ([g.sum(dim=0)] if case["bias"] else [])
    x = s["x"].double()
    if case["kind"] == "fp8_linear":
        N, blocks = case["N"], s["wq"].shape[1] // 128
        r, b = torch.arange(N, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None, :]
        e = s["wscale"][r // 128, b // 4, r % 32, r % 128 // 32, b % 4].double() - 127
        w = (s["wq"].double() * torch.pow(2.0, e).repeat_interleave(128, dim=1))[:, :case["K"]]
        y = torch.einsum("mk,nk->mn", _exact_fp8(x, case["format"], 1), w)
        return [y + s["bias"].double() if case["bias"] else y]
    w, dy, grad = s["w"].double(), s["dy"].double(), case["gradient"]
    wq = _exact_fp8(w, "e4m3", 128)  # a block and its transpose have the same scale
    y = torch.einsum("mk,nk->mn", _exact_fp8(x, "e4m3", 1), wq)
    dx = torch.einsum("mn,nk->mk", _exact_fp8(dy, grad, 1), wq)
    dw = torch.einsum("nm,km->nk", _exact_fp8(dy.t().contiguous(), grad, 1), _exact_fp8(x.t().contiguous(), "e4m3", 1))
    return [y, dx, dw]
