"""Softmax cross entropy over the vocabulary and its gradients, against 64 bits and against differences."""
import pytest
import torch

import paper_1909_05840_b200 as qb

pytestmark = pytest.mark.gpu


def inputs(T, V, D, seed=0, bias=True, ignored=True):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + T + V + D)
    w = (torch.randn(V, D, device="cuda", generator=g) * (1.0 / D**0.5)).bfloat16()
    targets = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
    sure = 6 * torch.rand(T, 1, device="cuda", generator=g)
    h = (torch.randn(T, D, device="cuda", generator=g) + sure * w[targets.long()].float()).bfloat16()
    b = torch.randn(V, device="cuda", generator=g) * 0.5 if bias else None
    if ignored:
        targets[torch.rand(T, device="cuda", generator=g) < 0.2] = -100
    gl = torch.rand(T, device="cuda", generator=g) / T
    return h, w, b, targets, gl


def reference(h, w, b, targets, gl):
    """Values and bounds in 64 bits.

    A logit is D exact products accumulated in fp32: at most 2^-23 of the terms' absolute sum for each of D / 16 accumulations and of
    16 additions inside one (ez).  lse: the largest ez of its row, exponents rounded at 2^-24 of the logits (twice, and once for
    lse itself; 2^-21 for all), exponentials good to 2^-21 and the sums' roundings (at most 64 + V / 1024 in a chain).  A
    probability's relative error is the sum of both (ep).  g is rounded to bfloat16 (2^-8) for its products and accumulated over
    V (T) terms like the logits; the bias's gradient is summed in fp32; the outputs in bfloat16 are rounded once more.
    Below 2^-126 a probability, an entry of g (fp32 and bfloat16 have the same least normal number) and a product of the two
    matrix products may become 0: three times up to 2^-126 in every entry of g, which the products multiply by |w| (|h|) and sum, and
    2^-126 for each of the V (T) terms."""
    hd, wd = h.double(), w.double()
    (T, D), V = h.shape, w.shape[0]
    z = hd @ wd.t()
    if b is not None:
        z = z + b.double()
    ez = (hd.abs() @ wd.abs().t()) * (D / 16 + 16) * 2.0**-23
    if b is not None:
        ez = ez + z.abs() * 2.0**-24
    lse = torch.logsumexp(z, dim=1)
    valid = (targets >= 0) & (targets < V)
    at = targets.clamp(0, V - 1).long()[:, None]
    finite = torch.where(torch.isfinite(z), z.abs(), 0.0)
    e_lse = torch.where(torch.isfinite(ez), ez, 0.0).amax(1) + (finite.amax(1) + lse.abs() + 1) * 2.0**-21 + 2.0**-20 + (64 + V / 1024) * 2.0**-24
    loss = torch.where(valid, lse - z.gather(1, at)[:, 0], 0.0)
    e_loss = torch.where(valid, e_lse + ez.gather(1, at)[:, 0] + loss.abs() * 2.0**-23, 0.0)
    p = torch.exp(z - lse[:, None])
    ep = torch.where(torch.isfinite(ez), ez, 0.0) + e_lse[:, None] + (finite + lse.abs()[:, None]) * 2.0**-22
    hot = torch.zeros_like(z).scatter_(1, at, 1.0) * valid[:, None]
    weight = torch.where(valid, gl.double(), 0.0)[:, None]
    g = (p * valid[:, None] - hot) * weight
    least = 2.0**-126
    eg = p * ep * weight.abs() + g.abs() * 2.0**-23 + 3 * least
    half = 2.0**-8
    eg16 = eg * (1 + half) + g.abs() * half
    gh, gw = g @ wd, g.t() @ hd
    e_gh = eg16 @ wd.abs() + (g.abs() @ wd.abs()) * (V / 16 + 80) * 2.0**-23 + V * least
    e_gw = eg16.t() @ hd.abs() + (g.abs().t() @ hd.abs()) * (T / 16 + 16) * 2.0**-23 + T * least
    gb, e_gb = g.sum(0), eg.sum(0) + g.abs().sum(0) * (T + 8) * 2.0**-24
    return {"loss": (loss, e_loss + least), "lse": (lse, e_lse), "grad_h": (gh, e_gh * (1 + half) + gh.abs() * half + least),
            "grad_w": (gw, e_gw * (1 + half) + gw.abs() * half + least), "grad_bias": (gb, e_gb + least)}


def check(name, got, ref):
    want, tol = ref[name]
    off = (got.double() - want).abs()
    assert (off <= tol).all(), f"{name}: {int((off > tol).sum())} of {off.numel()} off, worst {float((off / tol).max()):.3g} of the bound"


def poisoned(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def run(h, w, b, targets, gl, ws):
    (T, D), V = h.shape, w.shape[0]
    loss, lse = qb.vocab_loss(h, w, b, targets, ws, poisoned(T, dtype=torch.float32), poisoned(T, dtype=torch.float32))
    # canaries behind the matrices: rows behind the last token and word stay as they were
    gh, gw = poisoned(T + 3, D, dtype=torch.bfloat16), poisoned(V + 3, D, dtype=torch.bfloat16)
    gb = poisoned(V + 3, dtype=torch.float32) if b is not None else None
    grads = qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws, gh[:T], gw[:V], None if gb is None else gb[:V])
    assert torch.isnan(gh[T:]).all() and torch.isnan(gw[V:]).all() and (gb is None or torch.isnan(gb[V:]).all())
    return {"loss": loss, "lse": lse, "grad_h": grads[0], "grad_w": grads[1], "grad_bias": grads[2]}


def check_all(h, w, b, targets, gl, ws):
    got, ref = run(h, w, b, targets, gl, ws), reference(h, w, b, targets, gl)
    for name in ref:
        if got[name] is not None:
            check(name, got[name], ref)
    return got


SHAPES = [(1, 1, 8), (1, 500, 64), (3, 257, 72), (31, 256, 128), (77, 1000, 768), (128, 129, 1024), (255, 300, 8), (256, 512, 64), (257, 513, 136),
          (300, 5000, 320), (613, 3001, 768), (1030, 2100, 1000), (2049, 4097, 256), (40, 30522, 192),
          (32, 300, 64), (33, 700, 136), (96, 520, 64), (97, 257, 192), (161, 600, 72), (225, 1100, 64), (320, 900, 64), (672, 1300, 128)]


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_forward_and_gradients(T, V, D, bias):
    ws = qb.vocab_loss_workspace(T, V, D)
    check_all(*inputs(T, V, D, bias=bias), ws)
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("T,V,D", [(100, 3000, 264), (613, 5000, 768), (1500, 2600, 72)])
def test_pieces(T, V, D):
    """The same result, up to the order of the additions, from any number of pieces; too little workspace is refused."""
    args = inputs(T, V, D)
    ref = reference(*args)
    full = qb.vocab_loss_workspace_bytes(T, V, D)
    big = torch.zeros(full + (64 << 20), dtype=torch.uint8, device="cuda")
    loss, lse = qb.vocab_loss(*args[:4], big)

    def least(call):  # the smallest workspace that is accepted, to 4 KB
        lo, hi = 0, full
        while hi - lo > 4096:
            mid = (lo + hi) // 2
            try:
                call(big[:mid])
                hi = mid
            except qb.QbertError as e:
                assert e.status == qb.QB_ERR_WORKSPACE
                lo = mid
        return hi
    forward = least(lambda ws: qb.vocab_loss(*args[:4], ws))
    least = least(lambda ws: qb.vocab_loss_backward(*args[:4], lse, args[4], ws))
    assert max(forward, least) <= full and least < full  # less is taken, in more pieces
    rows = 256 * 2 * (T + 63)
    for nbytes in sorted({least, least + 3 * rows, (full + least) // 2, full, full + (64 << 20)}):
        ws = big[:max(nbytes, forward)]
        got = run(*args, ws)
        for name in ref:
            check(name, got[name], ref)
        again = run(*args, ws)
        assert all(torch.equal(got[k], again[k]) for k in got)  # the same order every time
    assert qb.read_status(big) == qb.QB_OK


def test_differences():
    """The gradients against central differences of the 64-bit loss along random directions (error of the step: third derivative)."""
    T, V, D = 20, 300, 64
    h, w, b, targets, gl = inputs(T, V, D)
    ws = qb.vocab_loss_workspace(T, V, D)
    got = run(h, w, b, targets, gl, ws)

    def total(hd, wd, bd):
        z = hd @ wd.t() + bd
        valid = targets >= 0
        loss = torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0).long()[:, None])[:, 0]
        return (torch.where(valid, loss, 0.0) * gl.double()).sum()
    x = [h.double(), w.double(), b.double()]
    ref = reference(h, w, b, targets, gl)
    for i, name in enumerate(("grad_h", "grad_w", "grad_bias")):
        for seed in range(3):
            g = torch.Generator(device="cuda").manual_seed(seed)
            d = torch.randn(x[i].shape, device="cuda", dtype=torch.float64, generator=g)
            step = 1e-4
            plus, minus = list(x), list(x)
            plus[i], minus[i] = x[i] + step * d, x[i] - step * d
            want = (total(*plus) - total(*minus)) / (2 * step)
            have = (got[name].double() * d).sum()
            assert abs(float(want - have)) <= float((ref[name][1] * d.abs()).sum()) + 1e-6


def test_ignored_and_impossible_targets():
    T, V, D = 300, 700, 128
    h, w, b, targets, gl = inputs(T, V, D)
    targets[:] = -1
    ws = qb.vocab_loss_workspace(T, V, D)
    got = run(h, w, b, targets, gl, ws)
    for name in ("loss", "grad_h", "grad_w", "grad_bias"):
        assert (got[name] == 0).all()
    check("lse", got["lse"], reference(h, w, b, targets, gl))
    assert qb.read_status(ws) == qb.QB_OK
    targets = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    targets[5], targets[299], targets[7] = V, 2**31 - 1, -2**31
    got = check_all(h, w, b, targets, gl, ws)
    assert got["loss"][5] == 0 and got["loss"][299] == 0 and got["loss"][7] == 0
    assert qb.read_status(ws) == qb.QB_ERR_INVALID


def test_words_taken_out_by_their_bias():
    T, V, D = 70, 600, 64
    h, w, b, targets, gl = inputs(T, V, D, ignored=False)
    out = torch.arange(V, device="cuda") % 3 == 1
    out[256:512] = True  # a whole tile of words
    b[out] = -float("inf")
    targets = (targets // 3 * 3 % 255).to(torch.int32)
    ws = qb.vocab_loss_workspace(T, V, D)
    got = run(h, w, b, targets, gl, ws)
    keep = ~out
    part = reference(h, w[keep], b[keep], (torch.cumsum(keep.int(), 0) - 1)[targets.long()].int(), gl)
    for name in ("loss", "lse", "grad_h"):
        check(name, got[name], part)
    assert (got["grad_w"][out] == 0).all() and (got["grad_bias"][out] == 0).all()
    check("grad_w", got["grad_w"][keep], part)
    check("grad_bias", got["grad_bias"][keep], part)
    # a target that its bias takes out: an infinite loss, and a gradient all the same
    targets[3] = 257
    loss, lse = qb.vocab_loss(h, w, b, targets, ws)
    assert loss[3] == float("inf") and torch.isfinite(loss[:3]).all() and torch.isfinite(loss[4:]).all()


LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("mask", [-65504.0, -5e9, -1e20, -1e38, LOWEST])
@pytest.mark.parametrize("T", [1, 77, 128, 129, 300])
def test_words_masked_by_a_finite_bias(T, mask):
    """Words under a large finite negative bias (a padded vocabulary's mask), whole tiles of them among others: their probability is below
    2^-149, so that every result is that of the other words alone."""
    V, D = 900, 64
    h, w, b, targets, gl = inputs(T, V, D, ignored=False)
    out = torch.zeros(V, dtype=torch.bool, device="cuda")
    out[200:264] = out[330:800] = out[870:] = True
    out[5] = True
    b[out] = mask
    keep = ~out
    kept = torch.nonzero(keep)[:, 0]
    place = targets.long() % kept.numel()
    targets = kept[place].int()
    ws = qb.vocab_loss_workspace(T, V, D)
    got, part = run(h, w, b, targets, gl, ws), reference(h, w[keep], b[keep], place.int(), gl)
    for name in ("loss", "lse", "grad_h"):
        check(name, got[name], part)
    assert (got["grad_w"][out] == 0).all() and (got["grad_bias"][out] == 0).all()
    check("grad_w", got["grad_w"][keep], part)
    check("grad_bias", got["grad_bias"][keep], part)
    # a masked target: its loss is the mask's size, to the rounding of the logit, of lse and of their difference
    targets[0] = 400
    loss, _ = qb.vocab_loss(h, w, b, targets, ws)
    want = part["lse"][0][0] - ((h[0].double() * w[400].double()).sum() + mask)
    assert abs(float(loss[0]) - float(want)) <= abs(mask) * 2.0**-22
    assert qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("T", [1, 77, 128, 129, 300])
def test_sure_tokens(T, whole):
    """Targets that the model is sure of: the loss is never below 0, the gradient at the target never above.

    With whole numbers the logits are exact in fp32 whatever the order of their sums, and bias puts them at 3,000: the loss is then
    as far off as the sum of e^-d over the differences d to the maximum.  An exponent is d times log2(e), rounded twice (d * 2^-22
    bounds it), an exponential good to 2^-22, at most eight of them multiplied (2^-19), and the sum's additions 64 + V / 1024 in a
    chain; the logarithm and the last addition round at 2^-23 and 2^-24 of themselves."""
    V, D = 1200, 64
    g = torch.Generator(device="cuda").manual_seed(T)
    targets = torch.randperm(V, device="cuda", generator=g)[:T].int()
    sure = torch.randint(0, 3, (T, 1), device="cuda", generator=g)
    if whole:
        w = torch.randint(-1, 2, (V, D), device="cuda", generator=g).bfloat16()
        h = (sure * w[targets.long()] + torch.randint(-1, 2, (T, D), device="cuda", generator=g)).bfloat16()
        b = 3000 + torch.randint(0, 8, (V,), device="cuda", generator=g) / 4
    else:
        w = torch.randn(V, D, device="cuda", generator=g).bfloat16()
        h = (0.5 * sure * w[targets.long()] + 0.1 * torch.randn(T, D, device="cuda", generator=g)).bfloat16()
        b = torch.randn(V, device="cuda", generator=g) * 0.1
    gl = torch.full((T,), 1.0 / T, device="cuda")
    ws = qb.vocab_loss_workspace(T, V, D)
    got = run(h, w, b, targets, gl, ws)
    assert (got["loss"] >= 0).all()
    z = h.double() @ w.double().t() + b.double()
    at = targets.long()[:, None]
    most = z.amax(1)
    if whole:
        d = most[:, None] - z
        total = torch.exp(-d).sum(1)
        e_log = (torch.exp(-d) * (d * 2.0**-22 + 2.0**-19)).sum(1) / total + (64 + V / 1024) * 2.0**-24 + total.log() * 2.0**-23
        want = (most - z.gather(1, at)[:, 0]) + torch.log1p((torch.exp(-d).sum(1) - 1).clamp(min=0))
        assert ((got["loss"].double() - want).abs() <= e_log + want * 2.0**-23).all()
        lse = most + total.log()
        assert ((got["lse"].double() - lse).abs() <= e_log + lse * 2.0**-24).all()
    # a target's own term is (p - 1) / T, the others' p / T are not below 0
    p = torch.exp(z - torch.logsumexp(z, 1)[:, None]).scatter_(1, at, 0.0) * gl.double()[:, None]
    assert (got["grad_bias"].double()[targets.long()] <= p.sum(0)[targets.long()] * (1 + 2.0**-8) + 2.0**-126).all()


def test_large_logits():
    """Logits of hundreds: the maximum is taken out before the exponentials."""
    T, V, D = 65, 900, 64
    h, w, b, targets, gl = inputs(T, V, D)
    check_all((h.float() * 64).bfloat16(), w, b, targets, gl, qb.vocab_loss_workspace(T, V, D))
    b = torch.full_like(b, -5e4)
    b[::7] = 5e4
    check_all(h, w, b, targets, gl, qb.vocab_loss_workspace(T, V, D))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_finite(bad):
    T, V, D = 300, 600, 64
    h, w, b, targets, gl = inputs(T, V, D, ignored=False)
    ref = reference(h, w, b, targets, gl)
    h[290, 3] = bad
    ws = qb.vocab_loss_workspace(T, V, D)
    got = run(h, w, b, targets, gl, ws)
    keep = torch.arange(T, device="cuda") != 290
    for name in ("loss", "lse"):
        assert not torch.isfinite(got[name][290])
        assert ((got[name].double() - ref[name][0]).abs() <= ref[name][1])[keep].all()
    assert torch.isnan(got["grad_h"][290]).all()
    assert ((got["grad_h"].double() - ref["grad_h"][0]).abs() <= ref["grad_h"][1])[keep].all()
    assert torch.isnan(got["grad_w"]).all()  # the sum over the tokens meets it


@pytest.mark.parametrize("T", [3, 77, 129, 300])
def test_infinite_logits(T):
    """log sum exp with a term of +infinity is +infinity, with a NaN a NaN, of nothing but -infinity -infinity; other tokens' results stay."""
    V, D = 900, 64
    h, w, b, targets, gl = inputs(T, V, D, ignored=False)
    w[w[:, 5] == 0, 5] = 1.0
    ws = qb.vocab_loss_workspace(T, V, D)
    loss, lse = qb.vocab_loss(h, w, b, targets, ws)
    h[1, 5] = float("inf")  # logits of either infinity
    h[2, 5] = float("nan")
    got, got_lse = qb.vocab_loss(h, w, b, targets, ws)
    assert got_lse[1] == float("inf") and torch.isnan(got_lse[2]) and torch.isnan(got[2])
    up = float(w[int(targets[1]), 5]) > 0
    assert torch.isnan(got[1]) if up else got[1] == float("inf")
    keep = (torch.arange(T, device="cuda") != 1) & (torch.arange(T, device="cuda") != 2)
    assert torch.equal(got[keep], loss[keep]) and torch.equal(got_lse[keep], lse[keep])
    h[1, 5] = h[2, 5] = 0.0
    b[700] = float("inf")
    targets[0], targets[1], targets[2] = 700, -1, 3
    got, got_lse = qb.vocab_loss(h, w, b, targets, ws)
    assert (got_lse == float("inf")).all() and torch.isnan(got[0]) and got[1] == 0 and got[2] == float("inf")
    assert all(torch.isnan(grad).all() for grad in qb.vocab_loss_backward(h, w, b, targets, got_lse, gl, ws, needs=(False, True, True))[1:])
    got, got_lse = qb.vocab_loss(h, w, torch.full_like(b, -float("inf")), targets, ws)
    assert (got_lse == -float("inf")).all() and torch.isnan(got[0]) and got[1] == 0


@pytest.mark.parametrize("T", [77, 300])
def test_ignored_tokens_need_no_lse(T):
    """What the caller's lse holds for ignored tokens changes nothing."""
    V, D = 900, 64
    h, w, b, targets, gl = inputs(T, V, D)
    ws = qb.vocab_loss_workspace(T, V, D)
    _, lse = qb.vocab_loss(h, w, b, targets, ws)
    want = qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws)
    for other in (0.0, -200.0, float("nan"), -float("inf")):
        got = qb.vocab_loss_backward(h, w, b, targets, torch.where(targets < 0, torch.full_like(lse, other), lse), gl, ws)
        assert all(torch.equal(a, c) for a, c in zip(got, want))


@pytest.mark.parametrize("T", [1, 30, 77, 130, 300])
def test_infinite_weight(T):
    """A word whose logits are all -infinity by its weights: probability 0, so that its own gradients are 0."""
    V, D = 700, 64
    h, w, b, targets, gl = inputs(T, V, D, ignored=False)
    h[:, 9] = h[:, 9].abs() + 0.5
    out = torch.zeros(V, dtype=torch.bool, device="cuda")
    out[[5, 300, 699]] = True
    targets[out[targets.long()]] = 8
    ws = qb.vocab_loss_workspace(T, V, D)
    w[out] = 0.0
    b[out] = -float("inf")
    want = run(h, w, b, targets, gl, ws)
    w[out, 9] = -float("inf")
    got = run(h, w, torch.where(out, 0.0, b), targets, gl, ws)
    for name in ("loss", "lse", "grad_w", "grad_bias"):
        assert torch.equal(got[name], want[name]), name
    assert (got["grad_w"][out] == 0).all() and (got["grad_bias"][out] == 0).all()


def test_parts_of_the_gradient():
    T, V, D = 200, 1000, 192
    h, w, b, targets, gl = inputs(T, V, D)
    ws = qb.vocab_loss_workspace(T, V, D)
    _, lse = qb.vocab_loss(h, w, b, targets, ws)
    full = qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws)
    for needs in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        some = qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws, needs=needs)
        for n, s, f in zip(needs, some, full):
            assert (s is None) if not n else torch.equal(s, f)
    assert qb.vocab_loss_backward(h, w, None, targets, lse, gl, ws)[2] is None
    with pytest.raises(qb.QbertError):
        qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws, needs=(False, False, False))


def test_captured_shared_workspace_and_streams():
    """Graphs of two sizes over one workspace, replayed in turn with other calls of the library between them; another stream beside
    them with a workspace of its own."""
    ws, ws2 = qb.vocab_loss_workspace(700, 3000, 256), qb.vocab_loss_workspace(700, 3000, 256)
    s = torch.cuda.Stream()
    graphs = []
    for T, V, D in ((700, 3000, 256), (90, 1500, 128)):
        args = inputs(T, V, D)
        outs = [torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(args[0]), torch.empty_like(args[1]), torch.empty(V, device="cuda")]

        def call(args=args, outs=outs):
            qb.vocab_loss(*args[:4], ws, outs[0], outs[1])
            qb.vocab_loss_backward(*args[:4], outs[1], args[4], ws, *outs[2:])
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append((graph, args, outs))
    x = torch.randn(320, 1024, device="cuda")
    want = qb.quantize_act(x, qb.workspace())
    wt = torch.randn(768, 768, device="cuda")
    want_w = qb.quantize_pack_weights(wt, 4, 1, qb.workspace())
    for seed in (3, 4):
        for graph, args, outs in graphs:
            for old, new in zip(args, inputs(args[0].shape[0], args[1].shape[0], args[0].shape[1], seed)):
                old.copy_(new)
            s.wait_stream(torch.cuda.current_stream())
            graph.replay()
            with torch.cuda.stream(s):
                other = run(*args, ws2)
            got_x, got_w = qb.quantize_act(x, ws), qb.quantize_pack_weights(wt, 4, 1, ws)
            s.synchronize()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, other.values()))
            ref = reference(*args)
            for name, got in zip(ref, outs):
                check(name, got, ref)
            assert all(torch.equal(a, b) for a, b in zip(got_x, want)) and all(torch.equal(a, b) for a, b in zip(got_w, want_w))
    assert qb.read_status(ws) == qb.QB_OK and qb.read_status(ws2) == qb.QB_OK


def test_refusals():
    h, w, b, targets, gl = inputs(20, 50, 64)
    ws = qb.vocab_loss_workspace(20, 50, 64)
    _, lse = qb.vocab_loss(h, w, b, targets, ws)
    for args in ((h.float(), w, b, targets, ws), (h, w.t().contiguous(), b, targets, ws), (h, w.float(), b, targets, ws), (h, w, b.half(), targets, ws),
                 (h, w, b[:49], targets, ws), (h, w, b, targets.long(), ws), (h, w, b, targets[:19], ws), (h, w, b, None, ws), (h.cpu(), w, b, targets, ws),
                 (h[:, ::2], w[:, ::2], b, targets, ws), (h, w, b, targets, ws.cpu())):
        with pytest.raises(AssertionError):
            qb.vocab_loss(*args)
    for kw in (dict(grad_h=h.float()), dict(grad_h=h[:19]), dict(grad_w=w[:49]), dict(grad_bias=b[:49]), dict(grad_bias=b.half())):
        with pytest.raises(AssertionError):
            qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws, **kw)
    with pytest.raises(AssertionError):
        qb.vocab_loss_backward(h, w, b, targets, None, gl, ws)
    with pytest.raises(AssertionError):
        qb.vocab_loss_backward(h, w, b, targets, lse, gl.double(), ws)
    with pytest.raises(qb.QbertError):
        qb.vocab_loss(h[:, :60].contiguous(), w[:, :60].contiguous(), b, targets, ws)  # D not a multiple of 8
    with pytest.raises(qb.QbertError):
        qb.vocab_loss(h[:0], w, b, targets[:0], ws)


def test_gradients_of_another_shape():
    """As many elements in another shape are refused."""
    h, w, b, targets, gl = inputs(16, 48, 64)
    ws = qb.vocab_loss_workspace(16, 48, 64)
    _, lse = qb.vocab_loss(h, w, b, targets, ws)
    for kw in (dict(grad_h=torch.empty_like(h).view(64, 16)), dict(grad_h=torch.empty_like(h).view(-1)), dict(grad_w=torch.empty_like(w).view(64, 48))):
        with pytest.raises(AssertionError):
            qb.vocab_loss_backward(h, w, b, targets, lse, gl, ws, **kw)
