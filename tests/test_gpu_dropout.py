"""Dropout from a counter: masks word for word against Philox written in numpy, values against 64 bits."""
import numpy as np
import pytest
import torch

import paper_1909_05840_b200 as qb

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def philox(counter, key, rounds):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw, SC 2011) on Python whole numbers or numpy uint64 arrays."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def words(index, seed, sub):
    """The 32-bit words of the elements `index` (numpy int64)."""
    i = index.astype(np.uint64) // np.uint64(4)
    u = np.uint64
    c = [i & u(0xFFFFFFFF), i >> u(32), np.full_like(i, sub & 0xFFFFFFFF), np.full_like(i, sub >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & u(0xFFFFFFFF), (a >> u(32)) ^ c[3] ^ u(k[1]), a & u(0xFFFFFFFF)]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.choose(index % 4, c)


def test_philox_known_answers():
    """The published test vectors of the generator (key and counter of zeros and of ones), seven and ten rounds."""
    ones = 0xFFFFFFFF
    assert philox([0] * 4, [0] * 2, 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert philox([0] * 4, [0] * 2, 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox([ones] * 4, [ones] * 2, 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    i = np.array([0, 1, 2, 3, 4, 4 * 5 + 1, (1 << 34) + 2], dtype=np.int64)
    seed, sub = 0x0123456789ABCDEF, (7 << 32) + 9
    want = [philox([(n // 4) & ones, n // 4 >> 32, 9, 7], [0x89ABCDEF, 0x01234567], 7)[n % 4] for n in i.tolist()]
    assert words(i, seed, sub).tolist() == want


def rng(seed=0x0123456789ABCDEF, offset=(7 << 32) + 5):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def check(y, x, p, state, call, residual=None, index=None):
    """`y` against 64 bits.  Roundings: 1 / (1 - p) and its product with x (2^-24 each of |x s|), the sum (2^-24 of |y|), the
    type's own (half its step; half the step of its subnormals, 2^-25 for fp16)."""
    index = np.arange(x.numel(), dtype=np.int64) if index is None else index
    seed, offset = state.tolist()
    keep = words(index, seed, offset + call) >= np.uint64(min(round(p * 2**32), 2**32 - 1))
    xs, ys = x.reshape(-1).double().cpu().numpy(), y.reshape(-1).double().cpu().numpy()
    scaled = np.where(keep, xs, 0.0) / (1.0 - p)
    want = scaled + (0.0 if residual is None else residual.reshape(-1).double().cpu().numpy())
    half = torch.finfo(y.dtype).eps / 2
    least = 2.0**-25 if y.dtype == torch.float16 else 2.0**-150
    tol = np.abs(scaled) * 2.0**-23 * (1 + half) + np.abs(want) * (2.0**-24 + half) * (1 + half) + least
    finite = np.isfinite(want)
    assert (np.abs(ys - want)[finite] <= tol[finite]).all()
    if residual is None:
        assert (ys[~keep] == 0).all()
    return keep


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 3, 4, 5, 8, 4095, 4096, 4099, 1000003])
def test_values(n, kind, p, residual):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, device="cuda", generator=g).to(TYPES[kind])
    r = torch.randn(n, device="cuda", generator=g).to(TYPES[kind]) if residual else None
    state = rng()
    buffer = torch.full((n + 64,), 7.0, dtype=x.dtype, device="cuda")
    y = qb.dropout(x, p, state, call=3, residual=r, out=buffer[:n])
    keep = check(y, x, p, state, 3, r)
    assert (buffer[n:] == 7.0).all()
    if n > 1000000 and p > 0:  # binomial: six standard deviations
        assert abs(keep.mean() - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5


# rows of a matrix that begin at any address: the same values as aligned ones
@pytest.mark.gpu
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_any_alignment(kind, shift):
    n, state = 2049, rng()
    x = torch.randn(n + 8, device="cuda").to(TYPES[kind])
    r = torch.randn(n + 8, device="cuda").to(TYPES[kind])
    want = qb.dropout(x[shift:shift + n].clone(), 0.3, state, residual=r[:n].clone())
    out = torch.empty(n + 8, dtype=x.dtype, device="cuda")[8 - shift:8 - shift + n]
    assert torch.equal(qb.dropout(x[shift:shift + n], 0.3, state, residual=r[:n], out=out), want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_in_place_and_backward(kind):
    """The gradient is the same call on the gradient: against differences of the forward pass, which is linear in x."""
    state, M, N = rng(), 37, 129
    x = torch.randn(M, N, device="cuda").to(TYPES[kind])
    r = torch.randn(M, N, device="cuda").to(TYPES[kind])
    y = qb.dropout(x, 0.25, state, 11, r)
    z = x.clone()
    assert qb.dropout(z, 0.25, state, 11, r, out=z) is z and torch.equal(z, y)
    z = r.clone()
    assert torch.equal(qb.dropout(x, 0.25, state, 11, z, out=z), y)
    dy = torch.ones_like(x)
    dx = qb.dropout(dy, 0.25, state, 11)
    # powers of two: the difference quotient is exact up to the rounding of 1 / 0.75 to the type
    one, two = torch.full_like(x, 1.0), torch.full_like(x, 2.0)
    quotient = qb.dropout(two, 0.25, state, 11).double() - qb.dropout(one, 0.25, state, 11).double()
    assert ((quotient - dx.double()).abs() <= 2 * torch.finfo(x.dtype).eps * 1.34).all()
    assert torch.equal(dx != 0, qb.dropout(one, 0.25, state, 11) != 0)
    assert not torch.equal(dx, qb.dropout(dy, 0.25, state, 12))


@pytest.mark.gpu
def test_dropped_infinities():
    state, n = rng(), 4096
    keep = check(qb.dropout(torch.ones(n, device="cuda"), 0.5, state), torch.ones(n, device="cuda"), 0.5, state, 0)
    for bad in (float("inf"), -float("inf"), float("nan")):
        y = qb.dropout(torch.full((n,), bad, device="cuda"), 0.5, state).cpu().numpy()
        assert (y[~keep] == 0).all() and not np.isfinite(y[keep]).any()


@pytest.mark.gpu
def test_seeds_beyond_32_bits_and_wrapping_offsets():
    n = 8192
    x = torch.ones(n, device="cuda")
    for seed, offset, call in ((-1, -1, 1), (1 << 62, (1 << 63) - 1, 3), (5, 0, (1 << 64) - 1)):
        state = rng(seed, offset)
        got = qb.dropout(x, 0.5, state, call) != 0
        low = (1 << 64) - 1
        want = words(np.arange(n), seed & low, (offset + call) & low) >= np.uint64(1 << 31)
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.gpu
def test_more_than_2_to_32_elements():
    n = (1 << 32) + 1027
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    state = rng()
    qb.dropout(x, 0.5, state, 2, out=x)
    for lo in (0, (1 << 31) - 512, (1 << 32) - 512, n - 1000):
        index = np.arange(lo, min(lo + 1024, n), dtype=np.int64)
        part = x[lo:lo + index.size]
        check(part, torch.ones_like(part), 0.5, state, 2, index=index)


@pytest.mark.gpu
def test_captured_step_draws_new_masks():
    x = torch.ones(5000, device="cuda")
    state, y, dx = rng(9, 100), torch.empty(5000, device="cuda"), torch.empty(5000, device="cuda")

    def step():
        qb.dropout(x, 0.5, state, 1, out=y)
        qb.dropout(x, 0.5, state, 1, out=dx)
        state[1] += 2
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state[1] = 100
    seen = []
    for k in range(3):
        graph.replay()
        assert torch.equal(y, dx)
        check(y, x, 0.5, rng(9, 100 + 2 * k), 1)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


@pytest.mark.gpu
def test_other_stream():
    s, state = torch.cuda.Stream(), rng()
    x = torch.randn(100000, device="cuda")
    want = qb.dropout(x, 0.1, state)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = qb.dropout(x, 0.1, state)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_refusals():
    x, state = torch.ones(64, device="cuda"), rng()
    for p in (-0.1, 1.0, float("nan")):
        with pytest.raises(qb.QbertError):
            qb.dropout(x, p, state)
    with pytest.raises(qb.QbertError):
        qb.dropout(x[:0], 0.1, state)
    for bad in (dict(x=x.double()), dict(x=x.cpu()), dict(x=x.view(8, 8).t()), dict(rng=state.int()), dict(rng=state[:1]), dict(rng=state.cpu()),
                dict(residual=x[:32]), dict(residual=x.half()), dict(out=x[:32]), dict(out=x.bfloat16()), dict(out=torch.empty(64))):
        args = dict(x=x, p=0.1, rng=state)
        args.update(bad)
        with pytest.raises(AssertionError):
            qb.dropout(**args)
    with pytest.raises((OverflowError, TypeError)):
        qb.dropout(x, 0.1, state, call=-1)


@pytest.mark.gpu
def test_p_next_to_one():
    """Element 195 of this mask has the word 2^32 - 1: it is kept while round(p * 2^32) is no larger, and dropped beyond."""
    assert int(words(np.array([195]), 1, 9601978)[0]) == 2**32 - 1
    x, state = torch.ones(256, device="cuda"), rng(1, 9601978)
    kept = qb.dropout(x, 1 - 2.0**-32, state)
    assert kept[195] == 2.0**32 and int((kept != 0).sum()) == 1
    for p in (1 - 2.0**-34, 1 - 2.0**-53):
        assert not qb.dropout(x, p, state).any() and torch.equal(qb.dropout(x, p, state, residual=x), x)
