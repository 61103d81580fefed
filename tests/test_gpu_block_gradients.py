"""The gradients of an encoder block's step against differences of its loss, over enough directions to see a term of a few percent."""
import pytest
import torch

from test_gpu_block_step import EPS, Block
from test_gpu_checkpoint import gelu64
from test_gpu_layer_norm import forward64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("save", ["pre", "codes"])
def test_gradients_against_differences(save):
    """Along normal directions v the mean square of (quotient - grad . v) is the square of the gradient's error (of its norm, over 64 directions: to a
    fifth).  fp16 rounds six tensors between the loss and a gradient by 2^-11 of a value at most, 2^-8.4 of the norm if all of it added up;
    half a step of a code is 1 / 254 of its block's maximum, which is about 2.5 times the block's root mean square, 1 % of the norm at most and 0.6 % as a
    uniform error, in the slope and in h.  The differences' own error (h^2 times the third derivative) is below 2^-16.  A term of 5 % that was
    missing would show as 5 %."""
    b = Block(40, 64, 96, 5, torch.float16, save)
    got = b.run()

    def loss(x, w1, w2, b1, b2, gamma, beta):
        s = gelu64(x @ w1.t() + b1) @ w2.t() + b2 + x
        return (forward64(s, gamma, beta, EPS)[0] * b.dy.double()).sum()
    leaves = [t.double() for t in (b.x, b.w1, b.w2, b.b1, b.b2, b.gamma, b.beta)]
    h, n = 2.0**-12, 64
    for i, name in enumerate(("x", "w1", "w2", "b1", "b2", "dgamma", "dbeta")):
        g = torch.Generator(device="cuda").manual_seed(i)
        square = 0.0
        for _ in range(n):
            v = torch.randn(leaves[i].shape, device="cuda", generator=g, dtype=torch.float64)
            ends = []
            for sign in (1, -1):
                args = list(leaves)
                args[i] = args[i] + sign * h * v
                ends.append(loss(*args))
            square += ((ends[0] - ends[1]) / (2 * h) - (got[name].double() * v).sum()) ** 2 / n
        off = float(square.sqrt() / got[name].double().norm())
        assert off <= (2.0**-8 if save == "pre" else 2.0**-6) * 1.2, (name, off)
