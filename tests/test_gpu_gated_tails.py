"""The gated block's activations where they are small or their arguments large, element by element.

A weight of one entry a row makes G and U multiples of the input, without rounding (fp32: exactly
x).  Relative errors of GELU g s, s = 1 / (1 + exp(-2t)), t = k g (1 + 0.044715 g^2), in fp32: t is off by
four roundings; exp(-2t) by |2t| times those, the product with log2(e) and that constant's own, and by
one unit of its own; the other steps by six roundings: (5.5 |2t| + 8) 2^-24.  The derivative s (1 + 2 g (1 - s) t')
and the sum of both projections' terms lose up to a factor 2 each to cancellation at g <= -2.
"""
import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2501_08582_amd import ops
from tests.gpu_helpers import dev_to_f64

pytestmark = pytest.mark.gpu

K = np.sqrt(2.0 / np.pi)
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(x, up, act, dtype):
    """(x, H, dX / n) with G = x, U = up . x and dH = 1, in 64 bits."""
    L, n = len(x), 8
    X = torch.zeros(L, n)
    X[:, 0] = torch.from_numpy(x)
    X = X.to(DT[dtype]).cuda()
    M = ops.mask_pack(torch.ones(n, n, dtype=torch.bool, device="cuda"))
    pair = []
    for value in (1.0, up):
        W = torch.zeros(n, n, dtype=DT[dtype], device="cuda")
        W[:, 0] = value
        pair.append((W, M, torch.zeros(n, 1, dtype=DT[dtype], device="cuda"), torch.zeros(1, n, dtype=DT[dtype], device="cuda")))
    H, G, U = ops.gated_forward(X, *pair, 1.0, activation=act)
    x64 = dev_to_f64(X)[:, 0]
    assert np.array_equal(dev_to_f64(G)[:, 0], x64)
    dX = ops.gated_backward(torch.ones_like(H), X, *pair, G, U, 1.0, activation=act)[0]
    return x64, dev_to_f64(H)[:, 0], dev_to_f64(dX)[:, 0] / n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gelu_far_below_zero(dtype):
    """1 + tanh must not be a difference of nearly equal numbers there."""
    x, H, dX = run(-np.linspace(2.0, 9.5, 61).astype(np.float32), 1.0, "gelu", dtype)
    y, d = gelu(x)
    t = K * x * (1.0 + 0.044715 * x * x)
    err = (5.5 * np.abs(2 * t) + 8) * 2.0**-24
    one = 0.0 if dtype == "f32" else 2.0**-8  # H: a rounding; dX: of dG, dU and itself
    assert (np.abs(H - y * x) <= (err + one) * np.abs(y * x) * 1.01).all()
    parts = np.abs(d * x) + np.abs(y)
    assert (np.abs(dX - (d * x + y)) <= 4 * err * np.abs(d * x + y) + 1.01 * one * (parts + np.abs(d * x + y))).all()


def gelu(x):
    """The oracle's, without its own cancellation: 1 + tanh(t) = 2 s."""
    t = K * (x + 0.044715 * x**3)
    s = 1.0 / (1.0 + np.exp(-2.0 * t))
    y, d = x * s, s + 2.0 * x * s * (1.0 - s) * K * (1.0 + 3 * 0.044715 * x * x)
    far = x > -4.0  # where the two forms agree in 64 bits
    assert np.allclose(y[far], ob.act(x[far], "gelu")[0], rtol=1e-9) and np.allclose(d[far], ob.act(x[far], "gelu")[1], rtol=1e-9)
    return y, d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_arguments_whose_squares_overflow(act, dtype):
    """act(g) = g or 0 and its derivative 1 or 0 up to the largest numbers."""
    x = np.array([1e10, 1e19, 2e19, 1e25, 1e30, 3e38, -1e10, -2e19, -1e30, -3e38], np.float32)
    up = 2.0**-100
    x, H, dX = run(x, up, act, dtype)
    on = x > 0
    want = x[on] * (x[on] * up)
    want[want > torch.finfo(DT[dtype]).max] = np.inf
    assert np.allclose(H[on], want, rtol=2.0**-8 * 1.01)
    assert np.allclose(dX[on], 2 * x[on] * up, rtol=2.0**-6)
    assert not H[~on].any() and not dX[~on].any()
