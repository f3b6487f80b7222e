"""The gated block's forward where every sum is exact: H held to its one rounding, element by element.

Inputs are small multiples of powers of two.  W' has at most 8 bits, every sum of products fits
24, so that G and U are exact in fp32 whatever the order, and stored they are their one rounding,
bit for bit.  H = act(G) U out of the unrounded sums is off by the fp32 steps of act (below 2^-15 of it,
where |G| < 8) and by its rounding, 2^-8 of itself; in tiles of ranks above 48 act(G) is rounded to bf16 on
the way as well.
"""
import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2501_08582_amd import ops
from tests.gpu_helpers import dev_to_f64

pytestmark = pytest.mark.gpu

U8 = 2.0**-8

# few tokens; such of wide projections, on both sides of what is left to thin tiles; whole tiles and edges, thin tiles behind them, ragged K; half-feature tiles
FEW = [(3, 136, 104, 5), (16, 4104, 72, 16), (33, 520, 192, 17), (7, 1032, 520, 128), (100, 520, 72, 64)]
THIN = [(4, 10000, 264, 16), (16, 8224, 1032, 48), (32, 8192, 520, 40), (20, 9216, 512, 40), (64, 4352, 1032, 32),
        (40, 8192, 264, 24), (32, 9280, 136, 40), (200, 2560, 200, 48)]
TILES = [(577, 1032, 200, 31), (768, 1024, 128, 16), (3328, 2560, 128, 48), (3299, 2560, 72, 33)]
WIDE_RANKS = [(577, 1032, 200, 64), (600, 1032, 192, 100), (3328, 2560, 64, 64), (1030, 520, 72, 128)]


def case(L, R, C, r, fmt):
    """X, and both projections' device tensors and W' of multiples of 2^-5, below 4: |G| below 8."""
    g = torch.Generator(device="cuda").manual_seed(L + R + C + r)

    def whole(least, most, *shape):
        return torch.randint(least, most + 1, shape, generator=g, device="cuda").double()

    X = whole(-4, 4, L, C) * 2.0**(-4 if C < 300 else -5)
    pair, merged = [], []
    for _ in range(2):
        if fmt == "2:4":
            place = torch.rand((R, C // 4, 4), generator=g, device="cuda").topk(2, dim=2).indices
            keep = torch.zeros((R, C // 4, 4), dtype=torch.bool, device="cuda").scatter_(2, place, True).view(R, C)
        else:
            keep = torch.rand((R, C), generator=g, device="cuda") < 0.5
        W = whole(-31, 31, R, C) * 2.0**-5 * keep
        B, A = whole(-1, 1, R, r) * 0.25, whole(-1, 1, r, C) * (torch.rand((r, C), generator=g, device="cuda") < 32 / (32 + r))
        low = B @ A * 0.5
        assert float(low.abs().max()) <= 96 * 2.0**-5
        merged.append((W + low) * keep)
        pair.append((W.bfloat16(), ops.mask_pack(keep, fmt), B.bfloat16(), A.bfloat16()))
        assert all(torch.equal(t.double(), s) for t, s in zip((pair[-1][0], *pair[-1][2:], merged[-1].bfloat16()), (W, B, A, merged[-1])))
    return X, pair, merged


@pytest.mark.parametrize("i,shape,roundings", [(i, s, n) for n, part in ((1, FEW + THIN + TILES), (2, WIDE_RANKS)) for i, s in enumerate(part)])
def test_forward(i, shape, roundings):
    L, R, C, r = shape
    fmt, act = ("bitmap", "2:4")[i % 2], ("silu", "gelu")[i // 2 % 2]
    X, pair, merged = case(L, R, C, r, fmt)
    H, G, U = ops.gated_forward(X.bfloat16(), *pair, 0.5, fmt, act)
    G64, U64 = (X @ W.T for W in merged)
    assert torch.equal(G64.float().double(), G64) and float(G64.abs().max()) < 8
    assert torch.equal(G, G64.float().bfloat16()) and torch.equal(U, U64.float().bfloat16())
    want = ob.act(dev_to_f64(G64), act)[0] * dev_to_f64(U64)
    err = np.abs(dev_to_f64(H) - want)
    # GELU: exp(-2t), |2t| <= 50, is off by 5.5 |2t| 2^-24 and its other steps by 8 . 2^-24
    bound = ((1 + U8) ** roundings - 1 + 2.0**-14) * np.abs(want)
    assert (err <= bound).all(), (float((err / np.maximum(np.abs(want), 1e-300)).max()), int((err > bound).sum()))
    assert torch.equal(ops.gated_forward(X.bfloat16(), *pair, 0.5, fmt, act, save=False)[0], H)


BACK = [(1, 8, 8, 1), (5, 72, 40, 3), (65, 520, 200, 12), (200, 264, 512, 64), (577, 1032, 200, 100), (333, 72, 1032, 128),
        (3328, 64, 2560, 16), (3328, 128, 2560, 64), (3300, 72, 2552, 33), (260, 1032, 10000, 5), (512, 1088, 10240, 64),
        (2100, 1032, 8200, 33), (40, 1032, 520, 128), (150, 264, 2056, 70)]


@pytest.mark.parametrize("most", [1, 7])
@pytest.mark.parametrize("i,shape", list(enumerate(BACK)))
def test_backward(i, shape, most):
    """At G = 32 both activations are G and their derivatives 1, so that dG = dH U and dU = 32 dH are exact in
    bf16, and all sums of products in fp32.  D = d^T X are whole numbers (32 times such), of at most 8 bits where
    the inputs are at most 1 and of at most 16 where they go up to 7, both of which the adapters'
    gradients take whole: dX is its one rounding and they are exact, bit for bit, whatever the order of their sums."""
    L, R, C, r = shape
    fmt, act = ("2:4", "bitmap")[i % 2], ("silu", "gelu")[i // 2 % 2]
    _, pair, merged = case(L, R, C, r, fmt)
    g = torch.Generator(device="cuda").manual_seed(i)

    def whole(*shape):
        return torch.randint(-most, most + 1, shape, generator=g, device="cuda").double()

    X, dH, G = whole(L, C), whole(L, R), torch.full((L, R), 32.0, device="cuda").double()
    U = torch.where(torch.rand((L, R), generator=g, device="cuda") < 0.5, 1.0, -1.0).double()
    dX, gate, up = ops.gated_backward(*(t.bfloat16() for t in (dH, X)), *pair, G.bfloat16(), U.bfloat16(), 0.5, fmt, act)
    dG, dU = dH * U, dH * G
    assert torch.equal(dX, (dG @ merged[0] + dU @ merged[1]).float().bfloat16())
    for (dB, dA), d, (_, M, B, A) in zip((gate, up), (dG, dU), pair):
        D = (d.T @ X) * ops.mask_unpack(M, R, C, fmt).bool()
        first = D.bfloat16().double()
        assert torch.equal(first + (0.0 if most == 1 else (D - first).bfloat16().double()), D)
        assert torch.equal(dB, (0.5 * D @ A.double().T).float()) and torch.equal(dA, (0.5 * B.double().T @ D).float())


@pytest.mark.parametrize("r", [5, 40])
def test_infinite_gradients_reach_what_they_reach(r):
    """An Inf of dH makes the sums infinite that hold it with a kept weight, all terms being positive, and
    no other; in masked places it is nothing."""
    L, R, C = 70, 72, 136
    _, pair, _ = case(L, R, C, r, "bitmap")
    pair = [(W, M, B.abs() + 1, A.abs() + 1) for W, M, B, A in pair]
    X, dH = torch.ones(L, C, device="cuda").bfloat16(), torch.ones(L, R, device="cuda").bfloat16()
    dH[64, 7] = float("inf")
    G, U = torch.full((L, R), 32.0, device="cuda").bfloat16(), torch.ones(L, R, device="cuda").bfloat16()
    _, gate, up = ops.gated_backward(dH, X, *pair, G, U, 0.5)
    for (dB, dA), (_, M, _, _) in zip((gate, up), pair):
        kept = ops.mask_unpack(M, R, C).bool()
        assert kept[7].any() and not kept[7].all()
        wantB, wantA = torch.zeros(R, r, dtype=torch.bool, device="cuda"), kept[7].expand(r, C)
        wantB[7] = True
        assert torch.equal(dB == float("inf"), wantB) and torch.equal(dA == float("inf"), wantA)
        assert torch.isfinite(dB[~wantB]).all() and torch.isfinite(dA[~wantA]).all()
