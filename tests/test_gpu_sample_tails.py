"""Sampling of rows whose many smallest weights count, against their definition in whole numbers.

Logits are whole numbers and the temperature 1 / ln 2, so that weights are powers of two: the
definition is computed exactly, in integers.  (64-bit running sums are not: 40000 entries of 2^-60 behind a
sum of 19, whose steps are 2^-48, each round away, and with them the border of top_p = 1/2, which
lies 20000 . 2^-60 above the sum before an entry.)  The kernels' sums are off by a few 2^-48, the borders
at least 2^-46 from an entry: tokens are equal.  logp is rounded once (2^-24).
"""
import itertools
import math
from bisect import bisect_left, bisect_right
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2501_08582_amd import train

pytestmark = pytest.mark.gpu

T = 1.44269504088896340736
BELOW_ONE = float(np.nextafter(np.float32(1), np.float32(0)))


class Row:
    """Weights times 2^256 of one row (those below it are 0), by index and in their order."""

    def __init__(self, z, dtype):
        self.t = torch.from_numpy(z.astype(np.float32)).to(dtype).cuda().unsqueeze(0)
        assert np.array_equal(self.t[0].double().cpu().numpy(), z)
        power = [1 << i for i in range(257)]
        self.w = [power[256 + int(x)] if x >= -256 else 0 for x in z]
        self.order = np.argsort(-z, kind="stable")
        self.run = list(itertools.accumulate(self.w[i] for i in self.order))

    def sample(self, u, top_p, top_k=0):
        """(token, its weight over the whole)"""
        k = top_k or len(self.w)
        goal = Fraction(top_p) * self.run[k - 1]
        n = min(k, 1 + bisect_left(self.run, goal))  # the first entry, and those with less than the goal before them
        at = np.sort(self.order[:n])
        run = list(itertools.accumulate(self.w[i] for i in at))
        j = bisect_right(run, Fraction(float(np.float32(u))) * run[-1])
        return int(at[j]), Fraction(self.w[at[j]], run[-1])


def check(row, u, **kw):
    token, logp = train.sample(row.t, torch.tensor([u], device="cuda"), T, **kw)
    want, share = row.sample(u, **kw)
    low = math.log1p(float(share - 1)) if 2 * share > 1 else math.log(share)
    # logp: the temperature's rounding moves a weight of 2^-43 by 2^-53 of its logarithm
    assert int(token) == want and abs(float(logp) - low) <= 2.0**-24 * abs(low) + 2.0**-40, (int(token), want)
    return want


def tail(V, depth, dtype):
    """One entry of weight 1 before V - 1 of 2^-depth; in bf16 with one that no value stands for."""
    z = np.full(V, -float(depth))
    z[0] = 0.0
    if dtype == torch.bfloat16:
        z[V - 1] = -2.0**20
    return z


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,depth", [(1200007, 43), (1200007, 42), (131071, 40), (600011, 41)])
def test_a_tail_of_tiny_weights_is_kept_as_far_as_top_p_goes(V, depth, dtype):
    """Weights that fixed point of the whole row's range would round away or up."""
    row = Row(tail(V, depth, dtype), dtype)
    w = 2.0**-depth
    n = V - 1 if dtype == torch.float32 else V - 2
    seen = set()
    for share in (0.1, 0.55, 0.9):  # of the tail: borders half a weight from an entry
        p = (1.0 + (int(share * n) - 0.5) * w) / (1.0 + n * w)
        for u in (0.5, BELOW_ONE):
            seen.add(check(row, u, top_p=p))
            seen.add(check(row, u, top_p=p, top_k=int(0.95 * V)))
    # the largest random number lies in the tail of the longest rows
    assert (max(seen) > 0) == (0.9 * n * w > 2.0**-24)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tails_of_several_depths(dtype):
    """Every bin of the first pass and the last one's far entries, each depth as heavy as the one before."""
    parts = [np.full(1 << k, -float(k)) for k in range(19)] + [np.full(40000, -60.0), np.full(20000, -200.0)]
    rng = np.random.default_rng(0)
    z = rng.permutation(np.concatenate(parts))
    if dtype == torch.bfloat16:
        z[rng.integers(len(z))] = -2.0**20
    row = Row(z, dtype)
    for p in (0.03, 0.2, 0.5, 0.77, 0.999, 1.0 - 2.0**-40):
        for u in (0.0, 0.3, 0.8, BELOW_ONE):
            check(row, u, top_p=p)
            check(row, u, top_p=p, top_k=300001)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_at_the_end_of_the_range(dtype):
    """The least weights that 64 bits hold count: u = 0 takes the first, and the next below it is none."""
    for depth, first in ((1001, True), (1022, True), (1074, True), (1076, False), (2000, False)):
        z = np.full(40, -np.inf)
        z[[3, 5, 30]] = -2000.0
        z[7] = -depth if dtype == torch.float32 else -1000.0
        z[9] = 0.0
        # bf16 has not all these numbers: -1000, by the temperature
        temperature = T if dtype == torch.float32 else T * 1000.0 / depth
        t = torch.from_numpy(z.astype(np.float32)).to(dtype).cuda().unsqueeze(0)
        token, logp = train.sample(t, torch.zeros(1, device="cuda"), temperature)
        assert int(token) == (7 if first else 9), depth
        # (of 2^-1074 and what rounds to it the logarithm is that number's)
        assert abs(float(logp) + (depth * math.log(2.0) if first else 0.0)) <= 2.0**-24 * 745
        token, _ = train.sample(t, torch.ones(1, device="cuda"), temperature)
        assert int(token) == 9  # nothing behind it has a weight
