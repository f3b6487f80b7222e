"""CPU tests that pin the fp64 definitions of the gated block, the orthogonalised
updates and the sampling: by differences, singular values, enumeration."""
import itertools

import numpy as np
import pytest

from oracle import block as ob


# ---------------------------------------------------------------------------
# gated
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activations(kind):
    g = np.linspace(-12, 12, 481)
    y, d = ob.act(g, kind)
    h = 1e-6
    # central differences: h^2 / 6 of the third derivative (below 2) and roundings of 2^-53 / h
    assert np.abs((ob.act(g + h, kind)[0] - ob.act(g - h, kind)[0]) / (2 * h) - d).max() < 1e-8
    assert y[240] == 0.0 and d[240] == 0.5
    # far out the identity, or nothing: silu's tail is |g| exp(-|g|), the other's much smaller
    tail = np.abs(g) * np.exp(-np.abs(g)) + 1e-15 if kind == "silu" else 1e-6 + 0 * g
    assert (np.abs(y - np.maximum(g, 0.0))[np.abs(g) > 5] <= tail[np.abs(g) > 5]).all()


def block(seed, L=5, R=8, C=12, r=3):
    rng = np.random.default_rng(seed)

    def projection():
        keep = rng.random((R, C)) < 0.5
        return [rng.standard_normal((R, C)) * keep, keep, rng.standard_normal((R, r)), rng.standard_normal((r, C))]

    return rng, rng.standard_normal((L, C)), projection(), projection()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_gradients_by_differences(kind):
    rng, X, gate, up = block(1)
    s = 0.7
    H, G, U = ob.gated_forward(X, gate, up, s, kind, "f32")
    dH = rng.standard_normal(H.shape)
    dX, (dBg, dAg), (dBu, dAu) = ob.gated_backward(dH, X, gate, up, G, U, s, kind, "f32")

    def value(X, gate, up):
        return (dH * ob.gated_forward(X, gate, up, s, kind, "f32")[0]).sum()

    h = 1e-5
    for got, which in ((dX, None), (dBg, (0, 2)), (dAg, (0, 3)), (dBu, (1, 2)), (dAu, (1, 3))):
        for _ in range(5):
            step = rng.standard_normal(got.shape)
            ends = []
            for sign in (h, -h):
                x, q = X, [list(gate), list(up)]
                if which is None:
                    x = X + sign * step
                else:
                    q[which[0]][which[1]] = q[which[0]][which[1]] + sign * step
                ends.append(value(x, *q))
            want = (got * step).sum()
            # h^2 of third derivatives of about the value's own size, and its roundings over h
            assert abs((ends[0] - ends[1]) / (2 * h) - want) <= 1e-6 * (abs(want) + abs(ends[0]))


def test_pruned_weights_stay_out():
    _, X, gate, up = block(2)
    other = list(gate)
    other[0] = gate[0] + 5.0 * ~gate[1]  # values under the mask
    a, b = (ob.gated_forward(X, q, up, 0.7, "silu", "f32")[0] for q in (gate, other))
    assert np.array_equal(a, b)
    assert not ob.weight(other, 0.7, "f32")[~gate[1]].any()


# ---------------------------------------------------------------------------
# update
# ---------------------------------------------------------------------------
ABC = (3.4445, -4.775, 2.0315)


@pytest.mark.parametrize("shape", [(4, 9), (9, 4), (6, 6), (1, 5)])
@pytest.mark.parametrize("steps", [1, 5])
def test_direction_acts_on_singular_values(shape, steps):
    v = np.random.default_rng(3).standard_normal(shape)
    u, sv, w = np.linalg.svd(v, full_matrices=False)
    s = sv / (np.sqrt((sv * sv).sum()) + 1e-7)
    a, b, c = ABC
    for _ in range(steps):
        s = a * s + b * s**3 + c * s**5
    # roundings of 2^-53 and the steps' gain, 485 at most
    assert np.abs(ob.direction(v, steps, *ABC, 1e-7) - (u * s) @ w).max() < 1e-11


def test_cubic_steps_reach_the_orthogonal_factor():
    v = np.random.default_rng(4).standard_normal((5, 11))
    u, _, w = np.linalg.svd(v, full_matrices=False)
    assert np.abs(ob.direction(v, 40, 1.5, -0.5, 0.0, 0.0) - u @ w).max() < 1e-12


@pytest.mark.parametrize("nesterov", [False, True])
def test_update(nesterov):
    rng = np.random.default_rng(5)
    g, m, w = (rng.standard_normal((3, 8)) for _ in range(3))
    m1, w1 = ob.update(g, m, w, 0.8, nesterov, 0.3, 0.05, 5, *ABC, 1e-7)
    assert np.allclose(m1, 0.8 * m + 0.2 * g, rtol=1e-15, atol=1e-15)
    v = 0.8 * m1 + 0.2 * g if nesterov else m1
    assert np.allclose(w1, 0.95 * w - 0.3 * ob.direction(v, 5, *ABC, 1e-7), rtol=1e-14, atol=1e-14)


# ---------------------------------------------------------------------------
# sample
# ---------------------------------------------------------------------------
def slow(z, u, temperature, top_k, top_p, min_p):
    """One step after the other in plain Python."""
    order = sorted(range(len(z)), key=lambda i: (-z[i], i))
    if temperature == 0:
        return order[0], 0.0
    w = {i: np.exp((z[i] - z[order[0]]) / temperature) for i in order}
    if top_k > 0:
        order = order[:top_k]
    whole, run, held = sum(w[i] for i in order), 0.0, []
    for i in order:
        if top_p < 1.0 and held and run >= top_p * whole:
            break
        held.append(i)
        run += w[i]
    held = [held[0]] + [i for i in held[1:] if w[i] >= min_p]
    whole, run = sum(w[i] for i in sorted(held)), 0.0
    for i in sorted(held):
        run += w[i]
        if run > u * whole:
            return i, np.log(w[i] / whole)
    last = [i for i in sorted(held) if w[i] > 0][-1]
    return last, np.log(w[last] / whole)


@pytest.mark.parametrize("seed", range(3))
def test_sample_against_plain_steps(seed):
    rng = np.random.default_rng(seed)
    for V, T, k, p, low in itertools.product((1, 2, 9, 40), (0.0, 0.6, 1.0, 3.0), (0, 1, 4), (0.0, 0.5, 0.93, 1.0), (0.0, 0.1, 1.0)):
        z = np.round(2 * rng.standard_normal(V), 1)  # with equal entries
        u = float(rng.random())
        t, logp = ob.sample(z, u, T, k, p, low)
        wt, wl = slow(list(z), u, T, k, p, low)
        assert t == wt and abs(logp - wl) < 1e-12, (z, u, T, k, p, low)


def test_sample_frequencies():
    """Every u of a fine grid: each token as often as its share, to two grid steps."""
    z = np.array([0.3, -1.0, 2.0, 0.3, -0.5])
    n = 4000
    hits = np.bincount([ob.sample(z, (i + 0.5) / n)[0] for i in range(n)], minlength=5)
    w = np.exp(z - z.max())
    assert np.abs(hits - n * w / w.sum()).max() <= 2


def test_rows_without_a_distribution():
    for z in ([np.nan, 1.0], [np.inf, 1.0], [-np.inf, -np.inf]):
        t, logp = ob.sample(z, 0.5)
        assert t == -1 and np.isnan(logp)
    assert ob.sample([-np.inf, 0.0, -np.inf], 0.9)[0] == 1
