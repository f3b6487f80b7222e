"""CPU pins of the oracle of the operators around the layer: known answers of the
generator, closed forms, and central differences of every gradient.

Differences are taken in fp64 with a step of 1e-5: truncation and rounding are both
below 1e-9 of the values here, and 1e-6 is asserted."""
import numpy as np
import pytest

from oracle import train as ot

STEP, TOL = 1e-5, 1e-6


def _difference(f, x, rng):
    """(numerical, direction) of the scalar f at x along a random direction."""
    v = rng.standard_normal(x.shape)
    return (f(x + STEP * v) - f(x - STEP * v)) / (2 * STEP), v


# the published known answers of philox4x32-10
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, want):
    assert tuple(ot.philox_block(counter, key)) == want


def test_random16_takes_blocks_by_column_and_row():
    seed, offset = 0x299F31D0A4093822, 0x0370734413198A2E
    got = ot.random16(5, 19, seed, offset)
    for n in range(5):
        for c in range(19):
            w = ot.philox_block((c // 8, n, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0))
            assert got[n, c] == w[c % 8 // 2] >> 16 * (c % 2) & 0xFFFF


def test_dropout_rate_and_scale():
    x = np.ones((400, 1000))
    for p in (0.0, 0.05, 0.5, 0.9):
        y, kept = ot.dropout(x, p, 1234, 5)
        q = 1 - ot.threshold(p) / 65536
        # 4e5 draws: six standard deviations
        assert abs(kept.mean() - q) <= 6 * np.sqrt(q * (1 - q) / x.size)
        assert np.array_equal(y, np.where(kept, 1 / q, 0.0)) or np.allclose(y[kept], 1 / q, rtol=1e-15)
    a, b = (ot.dropout(x, 0.5, s, o)[1] for s, o in ((1, 0), (1, 1)))
    assert abs((a == b).mean() - 0.5) < 6 * 0.5 / np.sqrt(x.size)


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradient_by_differences(rms):
    rng = np.random.default_rng(3)
    z, w, b = rng.standard_normal((4, 11)) * 2 + 0.5, rng.standard_normal(11), rng.standard_normal(11)
    dy, dz = rng.standard_normal((2, 4, 11))
    got = ot.norm_backward(dy, z, w, 1e-3, rms, dz)
    num, v = _difference(lambda q: (dy * ot.norm(q, w, b, 1e-3, rms)).sum() + (dz * q).sum(), z, rng)
    assert abs(num - (got[0] * v).sum()) < TOL
    num, v = _difference(lambda q: (dy * ot.norm(z, q, b, 1e-3, rms)).sum(), w, rng)
    assert abs(num - (got[1] * v).sum()) < TOL
    num, v = _difference(lambda q: (dy * ot.norm(z, w, q, 1e-3, rms)).sum(), b, rng)
    assert abs(num - (got[2] * v).sum()) < TOL


def test_norm_closed_forms():
    z = np.array([[1.0, 3.0], [-2.0, -2.0]])
    assert np.allclose(ot.norm(z[:1], None, None, 0.0, False)[0], [-1, 1])
    assert np.allclose(ot.norm(z, None, None, 1.0, False)[1], [0, 0])
    assert np.allclose(ot.norm(z, None, None, 0.0, True), [z[0] / np.sqrt(5), z[1] / 2])


def test_embedding_gradient_by_differences():
    rng = np.random.default_rng(4)
    ids = np.array([2, -1, 0, 2, 7, 2, 5])
    table, dy = rng.standard_normal((6, 5)), rng.standard_normal((7, 5))
    y = ot.embedding(ids, table, 0.5)
    assert not y[1].any() and not y[4].any() and np.array_equal(y[0], 0.5 * table[2])
    got = ot.embedding_backward(dy, ids, 6, 0.5)
    num, v = _difference(lambda q: (dy * ot.embedding(ids, q, 0.5)).sum(), table, rng)
    assert abs(num - (got * v).sum()) < TOL


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_gradient_by_differences(smoothing):
    rng = np.random.default_rng(5)
    P, S, V, beta = 3, 4, 9, 0.3
    x = rng.standard_normal((2 * P * S, V)) * 2
    t = rng.integers(0, V, 2 * P * S)
    t[[0, 5, 6]] = -100
    counts = (t >= 0).reshape(2 * P, S)
    ref = rng.standard_normal((2 * P, S)) - 2

    def loss(q):
        return ot.preference(ot.logprobs(q, t)[0].reshape(2 * P, S), counts, ref, beta, smoothing)[0]

    dseq = ot.preference(ot.logprobs(x, t)[0].reshape(2 * P, S), counts, ref, beta, smoothing)[2]
    got = ot.logprobs_backward(np.repeat(dseq, S), x, t)
    num, v = _difference(loss, x, rng)
    assert abs(num - (got * v).sum()) < TOL
    assert not got[[0, 5, 6]].any()


def test_preference_closed_forms():
    counts = np.ones((2, 1), bool)
    loss, reward, d = ot.preference(np.array([[-1.0], [-1.0]]), counts, None, 0.5, 0.1)
    assert np.isclose(loss, np.log(2)) and np.allclose(reward, -0.5) and np.allclose(d, [-0.2, 0.2])
    for x in (0.0, -3e38):
        logp, top, total = ot.logprobs(np.full((1, 8), x), np.array([3]))
        assert np.isclose(logp[0], -np.log(8)) and top[0] == x and total[0] == 8
