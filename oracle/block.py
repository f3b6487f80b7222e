"""fp64 numpy definitions of the gated block, the orthogonalised update and
sampling -- TEST INFRASTRUCTURE ONLY.

Parity status: pinned by the CPU tests (finite differences, a full singular value
decomposition, enumeration of small distributions)."""
import numpy as np

from oracle import bf16 as obf16
from oracle import lors as olors


# ---------------------------------------------------------------------------
# gated block
# ---------------------------------------------------------------------------
def act(g, kind):
    """(act(g), its derivative)."""
    if kind == "silu":
        with np.errstate(over="ignore"):
            y = 1.0 / (1.0 + np.exp(-g))
        return g * y, y * (1.0 + g * (1.0 - y))
    k = np.sqrt(2.0 / np.pi)
    t = np.tanh(k * (g + 0.044715 * g**3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)


def weight(q, s, dtype):
    """W' of a projection q = (W, mask, B, A) in the dtype of its weight."""
    W = olors.merged_weight(*q, s)
    return obf16.to_f64(obf16.from_f64_rne(W)) if dtype == "bf16" else W


def gated_forward(X, gate, up, s, kind, dtype):
    """(H, G, U)."""
    G, U = X @ weight(gate, s, dtype).T, X @ weight(up, s, dtype).T
    return act(G, kind)[0] * U, G, U


def gated_backward(dH, X, gate, up, G, U, s, kind, dtype):
    """(dX, (dB, dA) of the gate, (dB, dA) of the up projection), from G and U as stored."""
    y, d = act(G, kind)
    dG, dU = dH * U * d, dH * y
    dX = dG @ weight(gate, s, dtype) + dU @ weight(up, s, dtype)

    def adapters(q, D):
        _, dB, dA, _ = olors.backward(D, X, *q, s)
        return dB, dA

    return dX, adapters(gate, dG), adapters(up, dU)


# ---------------------------------------------------------------------------
# orthogonalised update
# ---------------------------------------------------------------------------
def direction(v, steps, a, b, c, eps):
    """The Newton-Schulz iterates themselves, on the shorter side."""
    x = v if v.shape[0] <= v.shape[1] else v.T
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        S = x @ x.T
        x = a * x + (b * S + c * (S @ S)) @ x
    return x if v.shape[0] <= v.shape[1] else x.T


def update(grad, m, master, momentum, nesterov, rate, decay, steps, a, b, c, eps):
    """(m, master) after the step."""
    m = momentum * m + (1.0 - momentum) * grad
    v = momentum * m + (1.0 - momentum) * grad if nesterov else m
    return m, (1.0 - decay) * master - rate * direction(v, steps, a, b, c, eps)


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def kept(z, temperature, top_k, top_p, min_p):
    """Weights of one row's entries by index, 0 where not kept."""
    z = np.asarray(z, dtype=np.float64)
    order = np.argsort(-z, kind="stable")
    w = np.zeros(len(z))
    if not temperature > 0:
        w[order[0]] = 1.0
        return w
    r = np.exp((z[order] - z[order[0]]) / temperature)
    if top_k > 0:
        r[int(top_k):] = 0.0
    n = len(r)
    if top_p < 1.0:
        run = np.cumsum(r)
        n = 1 + int((run[:-1] < top_p * run[-1]).sum())
    if min_p > 0.0:
        n = min(n, max(1, int((r >= min_p).sum())))
    w[order[:n]] = r[:n]
    return w


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its probability) of one row; (-1, NaN) without a distribution."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all():
        return -1, float("nan")
    w = kept(z, temperature, top_k, top_p, min_p)
    run = np.cumsum(w)
    at = np.flatnonzero((run > float(u) * run[-1]) & (w > 0))
    t = int(at[0]) if at.size else int(np.flatnonzero(w)[-1])
    return t, float(np.log(w[t] / run[-1]))
