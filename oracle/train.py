"""fp64 numpy definitions of the operators around the layer -- TEST
INFRASTRUCTURE ONLY: dropout, norms, embedding, preference loss, each with its
gradient written out.

Parity status: pinned by the CPU tests (known answers of the generator, finite
differences of every gradient, closed forms)."""
import numpy as np

M32 = 0xFFFFFFFF


# ---------------------------------------------------------------------------
# Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011) and the dropout mask
# ---------------------------------------------------------------------------
def philox_block(counter, key):
    """One block in plain integers: four 32-bit words from four and a key of two."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def random16(rows, cols, seed, offset, first=0):
    """The 16 random bits of every element of rows first .. first + rows - 1."""
    blocks = -(-cols // 8)
    c0 = np.broadcast_to(np.arange(blocks, dtype=np.uint64), (rows, blocks))
    c1 = np.broadcast_to(np.arange(first, first + rows, dtype=np.uint64)[:, None], (rows, blocks))
    c = [c0, c1, np.full((rows, blocks), offset & M32, np.uint64), np.full((rows, blocks), offset >> 32 & M32, np.uint64)]
    k0, k1 = seed & M32, seed >> 32 & M32
    lo, sh = np.uint64(M32), np.uint64(32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> sh) ^ c[1] ^ np.uint64(k0), b & lo, (a >> sh) ^ c[3] ^ np.uint64(k1), a & lo]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    out = np.empty((rows, blocks, 8), np.uint16)
    for i in range(8):
        out[:, :, i] = (c[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF)
    return out.reshape(rows, -1)[:, :cols]


def threshold(p):
    return int(np.floor(p * 65536 + 0.5))


def dropout(x, p, seed, offset, residual=None):
    """(result, kept).  Dropping is a select."""
    rows, cols = x.shape
    t = threshold(p)
    kept = random16(rows, cols, seed, offset) >= t
    y = np.where(kept, x * (65536.0 / (65536 - t)), 0.0)
    return (y if residual is None else y + residual), kept


# ---------------------------------------------------------------------------
# norms over the last dimension of z
# ---------------------------------------------------------------------------
def stats(z, eps, rms):
    mean = np.zeros((z.shape[0], 1)) if rms else z.mean(1, keepdims=True)
    return mean, 1.0 / np.sqrt(((z - mean) ** 2).mean(1, keepdims=True) + eps)


def norm(z, weight, bias, eps, rms):
    mean, rstd = stats(z, eps, rms)
    y = (z - mean) * rstd
    if weight is not None:
        y = y * weight
    return y if bias is None else y + bias


def norm_backward(dy, z, weight, eps, rms, dz=None):
    """(gradient of z, of weight, of bias)."""
    mean, rstd = stats(z, eps, rms)
    h = (z - mean) * rstd
    g = dy if weight is None else dy * weight
    d = g - h * (g * h).mean(1, keepdims=True)
    if not rms:
        d = d - g.mean(1, keepdims=True)
    d = rstd * d
    return (d if dz is None else d + dz), (dy * h).sum(0), dy.sum(0)


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def embedding(ids, table, scale):
    ok = (ids >= 0) & (ids < table.shape[0])
    return np.where(ok[:, None], scale * table[np.where(ok, ids, 0)], 0.0)


def embedding_backward(dy, ids, vocab, scale):
    out = np.zeros((vocab, dy.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < vocab:
            out[v] += scale * dy[t]
    return out


# ---------------------------------------------------------------------------
# preference loss
# ---------------------------------------------------------------------------
def logprobs(logits, targets):
    """(logp, top, sum) of rows x vocab logits: the largest entry and the sum of exponentials
    below it; 0 where the target does not count."""
    n, V = logits.shape
    logp, tops, sums = np.zeros(n), np.zeros(n), np.zeros(n)
    for i in range(n):
        if 0 <= targets[i] < V:
            with np.errstate(invalid="ignore"):
                tops[i] = logits[i].max()
                sums[i] = np.exp(logits[i] - tops[i]).sum()
                logp[i] = (logits[i, targets[i]] - tops[i]) - np.log(sums[i])
    return logp, tops, sums


def logprobs_backward(dlogp, logits, targets):
    _, tops, sums = logprobs(logits, targets)
    out = np.zeros_like(logits)
    for i in range(logits.shape[0]):
        if 0 <= targets[i] < logits.shape[1]:
            out[i] = -dlogp[i] * np.exp(logits[i] - tops[i]) / sums[i]
            out[i, targets[i]] += dlogp[i]
    return out


def _log_sigmoid(x):
    return np.minimum(x, 0.0) - np.log1p(np.exp(-np.abs(x)))


def preference(logp, counts, ref, beta, smoothing):
    """(loss, reward, gradient by each sequence's sum) of 2 P x length log-probabilities."""
    P = logp.shape[0] // 2
    reward = beta * np.where(counts, logp - (0.0 if ref is None else ref), 0.0).sum(1)
    m = reward[:P] - reward[P:]
    loss = np.mean(-(1 - smoothing) * _log_sigmoid(m) - smoothing * _log_sigmoid(-m))
    slope = beta / P * (smoothing / (1 + np.exp(-m)) - (1 - smoothing) / (1 + np.exp(m)))
    return loss, reward, np.concatenate([slope, -slope])
