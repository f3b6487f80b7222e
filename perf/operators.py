"""Performance cases of the operators around the layer in a fine-tuning step.

Four operators, each through the calls a program makes of
``paper_2501_08582_amd.train``:

* ``norm``: residual + dropout(x) and the normalisation of the sum (layer norm,
  or by the root mean square), forward alone as in serving and with its
  gradients as in training;
* ``dropout``: dropout from a counter-based generator, its mask never stored,
  with and without the residual it is added to, and its gradient;
* ``embedding``: the scaled lookup, and the gradient of the table;
* ``preference``: log-probabilities of the target tokens out of the logits, the
  paired preference loss over sequences, and the gradient of the logits; the
  log-probabilities alone where a reference model scores a batch.

Widths and token counts are those of the projections and batches that the
benchmark and the tests use (4096, 5120, 14336; 4096 and 8192 tokens), with
generic and odd sizes between them.

The generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011): column c
of row n takes 16-bit half c % 8 of the block with counter (c / 8, n, offset low,
offset high) and the seed as key, and is kept where it is at least p * 65536.
"""
import functools
import math

import numpy as np
import torch

own = False

MASK32 = 0xFFFFFFFF
MOST = {"norm": 350e6, "dropout": 940e6, "embedding": 1.65e9, "preference": 2.2e9}  # bytes of the largest listed cases


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _norm(rows, cols, kind="layer", dtype="bf16", residual=True, p=0.0, bias=True, train=True, name=None):
    c = {"op": "norm", "rows": rows, "cols": cols, "kind": kind, "dtype": dtype, "residual": residual, "p": p,
         "bias": bias, "train": train}
    return {**c, "name": name} if name else c


def _dropout(rows, cols, p, dtype="bf16", residual=False, name=None):
    c = {"op": "dropout", "rows": rows, "cols": cols, "p": p, "dtype": dtype, "residual": residual}
    return {**c, "name": name} if name else c


def _embedding(tokens, vocab, cols, dtype="bf16", scale=1.0, padded=0.0, train=True, name=None):
    c = {"op": "embedding", "tokens": tokens, "vocab": vocab, "cols": cols, "dtype": dtype, "scale": scale,
         "padded": padded, "train": train}
    return {**c, "name": name} if name else c


def _preference(pairs, length, vocab, dtype="bf16", padded=0.2, smoothing=0.0, dead=0, train=True, name=None):
    c = {"op": "preference", "pairs": pairs, "length": length, "vocab": vocab, "dtype": dtype, "padded": padded,
         "smoothing": smoothing, "dead": dead, "train": train}
    return {**c, "name": name} if name else c


def listed():
    return [
        # four sequences decoding: the residual's sum and its norm before a projection, all latency
        _norm(4, 4096, kind="rms", bias=False, train=False, name="norm_decode_rms"),
        # a fine-tuning batch between two blocks of the 13B width, dropout on the branch
        _norm(4096, 5120, p=0.1, name="norm_train_layer"),
        # unpadded sequences (an odd token count) of an odd width in 32 bits, no dropout
        _norm(1733, 2047, kind="rms", dtype="f32", bias=False, name="norm_train_odd_f32"),
        # hidden activations of the widest projection of the benchmark's batch, and the gradient
        _dropout(8192, 14336, 0.05, name="dropout_hidden"),
        # a small odd branch added to its residual in 32 bits
        _dropout(777, 1003, 0.1, dtype="f32", residual=True, name="dropout_odd_f32"),
        # one token each of 32 decoding sequences
        _embedding(32, 32768, 4096, train=False, name="embed_decode"),
        # a fine-tuning batch and the gradient of the whole table
        _embedding(8192, 32768, 4096, name="embed_train"),
        # the same with the larger vocabulary and a scaled table
        _embedding(16384, 131072, 4096, scale=0.5, padded=0.1, name="embed_train_large"),
        # a short odd batch in 32 bits, a quarter of it padding
        _embedding(1501, 50021, 771, dtype="f32", padded=0.25, scale=27.77, name="embed_train_odd_f32"),
        # a reference model scores a few tokens over a large vocabulary
        _preference(1, 4, 131072, padded=0.0, train=False, name="score_few"),
        # two pairs of 257 tokens in 32 bits, an odd vocabulary whose last entries are masked
        _preference(2, 257, 50021, dtype="f32", smoothing=0.1, dead=37, name="prefer_odd_f32"),
        # a fine-tuning batch of four pairs
        _preference(4, 1024, 65536, name="prefer_train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fit(case, *extents):
    """The case with its first extents halved until it costs no more than the largest listed one."""
    return next(c for i in range(64) for c in [{**case, **{e: max(1, case[e] >> i) for e in extents}}]
                if work(c)["bytes"] <= MOST[case["op"]])


def draw(rng):
    op = rng.choice(["norm", "norm", "dropout", "embedding", "embedding", "preference", "preference"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        return _fit(_norm(_log(rng, 1, 8192), _log(rng, 64, 16384), kind=rng.choice(["layer", "rms"]), dtype=dtype,
                          residual=rng.random() < 0.7, p=rng.choice([0.0, 0.0, 0.05, 0.1, 0.5]),
                          bias=rng.random() < 0.5, train=rng.random() < 0.7), "rows")
    if op == "dropout":
        return _fit(_dropout(_log(rng, 16, 16384), _log(rng, 64, 16384), rng.choice([0.05, 0.1, 0.3, 0.5]), dtype=dtype,
                             residual=rng.random() < 0.5), "rows")
    if op == "embedding":
        return _fit(_embedding(_log(rng, 1, 32768), _log(rng, 256, 131072), _log(rng, 64, 8192), dtype=dtype,
                               scale=rng.choice([1.0, 1.0, 0.5, 64.0]), padded=rng.choice([0.0, 0.0, 0.1, 0.5]),
                               train=rng.random() < 0.75), "tokens", "vocab")
    return _fit(_preference(_log(rng, 1, 16), _log(rng, 1, 2048), _log(rng, 1000, 131072), dtype=dtype,
                            padded=rng.choice([0.0, 0.2, 0.5]), smoothing=rng.choice([0.0, 0.0, 0.1]),
                            dead=rng.choice([0, 0, 128]), train=rng.random() < 0.75), "length", "pairs")


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
BETA = 0.1


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ids(n, vocab, padded, g):
    """Tokens by rank as in text (the k-th most frequent about 1/k as often), spread over the ids; -1 where padded."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp_(0, vocab - 1)
    ids = (rank * 40503 + 17) % vocab
    return torch.where(torch.rand(n, generator=g, device="cuda") < padded, torch.full_like(ids, -1), ids)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dt(case)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dt)

    st = {"case": case}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        scale = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))  # channels of unequal size, off zero
        mean = 0.2 * torch.randn(cols, generator=g, device="cuda")
        st["x"] = (torch.randn(rows, cols, generator=g, device="cuda") * scale + mean).to(dt)
        st["residual"] = (2.0 * torch.randn(rows, cols, generator=g, device="cuda") * scale).to(dt) if case["residual"] else None
        st["weight"] = (1.0 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(dt)
        st["bias"] = normal(cols, std=0.1) if case["bias"] else None
        if case["train"]:
            st["dy"] = normal(rows, cols, std=1e-2)
            st["dz"] = normal(rows, cols, std=1e-2) if case["residual"] else None
        st["seed"], st["offset"] = 0x9E3779B97F4A7C15 ^ seed, 3 + seed
    elif case["op"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        st["x"] = normal(rows, cols)
        st["residual"] = normal(rows, cols, std=2.0) if case["residual"] else None
        st["dy"] = normal(rows, cols, std=1e-2)
        st["seed"], st["offset"] = 0xD1B54A32D192ED03 ^ seed, 5 + seed
    elif case["op"] == "embedding":
        st["ids"] = _ids(case["tokens"], case["vocab"], case["padded"], g)
        st["table"] = normal(case["vocab"], case["cols"], std=0.02)
        if case["train"]:
            st["dy"] = normal(case["tokens"], case["cols"], std=1e-2)
    else:
        B, S, V = 2 * case["pairs"], case["length"], case["vocab"]
        logits = torch.randn(B, S, V, generator=g, device="cuda", dtype=dt) * 2.0
        targets = _ids(B * S, V - case["dead"], 0.0, g).view(B, S)
        # a trained model gives its targets a better chance than the rest
        up = 6.0 * torch.rand(B, S, 1, generator=g, device="cuda")
        logits.scatter_add_(2, targets.unsqueeze(2), up.to(dt))
        if case["dead"]:
            logits[:, :, V - case["dead"]:] = -math.inf
        # prompts in front and padding behind do not count
        end = (S * (1.0 - case["padded"] * torch.rand(B, 1, generator=g, device="cuda"))).ceil()
        at = torch.arange(S, device="cuda").unsqueeze(0)
        st["targets"] = torch.where((at < end) & (at >= int(0.25 * case["padded"] * S)), targets, torch.full_like(targets, -100))
        st["logits"] = logits
        # the reference's log-probabilities of the same tokens, where this model has moved away from it
        at = targets.unsqueeze(2)
        ref = torch.stack([(x.float().gather(1, t) - torch.logsumexp(x.float(), 1, keepdim=True)).squeeze(1)
                           for x, t in zip(logits, at)])
        st["ref"] = ref + torch.randn(B, S, generator=g, device="cuda")
    return st


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _round(k, state):
    c0, c1, c2, c3, k0, k1 = state
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products: their bits are right, whatever the sign
    return ((p1 >> 32) & MASK32 ^ c1 ^ k0, p1 & MASK32, (p0 >> 32) & MASK32 ^ c3 ^ k1, p0 & MASK32,
            k0 + 0x9E3779B9 & MASK32, k1 + 0xBB67AE85 & MASK32)


def _keep(rows, cols, p, seed, offset):
    """The kept elements, and the factor that keeps the expectation."""
    c0 = torch.arange((cols + 7) // 8, device="cuda").unsqueeze(0).expand(rows, -1)
    c1 = torch.arange(rows, device="cuda").unsqueeze(1).expand_as(c0)
    start = (c0, c1, torch.full_like(c0, offset & MASK32), torch.full_like(c0, offset >> 32 & MASK32),
             seed & MASK32, seed >> 32 & MASK32)
    words = torch.stack(functools.reduce(lambda s, k: _round(k, s), range(10), start)[:4], dim=2)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=3).reshape(rows, -1)[:, :cols]
    drop = int(math.floor(p * 65536.0 + 0.5))
    return halves >= drop, 65536.0 / (65536.0 - drop)


def _drop(x, keep, factor):
    return torch.where(keep, x * factor, torch.zeros((), device="cuda"))


def _plain_norm(st):
    case, dt = st["case"], _dt(st["case"])
    rows, cols, rms = case["rows"], case["cols"], case["kind"] == "rms"
    keep, factor = _keep(rows, cols, case["p"], st["seed"], st["offset"]) if case["p"] else (None, 1.0)
    branch = _drop(st["x"].float(), keep, factor) if case["p"] else st["x"].float()
    z = (branch + st["residual"].float() if case["residual"] else branch).to(dt)  # the sum is stored, and normalised as stored
    zf, w = z.float(), st["weight"].float()
    mean = 0.0 if rms else zf.mean(1, keepdim=True)
    rstd = torch.rsqrt((zf - mean).square().mean(1, keepdim=True) + 1e-5)
    xhat = (zf - mean) * rstd
    y = xhat * w + st["bias"].float() if case["bias"] else xhat * w
    out = {"y": y.to(dt)}
    if case["residual"] or case["p"]:
        out["z"] = z
    if case["train"]:
        dy = st["dy"].float()
        gx = dy * w
        d = gx - xhat * (gx * xhat).mean(1, keepdim=True)
        d = rstd * (d if rms else d - gx.mean(1, keepdim=True))
        d = d + st["dz"].float() if case["residual"] else d
        out["dx"] = (_drop(d, keep, factor) if case["p"] else d).to(dt)
        if case["residual"]:
            out["dresidual"] = d.to(dt)
        out["dweight"] = (dy * xhat).sum(0).to(dt)
        if case["bias"]:
            out["dbias"] = dy.sum(0).to(dt)
    return out


def _plain_dropout(st):
    case, dt = st["case"], _dt(st["case"])
    keep, factor = _keep(case["rows"], case["cols"], case["p"], st["seed"], st["offset"])
    y = _drop(st["x"].float(), keep, factor)
    y = y + st["residual"].float() if case["residual"] else y
    return {"y": y.to(dt), "dx": _drop(st["dy"].float(), keep, factor).to(dt)}


def _plain_embedding(st):
    case, dt = st["case"], _dt(st["case"])
    known = ((st["ids"] >= 0) & (st["ids"] < case["vocab"])).unsqueeze(1)
    at = st["ids"].clamp(0, case["vocab"] - 1)
    zero = torch.zeros((), device="cuda")
    out = {"y": torch.where(known, st["table"][at].float() * case["scale"], zero).to(dt)}
    if case["train"]:
        total = torch.zeros(case["vocab"], case["cols"], device="cuda")
        out["dtable"] = total.index_add_(0, at, torch.where(known, st["dy"].float() * case["scale"], zero)).to(dt)
    return out


def _log_sigmoid(x):
    return x.clamp(max=0.0) - torch.log1p(torch.exp(-x.abs()))


def _plain_preference(st):
    case, P = st["case"], st["case"]["pairs"]
    z = st["logits"].float()
    counts = st["targets"] >= 0
    at = st["targets"].clamp(min=0).unsqueeze(2)
    top = z.amax(2, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(2, keepdim=True)
    zero = torch.zeros((), device="cuda")
    logp = torch.where(counts, (z.gather(2, at) - top - torch.log(total)).squeeze(2), zero)
    if not case["train"]:
        return {"logp": logp}
    reward = BETA * torch.where(counts, logp - st["ref"], zero).sum(1)
    margin, eps = reward[:P] - reward[P:], case["smoothing"]
    loss = -((1.0 - eps) * _log_sigmoid(margin) + eps * _log_sigmoid(-margin)).mean()
    up = (eps * torch.exp(_log_sigmoid(margin)) - (1.0 - eps) * torch.exp(_log_sigmoid(-margin))) * (BETA / P)
    dlogp = torch.where(counts, torch.cat([up, -up]).unsqueeze(1), zero).unsqueeze(2)
    dlogits = e * (-dlogp / total)
    dlogits.scatter_add_(2, at, dlogp)
    return {"logp": logp, "loss": loss, "reward": reward, "dlogits": torch.where(counts.unsqueeze(2), dlogits, zero).to(_dt(case))}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2501_08582_amd import train

    case = st["case"]
    if case["op"] == "norm":
        rng = {"p": case["p"], "seed": st["seed"], "offset": st["offset"]}
        y, z, mean, rstd = train.norm_forward(st["x"], st["weight"], st["bias"], 1e-5, case["kind"], residual=st["residual"],
                                              need_stats=case["train"], **rng)
        out = {"y": y}
        if case["residual"] or case["p"]:
            out["z"] = z
        if case["train"]:
            dx, dres, dweight, dbias = train.norm_backward(st["dy"], z, st["weight"], mean, rstd, case["kind"], dZ=st["dz"],
                                                           need_dresidual=case["residual"], need_dbias=case["bias"], **rng)
            out["dx"] = dx
            if case["residual"]:
                out["dresidual"] = dres
            out["dweight"] = dweight
            if case["bias"]:
                out["dbias"] = dbias
        return out
    if case["op"] == "dropout":
        return {"y": train.dropout(st["x"], case["p"], st["seed"], st["offset"], residual=st["residual"]),
                "dx": train.dropout(st["dy"], case["p"], st["seed"], st["offset"])}
    if case["op"] == "embedding":
        out = {"y": train.embedding_forward(st["ids"], st["table"], case["scale"])}
        if case["train"]:
            out["dtable"] = train.embedding_backward(st["dy"], st["ids"], case["vocab"], case["scale"])
        return out
    if not case["train"]:
        return {"logp": train.logprob_forward(st["logits"], st["targets"])[0]}
    loss, reward, logp, dlogits = train.preference_step(st["logits"], st["targets"], st["ref"], BETA, case["smoothing"])
    return {"logp": logp, "loss": loss, "reward": reward, "dlogits": dlogits}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "dropout": _plain_dropout, "embedding": _plain_embedding,
            "preference": _plain_preference}[state["case"]["op"]](state)


def work(case):
    """Each input read once and each output written once; a few operations an element."""
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        arrays = 2 + 2 * case["residual"] + (case["p"] > 0 and not case["residual"])  # x, y; residual, z
        params = 1 + case["bias"]
        if case["train"]:
            arrays += 2 + 2 * case["residual"]  # dy, dx; dz, dresidual
            params *= 2
        return {"bytes": es * (n * arrays + case["cols"] * params), "flops": n * (8 + 14 * case["train"])}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": es * n * (4 + case["residual"]), "flops": 4 * n}
    if case["op"] == "embedding":
        n = case["tokens"] * case["cols"]
        distinct = min(case["vocab"], case["tokens"]) * case["cols"]
        b = 8 * case["tokens"] + es * (distinct + n)
        if case["train"]:
            b += es * (n + case["vocab"] * case["cols"])
        return {"bytes": b, "flops": n * (1 + case["train"])}
    n = 2 * case["pairs"] * case["length"]
    return {"bytes": n * (16 + es * case["vocab"] * (1 + case["train"])), "flops": n * case["vocab"] * (4 + 3 * case["train"])}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_factor(case, st):
    """Dropout's factor of every element (0 where dropped), by Philox4x32-10 on the host."""
    rows, cols, key = case["rows"], case["cols"], st["seed"]
    blocks = (cols + 7) // 8
    u = np.uint64
    low, half = u(MASK32), u(32)

    def step(c, k):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        k0, k1 = u(((key & MASK32) + k * 0x9E3779B9) & MASK32), u(((key >> 32) + k * 0xBB67AE85) & MASK32)
        return [(b >> half) ^ c[1] ^ k0, b & low, (a >> half) ^ c[3] ^ k1, a & low]

    c = functools.reduce(step, range(10), [
        np.tile(np.arange(blocks, dtype=u), rows), np.repeat(np.arange(rows, dtype=u), blocks),
        np.full(rows * blocks, st["offset"] & MASK32, dtype=u), np.full(rows * blocks, st["offset"] >> 32 & MASK32, dtype=u)])
    bits = np.stack([(c[i // 2] >> u(16 * (i % 2))).astype(np.uint16) for i in range(8)], axis=1)
    drop = math.floor(case["p"] * 65536 + 0.5)
    kept = torch.from_numpy((bits >= drop).reshape(rows, -1)[:, :cols].copy()).cuda()
    return kept.double() / (1.0 - drop / 65536.0)


def _exact_norm(case, st):
    z = st["x"].double()
    f = None
    if case["p"]:
        f = _exact_factor(case, st)
        z = z * f
    if case["residual"]:
        z = z + st["residual"].double()
    z = z.to(_dt(case)).double()
    n, w = case["cols"], st["weight"].double()
    mu = z.sum(1, keepdim=True) / n if case["kind"] == "layer" else torch.zeros(case["rows"], 1, dtype=torch.float64, device="cuda")
    sigma = (((z - mu) ** 2).sum(1, keepdim=True) / n + 1e-5).sqrt()
    h = (z - mu) / sigma
    out = {"y": h * w + (st["bias"].double() if case["bias"] else 0.0)}
    if case["residual"] or case["p"]:
        out["z"] = z
    if case["train"]:
        dy = st["dy"].double()
        dh = dy * w
        # z enters through its own place, through sigma and (layer norm) through mu
        dz = dh / sigma - h * (dh * h).sum(1, keepdim=True) / (n * sigma)
        if case["kind"] == "layer":
            dz = dz - dh.sum(1, keepdim=True) / (n * sigma)
        if case["residual"]:
            dz = dz + st["dz"].double()
        out["dx"] = dz * f if f is not None else dz
        if case["residual"]:
            out["dresidual"] = dz
        out["dweight"] = (dy * h).sum(0)
        if case["bias"]:
            out["dbias"] = dy.sum(0)
    return out


def _exact_embedding(case, st):
    V = case["vocab"]
    ok = (st["ids"] > -1) & (st["ids"] < V)
    y = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
    y[ok] = st["table"][st["ids"][ok]].double() * case["scale"]
    out = {"y": y}
    if case["train"]:
        d = torch.zeros(V, case["cols"], dtype=torch.float64, device="cuda")
        out["dtable"] = d.index_put_((st["ids"][ok],), case["scale"] * st["dy"][ok].double(), accumulate=True)
    return out


def _exact_preference(case, st):
    P, ok = case["pairs"], st["targets"] != -100
    token = torch.where(ok, st["targets"], torch.zeros_like(st["targets"])).unsqueeze(2)
    logp = torch.stack([torch.log_softmax(x.double(), 1).gather(1, t).squeeze(1) for x, t in zip(st["logits"], token)]) * ok
    if not case["train"]:
        return {"logp": logp}
    reward = BETA * (logp - st["ref"].double() * ok).sum(1)
    margin, eps = reward[:P] - reward[P:], case["smoothing"]
    win = 1.0 / (1.0 + torch.exp(-margin))
    loss = (torch.log1p(torch.exp(-margin)) + eps * margin).mean()
    slope = (win - 1.0 + eps) * BETA / P
    up = torch.cat([slope, -slope]).unsqueeze(1) * ok

    def one(x, t, c):  # a sequence at a time, for the memory
        hit = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        hit.scatter_(1, t, 1.0)
        return c.unsqueeze(1) * (hit - torch.softmax(x.double(), 1))

    d = torch.stack([one(*a) for a in zip(st["logits"], token, up)])
    return {"logp": logp, "loss": loss, "reward": reward, "dlogits": d}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, st)
    if case["op"] == "dropout":
        f = _exact_factor(case, st)
        y = st["x"].double() * f
        return {"y": y + st["residual"].double() if case["residual"] else y, "dx": st["dy"].double() * f}
    return (_exact_embedding if case["op"] == "embedding" else _exact_preference)(case, st)
