"""Performance cases of three operators that a fine-tuning loop of sparse gated models needs.

* ``gated``: the gated half of a feed-forward block out of two sparsity-preserved LoRA projections,
  H = act(X.Wg'^T) * (X.Wu'^T) with W' = select(M, W + s.B.A, 0) in the weights' type (SiLU, or GELU by
  tanh), for serving (H alone) and for training (H and the two projections' results, which the
  backward reads), and its backward: the gradients of X and of both projections' adapters;
* ``ortho``: an update matrix orthogonalised by Newton-Schulz products, X <- a X + (b S + c S^2) X with
  S = X.X^T on the shorter side, alone and as a step of an optimiser over many adapters: momentum
  (Nesterov's form), orthogonalised direction, weight decay, fp32 masters and the parameters' copies;
* ``sample``: tokens drawn from logits with temperature, top-k, top-p and min-p, one given random number
  a row. Entries are ordered by logit, equal ones by index; top-k keeps the first k of that order,
  top-p the shortest run of those that holds p of their probability, min-p those of at least
  min-p times the largest probability. The token is the first kept one, by index, at which the kept
  entries' running sum of probabilities exceeds u times their whole.

Widths, ranks and token counts are those of the benchmark's projections (4096, 5120, 11008, 13824, 14336;
ranks 16 and 64; 4096 tokens) with generic and odd sizes between them.
"""
import functools
import math

import torch

own = False

SCALE = 2.0
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
BETA, LR, DECAY, EPS = 0.95, 0.02, 0.01, 1e-7


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _gated(L, R, C, r, mask="bitmap", dtype="bf16", act="silu", run="serve", scale=SCALE, name=None):
    c = {"op": "gated", "L": L, "R": R, "C": C, "r": r, "mask": mask, "dtype": dtype, "act": act, "run": run, "scale": scale}
    return {**c, "name": name} if name else c


def _ortho(shapes, dtype="bf16", run="step", name=None):
    """shapes: "rows x cols x count" of the matrices, joined by spaces."""
    c = {"op": "ortho", "shapes": shapes, "dtype": dtype, "run": run}
    return {**c, "name": name} if name else c


def _sample(rows, vocab, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, dead=0, name=None):
    """mixed: every row has parameters of its own, as the requests of a batch do."""
    c = {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
         "min_p": min_p, "mixed": mixed, "dead": dead}
    return {**c, "name": name} if name else c


def _adapters(projections, rank, count):
    """The A (rank x in) and B (out x rank) of `count` blocks of projections (out, in, how many)."""
    return " ".join(f"{rank}x{i}x{n * count} {o}x{rank}x{n * count}" for o, i, n in projections)


def listed():
    small = [(4096, 4096, 4), (11008, 4096, 2), (4096, 11008, 1)]
    large = [(5120, 5120, 4), (13824, 5120, 2), (5120, 13824, 1)]
    return [
        # four sequences decoding: one read of both sparse weights
        _gated(4, 11008, 4096, 16, name="gated_decode"),
        # an odd count of prompt tokens of a small model, ranks that fill no matrix instruction
        _gated(777, 2744, 1032, 24, act="gelu", scale=1.5, run="forward", name="gated_prompt_odd"),
        # the forward of a fine-tuning batch, 2:4 weights
        _gated(4096, 11008, 4096, 16, mask="2:4", run="forward", name="gated_train_forward"),
        # the backward of a fine-tuning batch of the larger width and rank
        _gated(4096, 13824, 5120, 64, run="backward", name="gated_train_backward"),
        # a small odd backward in 32 bits, as a debugging run makes it
        _gated(131, 268, 196, 8, dtype="f32", run="backward", name="gated_backward_odd_f32"),
        # one adapter's update direction
        _ortho("64x14336x1", run="direction", name="ortho_one"),
        # an odd one in 32 bits, taller than wide
        _ortho("5003x37x1", dtype="f32", run="direction", name="ortho_odd_f32"),
        # the optimiser's step over the adapters of eight blocks of the 7B widths
        _ortho(_adapters(small, 16, 8), name="ortho_step_rank16"),
        # the same of the 13B widths at rank 64
        _ortho(_adapters(large, 64, 8), name="ortho_step_rank64"),
        # one sequence decoding over a large vocabulary
        _sample(1, 131072, temperature=0.8, top_k=50, top_p=0.9, name="sample_one"),
        # an odd batch in 32 bits whose last entries are masked, each request with parameters of its own
        _sample(37, 50021, dtype="f32", mixed=True, dead=37, name="sample_mixed_odd_f32"),
        # the rollouts of a preference batch: the whole distribution's upper part
        _sample(256, 131072, temperature=1.0, top_p=0.95, min_p=0.001, name="sample_rollouts"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "ortho", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "gated":
        f32 = dtype == "f32"
        step, most = (4, 1024) if f32 else (8, 8192)
        mask = rng.choice(["bitmap", "2:4"])
        return _gated(_log(rng, 1, 512 if f32 else 4096), step * _log(rng, 8, most // step), step * _log(rng, 8, most // step),
                      rng.choice([4, 8, 16, 16, 32, 64, 64, 100, 128]), mask=mask, dtype=dtype, act=rng.choice(["silu", "silu", "gelu"]),
                      run=rng.choice(["serve", "forward", "backward"]), scale=rng.choice([2.0, 2.0, 0.5, 1.7]))
    if op == "ortho":
        rank = rng.choice([4, 8, 16, 16, 24, 32, 64, 64, 100, 128])
        kinds = [(rank, _log(rng, 32, 14336), _log(rng, 1, 8)) for _ in range(rng.randint(1, 4))]
        return _ortho(" ".join(f"{r}x{n}x{c}" if rng.random() < 0.5 else f"{n}x{r}x{c}" for r, n, c in kinds), dtype=dtype,
                      run=rng.choice(["step", "step", "direction"]))
    if rng.random() < 0.25:
        return _sample(_log(rng, 1, 256), _log(rng, 1000, 131072), dtype=dtype, mixed=True, dead=rng.choice([0, 128]))
    return _sample(_log(rng, 1, 256), _log(rng, 1000, 131072), dtype=dtype, temperature=rng.choice([1.0, 0.7, 1.3, 0.0]),
                   top_k=rng.choice([0, 0, 1, 20, 200]), top_p=rng.choice([1.0, 0.95, 0.9, 0.5]), min_p=rng.choice([0.0, 0.0, 0.05]),
                   dead=rng.choice([0, 0, 128]))


def _kinds(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split()]


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _mask(W, mask):
    """The pruner's choice: the larger half of each row, or the two largest of every four."""
    R, C = W.shape
    if mask == "2:4":
        top = W.abs().view(R, C // 4, 4).topk(2, dim=2).indices
        return torch.zeros(R, C // 4, 4, dtype=torch.bool, device="cuda").scatter_(2, top, True).view(R, C)
    return W.abs() >= W.abs().median(dim=1, keepdim=True).values


def _packed(keep, mask):
    """The frozen mask as the layer keeps it: a bit for each entry, or for each four the places p0 | p1 << 2 of the two kept."""
    R, C = keep.shape
    if mask == "2:4":
        at = keep.view(R, C // 4, 4).to(torch.int64)
        place = torch.arange(4, device="cuda")
        first = torch.where(at > 0, place, torch.full_like(place, 9)).amin(2)
        last = torch.where(at > 0, place, torch.full_like(place, -1)).amax(2)
        fields, wide = first | last << 2, 4
    else:
        fields, wide = keep.to(torch.int64), 1
    each = 32 // wide
    fields = torch.nn.functional.pad(fields, (0, -fields.shape[1] % each)).view(R, -1, each)
    words = (fields << wide * torch.arange(each, device="cuda")).sum(2)
    return torch.where(words >= 2**31, words - 2**32, words).to(torch.int32).contiguous()


def _projection(case, normal):
    R, C, r, dt = case["R"], case["C"], case["r"], _dt(case)
    W = normal(R, C, std=C**-0.5)
    keep = _mask(W, case["mask"])
    W = torch.where(keep, W, torch.zeros_like(W)).to(dt)
    return {"W": W, "keep": keep, "M": _packed(keep, case["mask"]), "B": normal(R, r, std=0.02).to(dt), "A": normal(r, C, std=r**-0.5).to(dt)}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dt(case)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std

    st = {"case": case}
    if case["op"] == "gated":
        st["gate"], st["up"] = _projection(case, normal), _projection(case, normal)
        size = torch.exp(0.5 * normal(case["C"]))  # channels of unequal size
        st["X"] = (normal(case["L"], case["C"]) * size).to(dt)
        if case["run"] == "backward":
            p = st["X"].float()
            st["G"], st["U"] = ((p @ q["W"].float().T).to(dt) for q in (st["gate"], st["up"]))
            st["dH"] = normal(case["L"], case["R"], std=1e-2).to(dt)
    elif case["op"] == "ortho":
        # all matrices of a kind of state lie in one buffer, one behind another, as an optimiser keeps them
        shapes = [(r, c) for r, c, n in _kinds(case) for _ in range(n)]
        sizes = [r * c for r, c in shapes]

        def low_rank(r, c):  # gradients: a few strong directions over weak noise
            k = max(1, min(r, c) // 4)
            return normal(r, k) @ (normal(k, c) * torch.exp(-0.5 * torch.arange(k, device="cuda", dtype=torch.float32))[:, None]) + 0.05 * normal(r, c)

        def split(flat):
            return [t.view(s) for t, s in zip(flat.split(sizes), shapes)]

        scale = 1e-3 * torch.exp(normal(len(shapes))).cpu()
        st["grad"] = torch.cat([(low_rank(*s) * float(x)).reshape(-1) for s, x in zip(shapes, scale)]).to(dt)
        st["grads"] = split(st["grad"])
        if case["run"] == "step":
            st["momentum"] = torch.cat([(low_rank(*s) * float(x)).reshape(-1) for s, x in zip(shapes, scale)])
            st["master"] = 0.05 * normal(sum(sizes))
            st["param"] = st["master"].to(dt)
            st["momenta"], st["masters"], st["params"] = (split(st[k]) for k in ("momentum", "master", "param"))
    else:
        rows, V = case["rows"], case["vocab"]
        logits = 2.5 * normal(rows, V)
        # a trained model: a head of likely tokens that falls off by rank
        likely = torch.randint(0, V, (rows, 64), generator=g, device="cuda")
        logits.scatter_add_(1, likely, 14.0 - 1.5 * torch.log(1.0 + torch.arange(64, device="cuda", dtype=torch.float32)).expand(rows, -1)
                            + normal(rows, 64))
        logits = logits.to(dt)
        if case["dead"]:
            logits[:, V - case["dead"]:] = -math.inf
        st["logits"] = logits
        st["u"] = torch.rand(rows, generator=g, device="cuda")
        if case["mixed"]:
            def pick(values, dtype):
                return torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(0, len(values), (rows,), generator=g, device="cuda")]

            st["temperature"] = pick([0.0, 0.6, 0.8, 1.0, 1.2], torch.float32)
            st["top_k"] = pick([0, 0, 1, 40, 1000], torch.int32)
            st["top_p"] = pick([1.0, 0.95, 0.9, 0.5], torch.float32)
            st["min_p"] = pick([0.0, 0.0, 0.02, 0.1], torch.float32)
        else:
            st.update({k: case[k] for k in ("temperature", "top_k", "top_p", "min_p")})
    return st


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _merged(p, s):
    """The merged sparse weight in the weights' own type, as the layer defines it."""
    W = p["W"].float() + s * (p["B"].float() @ p["A"].float())
    return torch.where(p["keep"], W, torch.zeros((), device="cuda")).to(p["W"].dtype).float()


def _gelu_parts(g):
    k = math.sqrt(2.0 / math.pi)
    e = torch.exp(-2.0 * (k * (g + 0.044715 * g * g * g)).abs())
    t = torch.sign(g) * (1.0 - e) / (1.0 + e)  # tanh
    return t, k * (1.0 + 0.134145 * g * g)


def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + _gelu_parts(g)[0])


def _act_slope(g, act):
    if act == "silu":
        y = 1.0 / (1.0 + torch.exp(-g))
        return y * (1.0 + g * (1.0 - y))
    t, inner = _gelu_parts(g)
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * inner


def _plain_gated(st):
    case, dt, s = st["case"], _dt(st["case"]), st["case"]["scale"]
    X = st["X"].float()
    Wg, Wu = _merged(st["gate"], s), _merged(st["up"], s)
    if case["run"] != "backward":
        G, U = X @ Wg.T, X @ Wu.T
        H = (_act(G, case["act"]) * U).to(dt)
        return {"H": H} if case["run"] == "serve" else {"H": H, "G": G.to(dt), "U": U.to(dt)}
    G, U, dH = st["G"].float(), st["U"].float(), st["dH"].float()
    dG, dU = dH * U * _act_slope(G, case["act"]), dH * _act(G, case["act"])

    def adapters(p, d):
        D = torch.where(p["keep"], d.T @ X, torch.zeros((), device="cuda"))
        return (s * (D @ p["A"].float().T)).to(dt), (s * (p["B"].float().T @ D)).to(dt)

    (dBg, dAg), (dBu, dAu) = adapters(st["gate"], dG), adapters(st["up"], dU)
    return {"dX": (dG @ Wg + dU @ Wu).to(dt), "dB_gate": dBg, "dA_gate": dAg, "dB_up": dBu, "dA_up": dAu}


def _newton_schulz(v):
    a, b, c = COEFFICIENTS
    wide = v.shape[0] <= v.shape[1]
    x = v if wide else v.T
    x = x / (x.square().sum().sqrt() + EPS)

    def step(x, _):
        S = x @ x.T
        return a * x + (b * S + c * (S @ S)) @ x

    x = functools.reduce(step, range(5), x)
    return x if wide else x.T


def _plain_ortho(st):
    case, dt = st["case"], _dt(st["case"])
    if case["run"] == "direction":
        return {"direction": torch.cat([_newton_schulz(g.float()).reshape(-1) for g in st["grads"]]).to(dt)}
    g = st["grad"].float()
    m = BETA * st["momentum"] + (1.0 - BETA) * g
    v = BETA * m + (1.0 - BETA) * g
    pieces = zip(v.split([t.numel() for t in st["grads"]]), st["grads"])
    moved = torch.cat([(math.sqrt(max(1.0, t.shape[0] / t.shape[1])) * _newton_schulz(x.view(t.shape))).reshape(-1) for x, t in pieces])
    st["momentum"].copy_(m)
    st["master"].copy_((1.0 - LR * DECAY) * st["master"] - LR * moved)
    st["param"].copy_(st["master"])
    return {"momentum": st["momentum"], "master": st["master"], "param": st["param"]}


def _column(v):
    return v.double().unsqueeze(1) if torch.is_tensor(v) else v


def _plain_sample(st):
    """In 64 bits: a token lies next to the border of another."""
    z = st["logits"].double()
    rows, V = z.shape
    T, k, p, low = (_column(st[name]) for name in ("temperature", "top_k", "top_p", "min_p"))
    T = torch.as_tensor(T, dtype=torch.float64, device="cuda")
    top = z.amax(1, keepdim=True)
    cold = torch.where(z == top, 1.0, 0.0) * torch.where((z == top).cumsum(1) == 1, 1.0, 0.0)  # the first of the largest
    w = torch.where(T > 0, torch.exp((z - top) / torch.where(T > 0, T, torch.ones_like(T))), cold)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    ranked = w.gather(1, order)
    rank = torch.arange(V, device="cuda", dtype=torch.float64).unsqueeze(0)
    k = torch.as_tensor(k, dtype=torch.float64, device="cuda")
    ranked = torch.where((k <= 0) | (rank < k), ranked, torch.zeros((), dtype=torch.float64, device="cuda"))
    run = ranked.cumsum(1)
    p = torch.as_tensor(p, dtype=torch.float64, device="cuda")
    kept = (ranked >= low) & ((p >= 1.0) | (run - ranked < p * run[:, -1:]))
    kept[:, 0] = True
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, ranked, torch.zeros((), dtype=torch.float64, device="cuda")))
    run = w.cumsum(1)
    token = (run <= st["u"].double().unsqueeze(1) * run[:, -1:]).sum(1, keepdim=True)
    last = torch.where(w > 0, torch.arange(V, device="cuda"), torch.full((), -1, device="cuda")).amax(1, keepdim=True)
    token = torch.minimum(token, last)
    return {"token": token.squeeze(1), "logp": torch.log(w.gather(1, token) / run[:, -1:]).squeeze(1).float()}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2501_08582_amd import ops, train

    case = st["case"]
    if case["op"] == "gated":
        gate, up = (tuple(st[k][n] for n in ("W", "M", "B", "A")) for k in ("gate", "up"))
        if case["run"] != "backward":
            H, G, U = ops.gated_forward(st["X"], gate, up, case["scale"], case["mask"], case["act"], save=case["run"] == "forward")
            return {"H": H} if case["run"] == "serve" else {"H": H, "G": G, "U": U}
        dX, (dBg, dAg), (dBu, dAu) = ops.gated_backward(st["dH"], st["X"], gate, up, st["G"], st["U"], case["scale"], case["mask"],
                                                        case["act"], grad_dtype=_dt(case))
        return {"dX": dX, "dB_gate": dBg, "dA_gate": dAg, "dB_up": dBu, "dA_up": dAu}
    if case["op"] == "ortho":
        if case["run"] == "direction":
            return {"direction": torch.cat([d.reshape(-1) for d in train.orthogonalize(st["grads"], coefficients=COEFFICIENTS, eps=EPS)])}
        if "optimizer" not in st:  # a program makes it once and keeps it
            st["optimizer"] = train.OrthogonalUpdate(st["masters"], st["params"], st["momenta"], momentum=BETA, nesterov=True,
                                                     weight_decay=DECAY, coefficients=COEFFICIENTS, eps=EPS)
        st["optimizer"].step(st["grads"], LR)
        return {"momentum": st["momentum"], "master": st["master"], "param": st["param"]}
    token, logp = train.sample(st["logits"], st["u"], st["temperature"], st["top_k"], st["top_p"], st["min_p"])
    return {"token": token, "logp": logp}


def run(state):
    if own:
        return _own(state)
    return {"gated": _plain_gated, "ortho": _plain_ortho, "sample": _plain_sample}[state["case"]["op"]](state)


def work(case):
    """Each input read once and each output written once; the products of the definition."""
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "gated":
        L, R, C, r = case["L"], case["R"], case["C"], case["r"]
        weights = 2 * (es * (R * C + (R + C) * r) + R * C // 8)
        if case["run"] == "backward":
            return {"bytes": weights + es * (2 * L * C + 3 * L * R + 2 * (R + C) * r), "flops": 2 * (4 * R * C * L + 6 * r * R * C)}
        return {"bytes": weights + es * (L * C + L * R * (1 if case["run"] == "serve" else 3)), "flops": 2 * (2 * R * C * L + 2 * r * R * C)}
    if case["op"] == "ortho":
        n = sum(r * c * k for r, c, k in _kinds(case))
        flops = sum(k * (4 * min(r, c) * r * c + 30 * min(r, c) ** 3) for r, c, k in _kinds(case))
        return {"bytes": n * (2 * es if case["run"] == "direction" else 2 * es + 16), "flops": flops}
    n = case["rows"] * case["vocab"]
    return {"bytes": es * n + 16 * case["rows"], "flops": 4 * n}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_gated(case, st):
    d = {k: st[k].double() for k in ("X", "G", "U", "dH") if k in st}

    def weight(p):
        W = torch.addmm(p["W"].double(), p["B"].double(), p["A"].double(), alpha=case["scale"])
        return (W * p["keep"]).to(_dt(case)).double()

    Wg, Wu = weight(st["gate"]), weight(st["up"])

    def act(g):
        g = g.detach().requires_grad_(True)
        if case["act"] == "silu":
            y = g * torch.sigmoid(g)
        else:
            y = g * 0.5 * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (g + 0.044715 * g**3)))
        (slope,) = torch.autograd.grad(y.sum(), g)
        return y.detach(), slope

    if case["run"] != "backward":
        G, U = torch.mm(d["X"], Wg.t()), torch.mm(d["X"], Wu.t())
        H = U * act(G)[0]
        return {"H": H} if case["run"] == "serve" else {"H": H, "G": G, "U": U}
    y, slope = act(d["G"])
    dU = d["dH"] * y
    dG = d["dH"] * d["U"] * slope

    def adapters(p, grad):
        D = torch.mm(grad.t(), d["X"]) * p["keep"] * case["scale"]
        return torch.mm(D, p["A"].double().t()), torch.mm(p["B"].double().t(), D)

    (dBg, dAg), (dBu, dAu) = adapters(st["gate"], dG), adapters(st["up"], dU)
    return {"dX": torch.mm(dU, Wu) + torch.mm(dG, Wg), "dB_gate": dBg, "dA_gate": dAg, "dB_up": dBu, "dA_up": dAu}


def _exact_direction(v):
    """By the eigenvalues of the shorter side's Gram matrix: the steps act on each of them alone."""
    x = v if v.shape[0] <= v.shape[1] else v.t()
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    lam, vec = torch.linalg.eigh(torch.mm(x, x.t()))
    lam = lam.clamp(min=0.0)
    a, b, c = COEFFICIENTS

    def once(factor, _):
        t = lam * factor * factor
        return factor * (a + t * (b + c * t))

    factor = functools.reduce(once, range(5), torch.ones_like(lam))
    out = torch.mm(vec * factor, torch.mm(vec.t(), x))
    return out if v.shape[0] <= v.shape[1] else out.t()


def _exact_ortho(case, st):
    if case["run"] == "direction":
        return {"direction": torch.cat([_exact_direction(t.double()).reshape(-1) for t in st["grads"]])}

    def one(g, m, w):
        m = torch.lerp(m.double(), g.double(), 1.0 - BETA)
        o = _exact_direction(torch.lerp(m, g.double(), 1.0 - BETA)) * max(1.0, w.shape[0] / w.shape[1]) ** 0.5
        return m.reshape(-1), (w.double() - LR * (DECAY * w.double() + o)).reshape(-1)

    momentum, master = zip(*(one(*t) for t in zip(st["grads"], st["momenta"], st["masters"])))
    return {"momentum": torch.cat(momentum), "master": torch.cat(master), "param": torch.cat(master)}


def _exact_token(z, u, T, k, p, low):
    """(token, log of its probability) of one row."""
    order = torch.argsort(-z, stable=True)
    if T == 0.0:
        return int(order[0]), 0.0
    order = order[: int(k)] if k >= 1 else order
    w = torch.softmax(z[order] / T, 0)
    n = len(w) if p >= 1.0 else 1 + int((w.cumsum(0)[:-1] < p).sum())
    n = max(1, min(n, int((w >= low * w[0]).sum())))
    at, by = order[:n].sort()
    w = w[by]
    run = w.cumsum(0)
    j = min(int(torch.searchsorted(run, u * run[-1], right=True)), int(torch.nonzero(w).max()))
    return int(at[j]), math.log(float(w[j] / run[-1]))


def _exact_sample(case, st):
    """A row at a time, on the host."""
    v = [(st[n] if torch.is_tensor(st[n]) else torch.full((case["rows"],), st[n], dtype=torch.float64)).double().tolist()
         for n in ("temperature", "top_k", "top_p", "min_p")]
    got = [_exact_token(*row) for row in zip(st["logits"].double().cpu(), st["u"].double().cpu(), *v)]
    return {"token": torch.tensor([t for t, _ in got]), "logp": torch.tensor([l for _, l in got], dtype=torch.float64)}


def exact(case, seed):
    st = prepare(case, seed)
    return {"gated": _exact_gated, "ortho": _exact_ortho, "sample": _exact_sample}[case["op"]](case, st)
