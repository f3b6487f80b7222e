"""The operators around the layer on the GPU against their fp64 oracle.

Every output is compared element by element with a bound on its rounding:

    |got - ref| <= u |ref| + c 2^-24 scale

with u = 2^-8 (1 + 2^-7) for a bf16 result (8 significant bits) and 2^-23 for an fp32 one (its
own rounding, and a second one where the fp32 value lands on the other side of a tie), and with
`scale` the size of the terms that fp32 arithmetic rounds on the way and `c` the
number of such roundings.  Each test says how its c comes about.
"""
import gc

import numpy as np
import pytest
import torch

from oracle import train as ot
from paper_2501_08582_amd import _lib, train

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8 * (1 + 2.0**-7), torch.float32: 2.0**-23}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED, OFFSET = 0x9E3779B97F4A7C15, (5 << 32) + 77


@pytest.fixture(scope="module", autouse=True)
def no_tensors_left_behind():
    """A caught exception that a test keeps holds that test's frame, and so its tensors,
    in a cycle.  It is collected here, not while a later test watches the allocator."""
    yield
    gc.collect()


def f64(t):
    return t.detach().double().cpu().numpy()


def to_dev(a, dtype):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DT[dtype]).cuda()


def normal(rng, shape, dtype, std=1.0, mean=0.0):
    """A random device tensor, and its values in 64 bits."""
    t = to_dev(rng.standard_normal(shape) * std + mean, dtype)
    return t, f64(t)


def check(what, got, ref, scale, c):
    g = f64(got)
    assert g.shape == ref.shape, what
    bound = U[got.dtype] * np.abs(ref) + c * 2.0**-24 * np.broadcast_to(scale, ref.shape) + 1e-38
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(g - ref) <= bound) & ~(np.isnan(g) & np.isnan(ref)) & ~(np.isinf(ref) & (g == ref))
    if bad.any():
        k = np.unravel_index(int(np.argmax(bad)), bad.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, first at {k}: {g[k]!r} for {ref[k]!r}, "
                             f"bound {bound[k]:.3e}")


def odd_view(t):
    """The same values at an address that is a multiple of the element only."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    v = buf[1:].view(t.shape)
    v.copy_(t)
    assert v.data_ptr() % 16 != 0
    return v


# ---------------------------------------------------------------------------
# dropout: a product and a sum before the rounding, c = 2
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,p,residual", [
    (1, 1, 0.5, False), (3, 5, 0.3, True), (7, 64, 0.05, False), (130, 1003, 0.1, True), (2, 70001, 0.5, False),
    (5000, 3, 0.25, True), (33, 4096, 65535 / 65536, False), (9, 100, 0.0, True), (2100, 2048, 0.1, True)])
def test_dropout(rows, cols, p, residual, dtype):
    rng = np.random.default_rng(rows + cols)
    x, x64 = normal(rng, (rows, cols), dtype)
    r, r64 = normal(rng, (rows, cols), dtype, 2.0) if residual else (None, None)
    y = train.dropout(x, p, SEED, OFFSET, r)
    ref, kept = ot.dropout(x64, p, SEED, OFFSET, r64)
    f = 65536 / (65536 - ot.threshold(p))
    check("y", y, ref, np.abs(x64) * f + np.abs(ref), 2)
    if not residual:
        assert np.array_equal(f64(y) != 0, kept & (x64 != 0))
    again = train.dropout(odd_view(x), p, SEED, OFFSET, None if r is None else odd_view(r))
    assert torch.equal(y, again)


def test_dropout_selects_and_other_offsets_differ():
    x = torch.full((64, 1000), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = f64(train.dropout(x, 0.5, 1, 2))
    kept = ot.dropout(np.ones((64, 1000)), 0.5, 1, 2)[1]
    assert (y[~kept] == 0).all() and not np.isfinite(y[kept]).any()
    one = torch.ones(64, 1000, device="cuda")
    a, b, c = (train.dropout(one, 0.5, s, o) for s, o in ((1, 2), (1, 3), (2, 2)))
    assert not torch.equal(a, b) and not torch.equal(a, c)


def test_dropout_state_on_the_device():
    x = torch.randn(20, 300, device="cuda")
    state = torch.tensor([3, (1 << 33) + 4], device="cuda")
    assert torch.equal(train.dropout(x, 0.3, 10, 20, rng_state=state), train.dropout(x, 0.3, 13, 24 + (1 << 33)))


# ---------------------------------------------------------------------------
# norm.  A sum over a row goes through at most 4 units of 8 in a lane, 6 steps over
# the lanes and 16 over the waves: 54 roundings, with those of the terms below 64.
# The mean is off by 64 units of |z|, rstd by 34 of itself, h = (z - mean) rstd by
# both: c = 128 of |w| (max|z| rstd + |h|) covers the result.
# ---------------------------------------------------------------------------
NORM_COLS = [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 255, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2560, 2561, 4096,
             4097, 5120, 5121, 8191, 8192, 8193, 16384, 16385, 32767, 32768]


def _norm_case(rows, cols, dtype, rms, residual, p, weight, bias, train_too=True):
    rng = np.random.default_rng(rows * 7 + cols)
    x, x64 = normal(rng, (rows, cols), dtype, 1.5, 0.7)
    r, r64 = normal(rng, (rows, cols), dtype, 2.0) if residual else (None, None)
    w, w64 = normal(rng, cols, dtype, 0.2, 1.0) if weight else (None, None)
    b, b64 = normal(rng, cols, dtype, 0.3) if bias else (None, None)
    kind = "rms" if rms else "layer"
    drop = dict(p=p, seed=SEED, offset=OFFSET)
    y, z, mean, rstd = train.norm_forward(x, w, b, 1e-5, kind, r, **drop)
    eps = float(np.float32(1e-5))
    zref, kept = ot.dropout(x64, p, SEED, OFFSET, r64) if p else ((x64 if r64 is None else x64 + r64), None)
    factor = 65536 / (65536 - ot.threshold(p))
    if residual or p:
        check("z", z, zref, np.abs(x64) * factor + np.abs(zref), 2)
    else:
        assert z is x
    z64 = f64(z)  # normalised as it is stored
    ref = ot.norm(z64, w64, b64, eps, rms)
    m64, s64 = ot.stats(z64, eps, rms)
    h = (z64 - m64) * s64
    big = np.abs(z64).max(1, keepdims=True) * s64
    aw = np.ones(cols) if w64 is None else np.abs(w64)
    check("y", y, ref, aw * (big + np.abs(h)) + (0 if b64 is None else np.abs(b64)), 128)
    if not rms:
        check("mean", mean, m64[:, 0], np.abs(z64).max(1), 64)
    # constant rows: the deviations are the mean's own error
    check("rstd", rstd, s64[:, 0], s64[:, 0] * (1 + big[:, 0]), 128)
    if not train_too:
        return
    dy, dy64 = normal(rng, (rows, cols), dtype)
    dz, dz64 = normal(rng, (rows, cols), dtype) if residual else (None, None)
    got = train.norm_backward(dy, z, w, mean, rstd, kind, dz, need_dresidual=residual, need_dweight=True, need_dbias=True,
                              grad_dtype=torch.float32, **drop)
    d, dw, db = ot.norm_backward(dy64, z64, w64, eps, rms, dz64)
    # h of the kernel is off by 128 of (big + |h|), and enters d = rstd (g - m1 - h m2) twice
    g = np.abs(dy64) * aw
    gm, hm = g.max(1, keepdims=True), big + np.abs(h).max(1, keepdims=True)
    scale = s64 * gm * (1 + hm) ** 2 + (0 if dz64 is None else np.abs(dz64))
    if residual:
        check("dresidual", got[1], d, scale, 256)
    dx = d if kept is None else np.where(kept, d * factor, 0.0)
    check("dx", got[0], dx, scale * factor, 256)
    if kept is not None and not residual:
        assert not f64(got[0])[~kept].any()
    # column sums: at most 64 rows in a workgroup's turn, 32 slots and 48 more to join (rows <= 20000 here)
    check("dweight", got[2], dw, (np.abs(dy64) * (hm + np.abs(h))).sum(0), 256)
    check("dbias", got[3], db, np.abs(dy64).sum(0), 256)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", NORM_COLS)
def test_norm_widths(cols, dtype):
    _norm_case(5, cols, dtype, False, True, 0.1, True, True)
    _norm_case(3, cols, dtype, True, False, 0.0, True, False)


@pytest.mark.parametrize("rows,cols", [(1, 4096), (2, 70), (700, 333), (1100, 2300), (20000, 40), (3000, 64), (1030, 1000),
                                       (600, 9000), (1300, 5120), (520, 16400)])
@pytest.mark.parametrize("rms,residual,p,weight,bias", [(False, True, 0.2, True, True), (False, False, 0.0, False, False),
                                                        (True, True, 0.0, True, False), (True, False, 0.3, False, True)])
def test_norm_rows_and_options(rows, cols, rms, residual, p, weight, bias):
    _norm_case(rows, cols, "bf16", rms, residual, p, weight, bias)
    if rows < 3000:
        _norm_case(rows, cols, "f32", rms, residual, p, weight, bias)


def test_norm_equals_dropout_then_norm():
    for dt in DT.values():
        x, r = torch.randn(50, 1111, device="cuda").to(dt), torch.randn(50, 1111, device="cuda").to(dt)
        y, z, mean, rstd = train.norm_forward(x, kind="layer", residual=r, p=0.2, seed=3, offset=4)
        z2 = train.dropout(x, 0.2, 3, 4, residual=r)
        y2 = train.norm_forward(z2)
        assert torch.equal(z, z2) and torch.equal(y, y2[0]) and torch.equal(mean, y2[2]) and torch.equal(rstd, y2[3])
        u = train.norm_forward(odd_view(x), residual=odd_view(r), p=0.2, seed=3, offset=4)
        assert torch.equal(u[0], y) and torch.equal(u[1], z)


def test_norm_without_a_dropped_element():
    """p that rounds to no drop at 2^-16, on both sides of the first that does."""
    x = torch.randn(5, 300, device="cuda")
    for p in (0.0, 1e-9, 2.0**-17 * (1 - 2.0**-40), np.nextafter(2.0**-17, 0), 2.0**-17, 2.0**-16):
        y, z, mean, rstd = train.norm_forward(x, p=p, seed=1)
        if ot.threshold(p) == 0:
            assert z is x
        else:
            assert z is not x and torch.equal(z, train.dropout(x, p, 1))
        dx, dres, _, _ = train.norm_backward(x, z, None, mean, rstd, p=p, seed=1, need_dresidual=True)
        assert (dres is dx) == (ot.threshold(p) == 0)


def test_norm_repeats_its_bits():
    x, w, dy = torch.randn(3000, 640, device="cuda"), torch.randn(640, device="cuda"), torch.randn(3000, 640, device="cuda")
    _, z, mean, rstd = train.norm_forward(x, w)
    a = train.norm_backward(dy, z, w, mean, rstd, need_dbias=True)
    for _ in range(3):
        b = train.norm_backward(dy, z, w, mean, rstd, need_dbias=True)
        assert all(torch.equal(p, q) for p, q in zip((a[0], *a[2:]), (b[0], *b[2:])))


def test_norm_of_no_rows_and_large_offsets():
    x = torch.empty(0, 64, device="cuda")
    y, z, mean, rstd = train.norm_forward(x)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, _, dw, db = train.norm_backward(x, x, torch.ones(64, device="cuda"), mean, rstd, need_dbias=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    # a row far from zero: the variance comes from the deviations
    x = torch.randn(4, 4096, device="cuda") + 4096.0
    ref = ot.norm(f64(x), None, None, 1e-5, False)
    # mean off by 64 of 2^-24 of 4099, times rstd about 1
    assert np.abs(f64(train.norm_forward(x)[0]) - ref).max() <= 128 * 2.0**-24 * 4110


# ---------------------------------------------------------------------------
# embedding: a product each way; sums over a token's rows in order, at most 62 at its
# ends and one for every 32 between
# ---------------------------------------------------------------------------
def _ids(rng, n, vocab, how):
    if how == "one":
        return np.full(n, vocab // 2)
    if how == "zipf":
        ids = np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1)
    else:
        ids = rng.integers(0, vocab, n)
    if how == "padded":
        ids[rng.random(n) < 0.4] = -1
        ids[rng.random(n) < 0.1] = vocab
        ids[rng.random(n) < 0.05] = 2**31 - 1
    return ids


@pytest.mark.parametrize("n,vocab,cols,how,dtype", [
    (1, 1, 1, "even", "f32"), (1, 100, 8, "even", "bf16"), (31, 7, 64, "even", "f32"), (32, 7, 65, "even", "bf16"),
    (33, 1000, 128, "padded", "f32"), (64, 3, 129, "one", "f32"), (65, 1, 512, "one", "bf16"), (500, 50, 513, "zipf", "f32"),
    (3000, 20011, 771, "zipf", "bf16"), (8192, 1000, 40, "padded", "f32"), (8193, 512, 520, "zipf", "f32"),
    (16384, 300, 24, "zipf", "bf16"), (16385, 300, 24, "zipf", "bf16"), (20000, 70001, 136, "zipf", "f32"),
    (40961, 300001, 9, "padded", "f32"), (33000, 2, 16, "padded", "f32"), (17000, 512, 8, "one", "f32"),
    (255, 60, 72, "zipf", "bf16"), (256, 9, 1030, "padded", "f32"), (257, 9, 1030, "padded", "bf16"), (200, 3000, 5, "even", "bf16"),
    (256, 40, 64, "one", "bf16"), (4096, 600, 72, "zipf", "bf16"), (4097, 600, 72, "zipf", "f32"), (65536, 5000, 8, "zipf", "f32"), (65537, 5000, 8, "padded", "f32"),
    (70001, 300001, 12, "zipf", "bf16")])
def test_embedding(n, vocab, cols, how, dtype):
    rng = np.random.default_rng(n + vocab)
    ids = _ids(rng, n, vocab, how)
    table, t64 = normal(rng, (vocab, cols), dtype)
    dy, dy64 = normal(rng, (n, cols), dtype)
    scale = float(np.float32(1.7))
    dev = torch.from_numpy(ids).cuda()
    check("y", train.embedding_forward(dev, table, 1.7), ot.embedding(ids, t64, scale), 0.0, 0)
    ref = np.zeros((vocab, cols))
    size = np.zeros((vocab, cols))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(ref, ids[ok], scale * dy64[ok])
    np.add.at(size, ids[ok], scale * np.abs(dy64[ok]))
    got = train.embedding_backward(dy, dev, vocab, 1.7, grad_dtype=torch.float32)
    check("dE", got, ref, size, 66 + n / 32)
    assert torch.equal(train.embedding_backward(odd_view(dy), dev.to(torch.int32), vocab, 1.7), got.to(DT[dtype]))
    assert torch.equal(train.embedding_forward(dev.to(torch.int32), odd_view(table), 1.7),
                       train.embedding_forward(dev, table, 1.7))
    assert torch.equal(train.embedding_backward(dy, dev, vocab, 1.7, grad_dtype=torch.float32), got)


def test_embedding_padding_ignores_its_values_and_empty_batches():
    table = torch.randn(10, 33, device="cuda")
    ids = torch.tensor([[3, -1], [10, 3]], device="cuda")
    y = train.embedding_forward(ids, table)
    assert y.shape == (2, 2, 33) and not y[0, 1].any() and not y[1, 0].any() and torch.equal(y[0, 0], table[3])
    dy = torch.ones(2, 2, 33, device="cuda")
    dy[0, 1] = float("nan")
    dy[1, 0] = float("inf")
    want = torch.zeros(10, 33, device="cuda")
    want[3] = 2
    assert torch.equal(train.embedding_backward(dy, ids, 10), want)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert train.embedding_forward(none, table).shape == (0, 33)
    assert not train.embedding_backward(torch.empty(0, 33, device="cuda"), none, 10).any()


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,cols", [
    (3, 9, 1), (40, 21, 31), (40, 21, 32), (300, 21, 33), (300, 50, 64), (300, 33, 257), (260, 40, 1030), (70, 16, 2049)])
def test_embedding_gradient_at_any_address(n, vocab, cols, grad):
    """A table that starts anywhere in a cache line: the same gradient, and nothing
    written around it."""
    rng = np.random.default_rng(n + cols)
    ids = torch.from_numpy(_ids(rng, n, vocab, "padded")).cuda()
    dy, _ = normal(rng, (n, cols), "bf16")
    want = train.embedding_backward(dy, ids, vocab, 0.5, grad_dtype=DT[grad])
    d = train._embedding(ids, vocab, cols, 0.5, _lib.DTYPE_BF16, _lib.DTYPE_BF16 if grad == "bf16" else _lib.DTYPE_F32)
    need = _lib.embedding_workspace_bytes(d)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for shift in (1, 2, 31, 33, 63, 64):
        buf = torch.full((vocab * cols + 256,), 7.0, dtype=DT[grad], device="cuda")
        dE = buf[shift:shift + vocab * cols]
        status = _lib.embedding_backward(d, ids.data_ptr(), dy.data_ptr(), dE.data_ptr(), ws.data_ptr(), need,
                                         torch.cuda.current_stream().cuda_stream)
        assert status == 0
        assert torch.equal(dE.view(vocab, cols), want), shift
        assert (buf[:shift] == 7).all() and (buf[shift + vocab * cols:] == 7).all(), shift


# ---------------------------------------------------------------------------
# log-probabilities.  With t = x - top, a term's exponent is rounded twice and its
# exponential once: (3 |t| + 2) 2^-24 of it.  The sum takes vocab / 2048 steps in a
# lane and fewer than 64 to join.  Terms beyond |t| = 100 do not count in fp32.
# ---------------------------------------------------------------------------
def _sum_roundings(x64):
    top = x64.max(1)
    with np.errstate(invalid="ignore"):
        t = np.where(np.isfinite(x64), top[:, None] - x64, 0.0)
    return 4 * np.minimum(t.max(1), 100.0) + 64 + x64.shape[1] / 2048


def _check_logprobs(logits, targets, dtype):
    V = logits.shape[-1]
    x64, t = f64(logits).reshape(-1, V), targets.cpu().numpy().reshape(-1)
    counts = (t >= 0) & (t < V)
    x64 = np.where(counts[:, None], x64, 0.0)
    logp, stats = train.logprob_forward(logits, targets)
    rp, top, total = ot.logprobs(x64, t)
    c = _sum_roundings(x64)
    check("logp", logp.reshape(-1), rp, c, 1)
    check("sum", stats[..., 1].reshape(-1), total, c * total, 1)
    assert np.array_equal(f64(stats[..., 0]).reshape(-1), top)
    assert not f64(logp).reshape(-1)[~counts].any()
    rng = np.random.default_rng(V)
    d, d64 = normal(rng, targets.shape, "f32")
    got = train.logprob_backward(d, logits, targets, stats)
    ref = ot.logprobs_backward(d64.reshape(-1), x64, t)
    p = np.exp(x64 - top[:, None]) / np.maximum(total, 1.0)[:, None]
    # the sum's roundings, the term's own, a division and two products
    size = np.abs(d64).reshape(-1, 1) * p * (c[:, None] + 3 * np.minimum(top[:, None] - x64, 1e3) + 6)
    assert got.shape == logits.shape and got.dtype == DT[dtype] and got.is_contiguous()
    g = got.reshape(-1, V)
    # exponentials below 2^-126 are 0
    check("dlogits", g, np.where(counts[:, None], ref, 0.0), size + np.abs(ref) + 2.0**-100, 2)
    assert not f64(g)[~counts].any()
    return stats


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,length,V", [(1, 1, 1), (2, 3, 2), (1, 5, 7), (3, 1, 8), (2, 2, 9), (1, 4, 2047), (2, 3, 8192),
                                            (1, 1, 131072), (1, 2, 50021), (2, 600, 1003), (4, 300, 8193), (1, 3, 300001)])
def test_logprobs(batch, length, V, dtype):
    rng = np.random.default_rng(V + length)
    logits, _ = normal(rng, (batch, length, V), dtype, 3.0)
    t = rng.integers(0, V, (batch, length))
    t[rng.random(t.shape) < 0.2] = -100
    t.flat[-1] = V if t.size > 2 else t.flat[-1]
    targets = torch.from_numpy(t).cuda()
    _check_logprobs(logits, targets, dtype)
    a, b = train.logprob_forward(logits, targets), train.logprob_forward(odd_view(logits), targets.to(torch.int32))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_of_masked_entries(dtype):
    rng = np.random.default_rng(9)
    low = float(torch.finfo(DT[dtype]).min)
    for V in (100, 5000, 40000):
        x = rng.standard_normal((8, V)) * 3
        x[0, V // 2:] = -np.inf                # a masked tail
        x[1, : V // 2] = low                   # masked by the lowest value
        x[2] = low                             # all at the lowest value: an even distribution
        x[3, :-1] = -np.inf                    # one entry left: log-probability 0
        x[4, 0] = 80.0                         # one far above the rest
        logits = torch.from_numpy(x).to(DT[dtype]).cuda()  # from 64 bits: the lowest value stays itself
        t = np.array([3, V - 1, 5, V - 1, 7, V - 3, -100, -100])
        logits[6] = float("nan")               # rows that do not count
        logits[7] = float("inf")
        stats = _check_logprobs(logits.unsqueeze(0), torch.from_numpy(t).cuda().unsqueeze(0), dtype)
        assert not f64(stats)[0, 6:].any()
        # a masked target, a row without entries, a NaN
        y = torch.randn(3, V, device="cuda").to(DT[dtype])
        y[0, 4] = -float("inf")
        y[1] = -float("inf")
        y[2, 9] = float("nan")
        logp, _ = train.logprob_forward(y, torch.tensor([4, 4, 4], device="cuda"))
        got = f64(logp)
        assert got[0] == -np.inf and np.isnan(got[1]) and np.isnan(got[2])


def test_logprobs_of_strided_logits():
    for dt in DT.values():
        big = torch.randn(3, 12, 1040, device="cuda").to(dt)
        t = torch.randint(0, 1003, (3, 11), device="cuda")
        for view in (big[:, :-1, :1003], big[:, 1:, 5:1008]):
            a, b = train.logprob_forward(view, t), train.logprob_forward(view.contiguous(), t)
            assert torch.equal(a[0], b[0])
            d = torch.randn(3, 11, device="cuda")
            assert torch.equal(train.logprob_backward(d, view, t, a[1]),
                               train.logprob_backward(d, view.contiguous(), t, b[1]))
        d = torch.randn(3, device="cuda")
        u = torch.tensor(0.5, device="cuda")
        assert torch.equal(train.logprob_backward(d, big[:, :-1, :1003], t, a[1], upstream=u),
                           train.logprob_backward((0.5 * d).unsqueeze(1).expand(3, 11).contiguous(), big[:, :-1, :1003], t, a[1]))


# ---------------------------------------------------------------------------
# the preference loss: sums and functions in 64 bits, one rounding (c = 0 with a
# thousandth of it for the 64-bit sums)
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("P,S,smoothing,ref", [(1, 1, 0.0, True), (1, 0, 0.0, False), (3, 5, 0.1, True), (20, 64, 0.0, False),
                                               (1, 8192, 0.0, True), (2, 8193, 0.3, True), (300, 100, 0.5, True),
                                               (1, 70000, 0.0, True), (70, 300, 0.0, False)])
def test_preference(P, S, smoothing, ref):
    rng = np.random.default_rng(P + S)
    logp, l64 = normal(rng, (2 * P, S), "f32", 2.0, -6.0)
    r, r64 = normal(rng, (2 * P, S), "f32", 2.0, -6.0) if ref else (None, None)
    t = rng.integers(0, 99, (2 * P, S))
    t[rng.random(t.shape) < 0.3] = -100
    if P > 1:
        t[1] = -100  # a sequence without a counted token
    counts = t >= 0
    nan = torch.from_numpy(~counts).cuda()
    logp[nan] = float("nan")  # what is not counted is not used
    if ref:
        r[nan] = float("nan")
    beta = 0.05 if ref else 1e-3
    targets = torch.from_numpy(t).cuda()
    loss, reward, dseq = train.preference_forward(logp, targets, 99, r, beta, smoothing)
    with np.errstate(over="ignore"):
        want = ot.preference(np.where(counts, l64, 0.0), counts, None if r64 is None else np.where(counts, r64, 0.0), beta, smoothing)
    size = beta * (np.abs(l64) + 6).sum(1) * 2.0**-20
    check("reward", reward, want[1], size, 1)
    m = size.max() * 4 + 1e-3 if S else 1e-3
    check("loss", loss, np.asarray(want[0]), m, 1)
    check("dseq", dseq, want[2], np.abs(want[2]) * (1 + m), 2)
    again = train.preference_forward(logp, targets.to(torch.int32), 99, r, beta, smoothing)
    assert all(torch.equal(a, b) for a, b in zip((loss, reward, dseq), again))


def test_preference_of_far_margins():
    for gap in (50.0, 800.0, 5000.0):
        logp = torch.tensor([[-gap], [0.0]], device="cuda")
        t = torch.zeros(2, 1, dtype=torch.int64, device="cuda")
        loss, _, d = train.preference_forward(logp, t, 3, None, 1.0)
        assert abs(float(loss) - gap) <= 2.0**-23 * gap and abs(float(d[0]) + 1) < 1e-6
        loss, _, d = train.preference_forward(logp.flip(0).contiguous(), t, 3, None, 1.0)
        assert 0 <= float(loss) < 1e-20 and abs(float(d[0])) < 1e-20


# ---------------------------------------------------------------------------
# autograd, differences, streams, graphs
# ---------------------------------------------------------------------------
def _difference(f, x, v, step):
    """The central difference of the scalar f along v, in 64 bits of fp32 values."""
    return (float(f(x + step * v)) - float(f(x - step * v))) / (2 * step)


def test_gradients_by_differences():
    """fp32 forwards with steps of 1/64 along a direction: rounding is 2^-24 of sums of
    about 100 over a step, truncation step^2 times third derivatives of order 10;
    2 % of the gradient's own size along the direction's length covers both."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def rand(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def compare(f, x):
        x = x.requires_grad_(True)
        (grad,) = torch.autograd.grad(f(x), x)
        v = rand(*x.shape)
        with torch.no_grad():
            num = _difference(lambda q: f(q).double(), x.detach(), v, 1.0 / 64)
        size = float(grad.double().norm()) * 1.0
        assert abs(num - float((grad.double() * v.double()).sum())) <= 0.02 * size + 1e-4

    c, cz = rand(6, 90), rand(6, 90)
    w, b, r = rand(90), rand(90), rand(6, 90)
    for kind in ("layer", "rms"):
        def both(x=None, w=w, b=b, r=r, kind=kind):
            y, z = train.norm(x, w, b, 1e-5, kind, residual=r, p=0.25, seed=5, offset=6)
            return (y.double() * c).sum() + (z.double() * cz).sum()

        x0 = rand(6, 90)
        compare(lambda q: both(q), x0.clone())
        compare(lambda q: both(x0, w=q), w.clone())
        compare(lambda q: both(x0, b=q), b.clone())
        compare(lambda q: both(x0, r=q), r.clone())
    compare(lambda q: (train.dropout_add(q, 0.4, 1, 2, r).double() * c).sum(), rand(6, 90))
    compare(lambda q: (train.dropout_add(r, 0.4, 1, 2, q).double() * c).sum(), rand(6, 90))
    ids = torch.tensor([1, 4, 1, -1, 0, 4], device="cuda")
    compare(lambda q: (train.embedding(ids, q, 2.0).double() * c).sum(), rand(5, 90))
    t = torch.randint(0, 50, (6, 4), generator=g, device="cuda")
    t[0, 2] = -100
    ref, k = -4 + rand(6, 4), rand(6, 4)
    compare(lambda q: (train.token_logprobs(q, t).double() * k).sum(), rand(6, 4, 50))
    compare(lambda q: 3.0 * train.preference_loss(q, t, ref, 0.5, 0.1)[0].double(), rand(6, 4, 50))


def test_autograd_matches_the_plain_calls():
    x = torch.randn(2, 9, 130, device="cuda", requires_grad=True)
    w = torch.randn(130, device="cuda", requires_grad=True)
    y, z = train.norm(x, w)
    assert torch.equal(z, x)
    dy, dz = torch.randn_like(y), torch.randn_like(y)
    gx, gw = torch.autograd.grad([y, z], [x, w], [dy, dz])
    _, _, mean, rstd = train.norm_forward(x.detach(), w.detach())
    want = train.norm_backward(dy, x.detach(), w.detach(), mean, rstd, dZ=dz)
    assert torch.equal(gx, want[0]) and torch.equal(gw, want[2])
    (gz,) = torch.autograd.grad(train.norm(x, w)[1].sum(), [x])  # only the residual stream is used
    assert torch.equal(gz, torch.ones_like(x))
    logits = torch.randn(4, 7, 99, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    t = torch.randint(0, 99, (4, 7), device="cuda")
    loss, reward, logp = train.preference_loss(logits, t, None, 0.2)
    (g,) = torch.autograd.grad(loss, logits)
    step = train.preference_step(logits.detach(), t, None, 0.2)
    assert torch.equal(loss, step[0]) and torch.equal(reward, step[1]) and torch.equal(logp, step[2]) and torch.equal(g, step[3])


def test_second_derivatives_are_refused():
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    t = torch.zeros(3, dtype=torch.int64, device="cuda")
    for y in (train.norm(x)[0], train.dropout_add(x, 0.5, 1), train.embedding(t, x), train.token_logprobs(x, t)):
        (g,) = torch.autograd.grad(y.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(g.sum(), x)


def _everything(x, w, b, r, dy, ids, table, logits, t, ref, state):
    y, z, mean, rstd = train.norm_forward(x, w, b, residual=r, p=0.1, seed=1, offset=2, rng_state=state)
    back = train.norm_backward(dy, z, w, mean, rstd, dZ=dy, p=0.1, seed=1, offset=2, rng_state=state, need_dresidual=True,
                               need_dbias=True)
    e = train.embedding_forward(ids, table, 2.0)
    de = train.embedding_backward(e, ids, table.shape[0], 2.0)
    return [y, z, *back, train.dropout(x, 0.3, 5, rng_state=state), e, de, *train.preference_step(logits, t, ref)]


def _inputs(n_ids):
    g = torch.Generator(device="cuda").manual_seed(11)

    def rand(*s):
        return torch.randn(*s, generator=g, device="cuda").bfloat16()

    t = torch.randint(-1, 3000, (4, 33), generator=g, device="cuda")
    return [rand(300, 777), rand(777), rand(777), rand(300, 777), rand(300, 777),
            torch.randint(-1, 900, (n_ids,), generator=g, device="cuda"), rand(900, 64), rand(4, 33, 3000), t,
            -8 + rand(4, 33).float(), torch.zeros(2, dtype=torch.int64, device="cuda")]


@pytest.mark.parametrize("n_ids", [700, 20000])
def test_graph_replays_match_eager(n_ids):
    args = _inputs(n_ids)
    state = args[-1]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _everything(*args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _everything(*args)
    last = None
    for rep in range(4):
        state.copy_(torch.tensor([rep, 7 * rep]))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = _everything(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"replay {rep}"
        if last is not None:
            assert not torch.equal(last, outs[1])  # another mask
        last = outs[1].clone()


def test_calls_run_on_the_current_stream():
    args = _inputs(5000)
    want = _everything(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fresh = [torch.empty_like(a) for a in args]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for f, a in zip(fresh, args):
            f.copy_(a)
        got = _everything(*fresh)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---------------------------------------------------------------------------
# refusals of the Python layer
# ---------------------------------------------------------------------------
def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        train.dropout(x.cpu(), 0.1, 0)
    with pytest.raises(ValueError):
        train.dropout(x.t(), 0.1, 0)
    with pytest.raises(ValueError):
        train.dropout(x, 0.1, 0, residual=x[:2])
    with pytest.raises(TypeError):
        train.dropout(x.half(), 0.1, 0)
    for p in (-0.1, 1.0, float("nan")):
        with pytest.raises(_lib.LorsError) as e:
            train.dropout(x, p, 0)
        assert e.value.status == _lib.ERR_SHAPE
    with pytest.raises(_lib.LorsError) as e:
        train.dropout(x, 0.1, 0, out=x)
    assert e.value.status == _lib.ERR_ALIAS
    with pytest.raises(ValueError):
        train.norm_forward(x, torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        train.norm_forward(x, kind="batch")
    with pytest.raises(_lib.LorsError):
        train.norm_forward(torch.zeros(1, 32769, device="cuda"))
    with pytest.raises(ValueError):
        train.norm_backward(x, x, None, None, torch.ones(4, device="cuda"))
    with pytest.raises(TypeError):
        train.embedding_forward(t.to(torch.int16), x)
    with pytest.raises(ValueError):
        train.embedding_backward(x, t[:3], 5)
    with pytest.raises(ValueError):
        train.embedding_backward(x, t, 0)
    with pytest.raises(ValueError):
        train.logprob_forward(x.t(), torch.zeros(8, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        train.logprob_forward(x, t[:3])
    with pytest.raises(ValueError):
        train.logprob_backward(t.float(), x, t, t)
    lp = torch.zeros(4, 2, device="cuda")
    tt = torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        train.preference_forward(lp[:3], tt[:3], 9)
    with pytest.raises(_lib.LorsError):
        train.preference_forward(lp, tt, 9, smoothing=0.6)
    with pytest.raises(_lib.LorsError):
        train.preference_forward(lp[:0], tt[:0], 9)


# ---------------------------------------------------------------------------
# arrays of more than 2^31 elements
# ---------------------------------------------------------------------------
def test_dropout_and_norm_past_32_bits():
    rows, cols, tail = 70001, 32768, 3
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    x[-tail:] = torch.randn(tail, cols, device="cuda")
    y = train.dropout(x, 0.25, SEED, OFFSET)
    kept = ot.random16(tail, cols, SEED, OFFSET, first=rows - tail) >= ot.threshold(0.25)
    x64 = f64(x[-tail:])
    check("y", y[-tail:], np.where(kept, x64 * (65536 / 49152), 0.0), np.abs(x64) * 2, 2)
    del y
    got = train.norm_forward(x, residual=x)
    small = x[-tail:].contiguous()
    want = train.norm_forward(small, residual=small)
    assert all(torch.equal(g[-tail:], w) for g, w in zip(got, want))
    y, z, mean, rstd = got
    dx = train.norm_backward(x, z, None, mean, rstd)[0]
    assert torch.equal(dx[-tail:], train.norm_backward(small, want[1], None, want[2], want[3])[0])


def test_embedding_past_32_bits():
    vocab, cols = 600001, 4096
    table = torch.zeros(vocab, cols, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 5, vocab - 2, vocab - 1], device="cuda")
    table[vocab - 2:] = torch.randn(2, cols, device="cuda")
    y = train.embedding_forward(ids, table)
    assert torch.equal(y[0], table[-1]) and torch.equal(y[2], table[-2]) and not y[1].any()
    table.fill_(3.0)
    dy = torch.randn(4, cols, device="cuda").bfloat16()
    dE = train.embedding_backward(dy, ids, vocab)
    assert torch.equal(dE[-2], dy[2]) and torch.equal(dE[5], dy[1])
    assert torch.equal(dE[-1], (dy[0].float() + dy[3].float()).bfloat16())
    dE[-2:] = 0
    dE[5] = 0
    assert all(not part.any() for part in dE.split(100000))


def test_logprobs_past_32_bits():
    rows, V, tail = 17001, 131072, 5
    x = torch.zeros(rows, V, dtype=torch.bfloat16, device="cuda")
    x[-tail:] = torch.randn(tail, V, device="cuda") * 3
    t = torch.full((rows,), -100, device="cuda")
    t[-tail:] = torch.tensor([0, 7, V - 1, V - 2, 12345], device="cuda")
    logp, stats = train.logprob_forward(x, t)
    dx = train.logprob_backward(torch.ones(rows, device="cuda"), x, t, stats)
    x64, t64 = f64(x[-tail:]), t[-tail:].cpu().numpy()
    rp, top, total = ot.logprobs(x64, t64)
    c = _sum_roundings(x64)
    check("logp", logp[-tail:], rp, c, 1)
    ref = ot.logprobs_backward(np.ones(tail), x64, t64)
    p = np.exp(x64 - top[:, None]) / total[:, None]
    check("dlogits", dx[-tail:], ref, p * (c[:, None] + 3 * (top[:, None] - x64) + 6) + np.abs(ref) + 2.0**-100, 2)
    assert not logp[:-tail].any() and all(not part.any() for part in dx[:-tail].split(4000))
