"""Edges of the operators around the layer on the GPU, against their fp64 oracle.
Bounds are those of ``test_gpu_train_ops.check``."""
import numpy as np
import pytest
import torch

from oracle import train as ot
from paper_2501_08582_amd import _lib, train
from test_gpu_train_ops import DT, check, f64, normal

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# log-probabilities of rows that begin with NaN, alone or among -Inf.  Many rows, a few
# rows, and rows that several workgroups share; each long enough for a lane that saw
# nothing else at first to see finite entries afterwards.
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(520, 9001), (520, 20000), (4, 8192), (4, 16384), (4, 100003), (1, 600001)])
def test_logprobs_keep_a_nan_before_finite_entries(rows, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    clean = torch.randn(rows, V, generator=g, device="cuda").to(DT[dtype])
    t = torch.full((rows,), V - 1, device="cuda")
    d = torch.ones(rows, device="cuda")
    for lead in (16 // clean.element_size(), V // 16, V // 8, V // 2):
        for rest in (float("nan"), -float("inf")):
            x = clean.clone()
            x[-1, :lead] = rest
            x[-1, 0] = float("nan")
            logp, stats = train.logprob_forward(x, t)
            assert torch.isnan(logp[-1]) and torch.isnan(stats[-1, 1]), (lead, rest)
            got = train.logprob_backward(d, x, t, stats)
            assert torch.isnan(got[-1]).all() and not torch.isnan(got[:-1]).any()
            # the other rows: V / 2048 steps, fewer than 64 joins and 4 |t| <= 4 . 12 roundings of the sum
            want, _, _ = ot.logprobs(f64(x[:-1][:4]), np.full(min(rows - 1, 4), V - 1))
            check("logp", logp[:-1][:4], want, 48 + 64 + V / 2048, 1)


# ---------------------------------------------------------------------------
# the paired loss of long sequences whose rewards are large and close: the margin is
# taken in 64 bits, where fewer than 2^13 roundings of 2^-53 of a reward are 2^-40 of it,
# and a pair's loss and the mean are rounded to fp32 once each
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("P,S,smoothing", [(8, 2048, 0.0), (4, 4096, 0.1), (1, 70000, 0.0), (600, 40, 0.2), (513, 1, 0.0)])
def test_preference_of_close_large_rewards(P, S, smoothing):
    rng = np.random.default_rng(P + S)
    won = rng.standard_normal((P, S)) * 2.0 - 60.0
    lost = won + rng.standard_normal((P, S)) * (10.0 / S**0.5)
    logp = torch.from_numpy(np.concatenate([won, lost]).astype(np.float32)).cuda()
    l64 = f64(logp)
    targets = torch.zeros(2 * P, S, dtype=torch.int64, device="cuda")
    loss, reward, dseq = train.preference_forward(logp, targets, 9, None, 0.1, smoothing)
    want = ot.preference(l64, np.ones_like(l64, dtype=bool), None, 0.1, smoothing)
    size = 0.1 * np.abs(l64).sum(1).max() * 2.0**-16
    check("reward", reward, want[1], size, 1)
    check("loss", loss, np.asarray(want[0]), size, 1)
    check("dseq", dseq, want[2], size * 0.1 / P, 1)
    assert torch.equal(dseq[:P], -dseq[P:])


# ---------------------------------------------------------------------------
# results of the paired loss under autograd, changed in place
# ---------------------------------------------------------------------------
def test_results_of_the_preference_loss_can_be_changed_in_place():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(4, 7, 99, generator=g, device="cuda", requires_grad=True)
    t = torch.randint(0, 99, (4, 7), generator=g, device="cuda")
    first, first_reward, _ = train.preference_loss(x, t, None, 0.2)
    (want,) = torch.autograd.grad(first, x)
    loss, reward, logp = train.preference_loss(x, t, None, 0.2)
    loss /= 2  # halves the gradient, exactly
    reward.mul_(3)
    logp.zero_()
    (got,) = torch.autograd.grad(loss, x)
    assert torch.equal(got, want / 2) and float(loss.detach()) == float(first.detach()) / 2
    assert torch.equal(reward, 3 * first_reward)
    loss, _, _ = train.preference_loss(x, t, None, 0.2)
    loss += x.square().sum()
    (got,) = torch.autograd.grad(loss, x)
    assert torch.equal(got, want + 2 * x.detach())
    loss, reward, _ = train.preference_loss(x, t, None, 0.2)
    loss.detach().mul_(0)
    (got,) = torch.autograd.grad(loss, x)
    assert torch.equal(got, want) and torch.equal(reward, first_reward)


# ---------------------------------------------------------------------------
# gradients of tables where the way of the sort changes, up to so many tokens that their
# digits' counts are scanned
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("n,vocab,cols", [(6144, 300, 24), (6145, 300, 24), (262144, 700, 8), (262145, 700, 9), (266241, 3, 1), (700001, 300001, 4), (1 << 21, 5000, 3)])
def test_embedding_gradient_of_many_tokens(n, vocab, cols):
    rng = np.random.default_rng(n + vocab)
    ids = rng.integers(-1, vocab + 1, n)  # some of them padding
    dy, dy64 = normal(rng, (n, cols), "f32")
    ok = (ids >= 0) & (ids < vocab)
    ref, size = (np.stack([np.bincount(ids[ok], a[ok, c], vocab) for c in range(cols)], 1) for a in (dy64, np.abs(dy64)))
    dev = torch.from_numpy(ids).cuda()
    got = train.embedding_backward(dy, dev, vocab)
    most = np.bincount(ids[ok]).max()  # in chunks of 32, then their sums, one after the other
    check("dE", got, ref, size, 66 + most / 32)
    assert torch.equal(train.embedding_backward(dy, dev.to(torch.int32), vocab), got)


def test_embedding_gradient_takes_time_in_proportion_to_its_tokens():
    times = []
    for n in (1 << 22, 1 << 26):
        ids = torch.randint(0, 512, (n,), dtype=torch.int32, device="cuda")
        dy = torch.ones(n, 1, device="cuda")
        got = train.embedding_backward(dy, ids, 512)  # sums of ones below 2^24 are exact
        assert torch.equal(got[:, 0].long(), torch.bincount(ids, minlength=512))
        best = float("inf")
        for _ in range(3):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            train.embedding_backward(dy, ids, 512)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        times.append(best)
    # 16 times the tokens; a term with their square would be 256 times as large
    assert times[1] < 40 * times[0], times


# ---------------------------------------------------------------------------
# empty batches: refusals are the same
# ---------------------------------------------------------------------------
def test_empty_batches_are_checked_too():
    x = torch.empty(0, 8, device="cuda")
    assert train.dropout(x, 0.1, 1, residual=x.clone()).shape == (0, 8)
    y, z, mean, rstd = train.norm_forward(x, torch.ones(8, device="cuda"), residual=x.clone(), p=0.1)
    assert y.shape == z.shape == (0, 8) and mean.shape == rstd.shape == (0,)
    for p in (-0.1, 1.0, float("nan")):
        for call in (lambda: train.dropout(x, p, 0), lambda: train.norm_forward(x, p=p)):
            with pytest.raises(_lib.LorsError) as e:
                call()
            assert e.value.status == _lib.ERR_SHAPE
            del e
    with pytest.raises(_lib.LorsError):
        train.norm_forward(x, eps=-1.0)
    with pytest.raises(_lib.LorsError):
        train.norm_forward(torch.empty(0, 32769, device="cuda"))


# ---------------------------------------------------------------------------
# the norm's weight gradients in bf16, the type that training asks for: those in fp32
# rounded once, and a bound of their own.  Each of its 8 sums of `rows` terms has fewer
# than 256 roundings in a chain, h is off by 128 of (|z| rstd + |h|).
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,kind", [(1, 40, "rms"), (7, 1000, "layer"), (700, 333, "rms"), (600, 5120, "layer"),
                                            (300, 20000, "rms")])
def test_norm_weight_gradients_in_bf16(rows, cols, kind, dtype):
    rng = np.random.default_rng(rows + cols)
    z, z64 = normal(rng, (rows, cols), dtype, 1.5, 0.7)
    dy, dy64 = normal(rng, (rows, cols), dtype)
    w, w64 = normal(rng, cols, dtype, 0.2, 1.0)
    _, _, mean, rstd = train.norm_forward(z, w, kind=kind)
    _, _, dw, db = train.norm_backward(dy, z, w, mean, rstd, kind, need_dbias=True, grad_dtype=torch.bfloat16)
    _, _, wide_w, wide_b = train.norm_backward(dy, z, w, mean, rstd, kind, need_dbias=True, grad_dtype=torch.float32)
    assert dw.dtype == db.dtype == torch.bfloat16
    assert torch.equal(dw, wide_w.bfloat16()) and torch.equal(db, wide_b.bfloat16())
    eps = float(np.float32(1e-5))
    _, want_w, want_b = ot.norm_backward(dy64, z64, w64, eps, kind == "rms")
    m64, s64 = ot.stats(z64, eps, kind == "rms")
    h = np.abs((z64 - m64) * s64)
    big = np.abs(z64).max(1, keepdims=True) * s64
    check("dweight", dw, want_w, (np.abs(dy64) * (big + h.max(1, keepdims=True) + h)).sum(0), 256)
    check("dbias", db, want_b, np.abs(dy64).sum(0), 256)
