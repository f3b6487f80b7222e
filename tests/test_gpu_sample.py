"""Sampling on the GPU against its fp64 definition.

Tokens are equal: weights and sums are in 64 bits on both sides, so that two of the
given random numbers would have to lie within 2^-40 of a border to differ.  logp is
rounded once to fp32 (2^-24 of its value), from a logarithm of 64-bit sums (2^-40).
"""
import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2501_08582_amd import _lib, train

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def device(z, dtype):
    t = torch.from_numpy(np.asarray(z, np.float32)).to(DT[dtype]).cuda()
    return t, t.double().cpu().numpy()


def check(z64, u, token, logp, T=1.0, k=0, p=1.0, low=0.0):
    rows = z64.shape[0]
    take = lambda v, i: v if np.ndim(v) == 0 else v[i]  # noqa: E731
    token, logp = token.cpu().numpy(), logp.double().cpu().numpy()
    assert token.shape == logp.shape == (rows,)
    for i in range(rows):
        t, l = ob.sample(z64[i], u[i], take(T, i), take(k, i), take(p, i), take(low, i))
        assert token[i] == t, (i, token[i], t, [take(v, i) for v in (T, k, p, low)])
        assert np.isnan(l) and np.isnan(logp[i]) or abs(logp[i] - l) <= 2.0**-24 * abs(l) + 2.0**-40, (i, logp[i], l)


def run(z, u, dtype, **kw):
    t, z64 = device(z, dtype)
    u32 = np.asarray(u, np.float32)
    token, logp = train.sample(t, torch.from_numpy(u32).cuda(), **kw)
    names = {"temperature": "T", "top_k": "k", "top_p": "p", "min_p": "low"}
    check(z64, u32, token, logp, **{names[n]: v for n, v in kw.items()})
    return token


FILTERS = [{}, {"temperature": 0.7}, {"temperature": 0.0}, {"top_k": 1}, {"top_k": 5}, {"top_k": 700}, {"top_p": 0.9}, {"top_p": 0.0},
           {"top_p": 0.999}, {"min_p": 0.05}, {"min_p": 1.0}, {"min_p": 2.0}, {"temperature": 1.5, "top_k": 50, "top_p": 0.8, "min_p": 0.02},
           {"top_k": 3, "top_p": 0.5}, {"temperature": 0.02, "top_p": 0.99}, {"temperature": 300.0, "top_k": 40, "top_p": 0.95}]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 65, 511, 513, 1000, 4097, 20011])
def test_filters(V, dtype):
    rng = np.random.default_rng(V)
    z = rng.standard_normal((6, V)) * 3
    u = [0.0, 0.1, 0.5, 0.77, 0.999, np.nextafter(np.float32(1), np.float32(0))]
    for kw in FILTERS:
        run(z, u, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_vocabularies(dtype):
    """Beyond one block of a run, a count that is no multiple of anything."""
    rng = np.random.default_rng(1)
    z = rng.standard_normal((3, 1200007)).astype(np.float32) * 2.5
    for kw in ({}, {"top_p": 0.95}, {"top_k": 1000, "top_p": 0.9}, {"top_k": 600000}, {"min_p": 0.001}):
        run(z, [0.03, 0.5, 0.98], dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_entry_of_a_small_distribution(dtype):
    """Random numbers on a grid give each entry its share of them."""
    rng = np.random.default_rng(2)
    z = np.tile(rng.standard_normal(37) * 2, (512, 1))
    z[:, 11] = -np.inf
    u = (np.arange(512) + 0.5) / 512
    token = run(z, u, dtype, temperature=0.9, top_p=0.97)
    t, z64 = device(z[:1], dtype)
    w = ob.kept(z64[0], 0.9, 0, 0.97, 0.0)
    share = np.bincount(token.cpu().numpy(), minlength=37) / 512
    assert np.abs(share - w / w.sum()).max() <= 1 / 512 and share[11] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 3000, 70001])
def test_equal_logits(V, dtype):
    """Ties go to the lowest index, also where more are equal than are sorted at a time."""
    z = np.zeros((4, V))
    z[1, :] = 5.0
    z[2, V // 3:] = -2.0
    z[3, ::2] = 1.5
    u = [0.2, 0.999, 0.6, 0.4]
    for kw in ({}, {"temperature": 0.0}, {"top_k": 7}, {"top_k": V - 1}, {"top_k": V // 2 + 1}, {"top_p": 0.3}, {"top_p": 0.77, "top_k": V // 2},
               {"min_p": 0.5}):
        run(z, u, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_clusters_far_from_the_largest(dtype):
    """Borders in a crowded last bin: a lone large logit over values that hardly differ, and denormal,
    huge and signed-zero logits, which keep their order."""
    rng = np.random.default_rng(3)
    V = 9000
    z = np.zeros((5, V))
    z[0] = 1e-3 * rng.standard_normal(V)
    z[0, 77] = 60.0
    z[1] = rng.standard_normal(V) * 1e-40
    z[2] = rng.standard_normal(V) * 1e36
    z[3] = rng.choice([0.0, -0.0, 1e-45, -1e-45], V)
    z[4] = -1e30 - rng.random(V) * 1e29
    u = [0.9999, 0.4, 0.5, 0.6, 0.7]
    for kw in ({}, {"top_k": 4000}, {"top_k": 2}, {"top_p": 0.6}, {"top_k": 5000, "top_p": 0.4}, {"temperature": 1e30, "top_p": 0.5},
               {"temperature": 1e-30, "top_k": 3}):
        run(z, u, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_distribution(dtype):
    low = float(torch.finfo(DT[dtype]).min)
    V = 300
    z = np.zeros((7, V))
    z[0, 5] = np.nan
    z[1, 299] = np.inf
    z[2] = -np.inf
    z[3] = low
    z[4] = -np.inf
    z[4, 123] = -7.0
    z[5] = low
    z[5, 200:210] = 3.0
    z[6, :100] = -np.inf
    u = [0.5] * 7
    for kw in ({}, {"temperature": 0.0}, {"top_k": 250}, {"top_p": 0.9, "min_p": 0.1}, {"top_k": 150, "top_p": 0.5}):
        run(z, u, dtype, **kw)


def test_random_numbers_at_the_ends():
    """u = 0 takes the first kept entry of positive weight, u of 1 and above and NaN the last."""
    z = np.full((5, 200), -np.inf)
    z[:, 20:180] = 0.25
    t, z64 = device(z, "f32")
    u = torch.tensor([0.0, 1.0, 7.0, float("nan"), -1.0], device="cuda")
    token, logp = train.sample(t, u)
    assert token.tolist() == [20, 179, 179, 179, 20]
    assert np.abs(logp.double().cpu().numpy() + np.log(160)).max() < 1e-6


def test_parameters_of_each_row():
    rng = np.random.default_rng(4)
    rows, V = 64, 5003
    z = rng.standard_normal((rows, V)) * 3
    t, z64 = device(z, "bf16")
    u = rng.random(rows).astype(np.float32)
    T = rng.choice([0.0, 0.5, 1.0, 1.7, -1.0, np.nan], rows).astype(np.float32)
    k = rng.choice([-3, 0, 1, 17, 2000, 9999], rows).astype(np.int32)
    p = rng.choice([1.0, 0.9, 0.3, 0.0, 1.5, np.nan], rows).astype(np.float32)
    low = rng.choice([0.0, 0.1, 0.9, -1.0, np.nan], rows).astype(np.float32)
    dev = [torch.from_numpy(a).cuda() for a in (u, T, k, p, low)]
    token, logp = train.sample(t, *dev)
    fix = lambda a, to: np.where(np.isnan(a), to, a).astype(np.float64)  # noqa: E731
    check(z64, u, token, logp, fix(T, 0.0), k, fix(p, 1.0), fix(low, 0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_rows(dtype):
    rng = np.random.default_rng(5)
    big, _ = device(rng.standard_normal((9, 1300)) * 3, dtype)
    part = big[1::2, 3:1002]  # rows start at any multiple of an element
    u = rng.random(4).astype(np.float32)
    token, logp = train.sample(part, torch.from_numpy(u).cuda(), top_p=0.9)
    check(part.double().cpu().numpy(), u, token, logp, p=0.9)
    same = big[:1].expand(4, -1)
    token, logp = train.sample(same, torch.from_numpy(u).cuda(), top_k=30)
    check(same.double().cpu().numpy(), u, token, logp, k=30)


def test_offsets_past_32_bits():
    stride, rows, V = (1 << 27) + 5, 20, 40
    flat = torch.zeros(stride * (rows - 1) + V, dtype=torch.bfloat16, device="cuda")
    z = flat.as_strided((rows, V), (stride, 1))
    rng = np.random.default_rng(6)
    z.copy_(device(rng.standard_normal((rows, V)) * 2, "bf16")[0])
    u = rng.random(rows).astype(np.float32)
    token, logp = train.sample(z, torch.from_numpy(u).cuda(), top_p=0.8)
    check(z.double().cpu().numpy(), u, token, logp, p=0.8)


def test_many_rows_leading_dims_and_none():
    rng = np.random.default_rng(7)
    z, z64 = device(rng.standard_normal((1500, 33)) * 2, "bf16")
    u = rng.random(1500).astype(np.float32)
    ud = torch.from_numpy(u).cuda()
    token, logp = train.sample(z, ud, top_k=9)
    check(z64, u, token, logp, k=9)
    t3, l3 = train.sample(z.view(15, 100, 33), ud.view(15, 100), top_k=9)
    assert t3.shape == (15, 100) and torch.equal(t3.view(-1), token) and torch.equal(l3.view(-1), logp)
    t1, l1 = train.sample(z[3], ud[3], top_k=9)
    assert t1.shape == () and int(t1) == int(token[3])
    t0, _ = train.sample(z[:0], ud[:0])
    assert t0.shape == (0,)


def test_nothing_is_written_past_the_end_and_logp_may_be_left_out():
    rng = np.random.default_rng(8)
    z, z64 = device(rng.standard_normal((5, 1001)), "bf16")
    u = torch.full((5,), 0.5, device="cuda")
    token = torch.full((9,), 77, dtype=torch.int64, device="cuda")
    logp = torch.full((9,), 77.0, device="cuda")
    d = _lib.Sample(5, 1001, 1001, 1.0, 0, 0.9, 0.0, _lib.DTYPE_BF16, 0)
    st = torch.cuda.current_stream().cuda_stream
    for l in (logp.data_ptr() + 8, None):
        token.fill_(77)
        _lib.check(_lib.sample(d, z.data_ptr(), u.data_ptr(), None, None, None, None, token.data_ptr() + 16, l, None, 0, st), "sample")
        torch.cuda.synchronize()
        assert token[:2].eq(77).all() and token[7:].eq(77).all() and logp[:2].eq(77).all() and logp[7:].eq(77).all()
        check(z64, np.full(5, 0.5, np.float32), token[2:7], logp[2:7], p=0.9)


def test_other_stream_graph_and_repeats():
    rng = np.random.default_rng(9)
    z, _ = device(rng.standard_normal((20, 30011)) * 3, "bf16")
    u = torch.from_numpy(rng.random(20).astype(np.float32)).cuda()
    kw = dict(temperature=0.9, top_k=3000, top_p=0.95, min_p=1e-4)
    want = train.sample(z, u, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = train.sample(z, u, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = train.sample(z, u, **kw)
    for k in range(3):
        u.copy_(torch.rand(20, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, train.sample(z, u, **kw)))


def test_refusals():
    z, u = torch.zeros(3, 10, device="cuda"), torch.zeros(3, device="cuda")
    for kw, what in (({"temperature": -1.0}, "SHAPE"), ({"temperature": float("nan")}, "SHAPE"), ({"top_p": -0.1}, "SHAPE"),
                     ({"top_p": float("nan")}, "SHAPE"), ({"min_p": -0.1}, "SHAPE"), ({"min_p": float("inf")}, "SHAPE")):
        with pytest.raises((ValueError, _lib.LorsError), match=f"invalid|{what}"):
            train.sample(z, u, **kw)
    with pytest.raises(ValueError, match="u:"):
        train.sample(z, u[:2].clone())
    with pytest.raises(ValueError, match="u:"):
        train.sample(z, u.double())
    with pytest.raises(ValueError, match="top_k"):
        train.sample(z, u, top_k=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="temperature"):
        train.sample(z, u, temperature=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        train.sample(z.t(), torch.zeros(10, device="cuda"))
    with pytest.raises(ValueError, match="on the GPU"):
        train.sample(z.cpu(), u)
    with pytest.raises(ValueError, match="at least one"):
        train.sample(z[:, :0], u)
    with pytest.raises(TypeError):
        train.sample(z.half(), u)
