"""Orthogonalised updates on the GPU against their fp64 definition.

The steps and the direction's sums are in 64 bits, so a direction is off by its one
rounding (u = 2^-24 in fp32, 2^-8 in bf16, relative) and by what fp64 roundings grow to: 2^-53 of S's
norm, times a^(2 steps) = 2^17.8 in the steps and 2^9 in their product, below 2^-25.
m takes two roundings in fp32 and v two more (fused multiply-adds on a rounded product), each of the
size of its larger term; they move the direction by that, relative to |v|, times the
steps' gain a^5 = 485, a bound that is checked as a norm.  The master adds two roundings.
"""
import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2501_08582_amd import _lib, train

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8 * (1 + 2.0**-7), torch.float32: 2.0**-23}
ABC = train.COEFFICIENTS
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().double().cpu().numpy()


def matrix(rng, rows, cols, dtype, rank=None):
    """Noise over a few strong directions, as gradients have."""
    k = rank or max(1, min(rows, cols) // 4)
    a = rng.standard_normal((rows, k)) @ (rng.standard_normal((k, cols)) * np.exp(-0.7 * np.arange(k))[:, None])
    if rank is None:
        a = a + 0.02 * rng.standard_normal((rows, cols))
    return torch.from_numpy((1e-3 * a).astype(np.float32)).to(DT[dtype]).cuda()


def close(what, got, ref, slack=2.0**-25):
    g = f64(got)
    bound = U[got.dtype] * np.abs(ref) + slack
    bad = ~(np.abs(g - ref) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(g - ref)[bad].max():.3e}"


# every size class of the short side at its ends and odd, one row or column, lengths of
# one, below a run of lanes, over a piece's end, and both orientations
SHAPES = [(1, 1), (1, 700), (5, 1), (3, 3), (16, 64), (13, 517), (517, 13), (16, 4096), (17, 33), (32, 1000), (1000, 31), (33, 513),
          (64, 1024), (1500, 64), (63, 2051), (37, 5003), (5003, 37), (65, 200), (128, 1025), (1025, 128), (100, 777), (777, 101),
          (128, 128), (2, 140001), (140001, 3),
          (48, 1000), (1000, 48), (2051, 41), (41, 700), (96, 1031), (1031, 96), (90, 300), (300, 70), (49, 500), (97, 300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_direction(shape, dtype):
    rng = np.random.default_rng(shape[0] * 1009 + shape[1])
    x = matrix(rng, *shape, dtype)
    close("direction", train.orthogonalize(x), ob.direction(f64(x), 5, *ABC, 1e-7))


@pytest.mark.parametrize("steps,abc", [(1, ABC), (2, ABC), (10, ABC), (7, (1.5, -0.5, 0.0)), (30, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(steps, abc):
    rng = np.random.default_rng(steps)
    for shape in ((24, 333), (300, 40), (100, 333), (200, 90)):
        x = matrix(rng, *shape, "f32")
        # ten steps of slope 2 to 3 around their cycle raise 2^-53 to 2^-37 at most
        close("direction", train.orthogonalize(x, steps=steps, coefficients=abc), ob.direction(f64(x), steps, *abc, 1e-7))


def test_singular_values_come_near_one():
    rng = np.random.default_rng(0)
    x = matrix(rng, 64, 500, "f32")
    s = np.linalg.svd(f64(train.orthogonalize(x)), compute_uv=False)
    assert s.min() > 0.6 and s.max() < 1.3


@pytest.mark.parametrize("shape", [(16, 300), (300, 64), (90, 300), (300, 128)])
def test_rank_deficient_and_zero(shape):
    rng = np.random.default_rng(1)
    x = matrix(rng, *shape, "f32", rank=3)
    # in the directions that x has by its own rounding alone (2^-24 of |x|) the steps' factor is 485
    close("low rank", train.orthogonalize(x), ob.direction(f64(x), 5, *ABC, 1e-7), slack=2.0**-25)
    z = torch.zeros(shape, device="cuda")
    assert not train.orthogonalize(z).any()
    assert torch.isnan(train.orthogonalize(z, eps=0.0)).all()  # 0 / 0, as the definition has it


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e18, 1e30])
def test_scales(scale):
    """Squares that fp32 could not hold."""
    rng = np.random.default_rng(2)
    x = torch.from_numpy((scale * rng.standard_normal((20, 90))).astype(np.float32)).cuda()
    close("scaled", train.orthogonalize(x, eps=0.0), ob.direction(f64(x), 5, *ABC, 0.0))


def test_one_bad_matrix_spoils_no_other():
    rng = np.random.default_rng(3)
    xs = [matrix(rng, 16, 200, "f32") for _ in range(4)]
    want = [train.orthogonalize(x) for x in xs]
    xs[1][3, 5] = float("nan")
    xs[2][0, 0] = float("inf")
    got = train.orthogonalize(xs)
    assert torch.isnan(got[1]).all() and torch.isnan(got[2]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])


def test_many_matrices_of_mixed_shapes():
    """More than a launch holds, of every size class; each as by itself, bit for bit."""
    rng = np.random.default_rng(4)
    shapes = [SHAPES[i % len(SHAPES)] for i in range(130)]
    xs = [matrix(rng, *s, "bf16") for s in shapes]
    got = train.orthogonalize(xs)
    for x, g in zip(xs, got):
        assert torch.equal(g, train.orthogonalize(x))


def group(shapes, gdt, pdt, seed=0):
    rng = np.random.default_rng(seed)
    grads = [matrix(rng, *s, gdt) for s in shapes]
    momenta = [matrix(rng, *s, "f32") for s in shapes]
    masters = [torch.from_numpy((0.05 * rng.standard_normal(s)).astype(np.float32)).cuda() for s in shapes]
    params = None if pdt is None else [w.to(DT[pdt], copy=True) for w in masters]
    return grads, momenta, masters, params


@pytest.mark.parametrize("gdt,pdt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", None), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("nesterov", [True, False])
def test_optimiser_steps(gdt, pdt, nesterov):
    shapes = [(16, 4096), (700, 16), (5, 33), (33, 5), (64, 1031), (1031, 60), (128, 300), (300, 100)]
    grads, momenta, masters, params = group(shapes, gdt, pdt)
    opt = train.OrthogonalUpdate(masters, params, momenta, momentum=0.9, nesterov=nesterov, weight_decay=0.1)
    lr = 0.02
    for k in range(2):
        before = [(f64(g), f64(m), f64(w)) for g, m, w in zip(grads, momenta, masters)]
        opt.step(grads, lr)
        for i, (g, m, w) in enumerate(before):
            rate = lr * max(1.0, g.shape[0] / g.shape[1]) ** 0.5
            rm, rw = ob.update(g, m, w, 0.9, nesterov, rate, lr * 0.1, 5, *ABC, 1e-7)
            size = 0.9 * np.abs(m) + 0.1 * np.abs(g)
            assert (np.abs(f64(momenta[i]) - rm) <= 2 * 2.0**-24 * size + 2.0**-24 * np.abs(rm)).all()
            # the direction's own error: v off by four roundings, the steps' gain 485; one fp32 rounding
            err = np.linalg.norm(f64(masters[i]) - rw)
            allowed = rate * (485 * 4 * 2.0**-24 + 2.0**-24 * np.sqrt(min(g.shape)) * 1.3) + 2 * 2.0**-24 * np.linalg.norm(np.abs(w) + rate)
            assert err <= allowed, (i, err, allowed)
            if params is not None:
                assert torch.equal(params[i], masters[i].to(params[i].dtype))
        grads = [g * -0.5 for g in grads]
    if pdt is None:
        assert opt.params is None


def test_parameters_that_are_their_own_masters():
    shapes = [(16, 300), (77, 9)]
    grads, momenta, masters, _ = group(shapes, "f32", None)
    twins = [w.clone() for w in masters], [m.clone() for m in momenta]
    train.OrthogonalUpdate(masters, masters, momenta).step(grads, 0.1)
    train.OrthogonalUpdate(twins[0], None, twins[1]).step(grads, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(masters + momenta, twins[0] + twins[1]))
    with pytest.raises(_lib.LorsError):  # another's master is not its own
        train.OrthogonalUpdate(masters[:1] + [twins[0][1]], [masters[0], masters[1][:, :].reshape(77, 9)],
                               momenta[:1] + [masters[1]]).step(grads, 0.1)


def test_momenta_start_at_zero_and_lr_changes():
    grads, _, masters, _ = group([(8, 40)], "f32", None)
    w0 = masters[0].clone()
    opt = train.OrthogonalUpdate(masters)
    opt.step(grads, 0.5)
    close("m", opt.momenta[0], 0.05 * f64(grads[0]), slack=2.0**-24 * 1e-2)
    d = ob.direction(f64(grads[0]), 5, *ABC, 1e-7)  # the first m is a multiple of the gradient
    assert np.abs(f64(masters[0]) - (f64(w0) - 0.5 * d)).max() < 1e-4
    w1 = masters[0].clone()
    opt.step(grads, 0.0)
    assert torch.equal(masters[0], w1)


@pytest.mark.parametrize("shape", [(16, 333), (333, 37), (64, 515), (100, 515), (333, 90)])
def test_nothing_is_written_past_the_end(shape):
    """Every array at an odd place between others; the workspace to its last byte."""
    rows, cols = shape
    n, pad = rows * cols, 257
    rng = np.random.default_rng(5)
    g = torch.zeros(n + 2 * pad, dtype=torch.bfloat16, device="cuda")
    m, w = (torch.full((n + 2 * pad,), 7.0, device="cuda") for _ in range(2))
    q = torch.full((n + 2 * pad,), 7.0, dtype=torch.bfloat16, device="cuda")
    inner = slice(pad, pad + n)
    g[inner] = matrix(rng, *shape, "bf16").view(-1)
    m[inner] = 0
    w[inner] = 1
    p = _lib.Update(0.95, 1e-7, *ABC, 5, 1, _lib.DTYPE_BF16, _lib.DTYPE_BF16, 0)
    items = (_lib.UpdateItem * 1)((rows, cols, g.data_ptr() + 2 * pad, m.data_ptr() + 4 * pad, w.data_ptr() + 4 * pad,
                                   q.data_ptr() + 2 * pad, 0.1, 0.0))
    need = _lib.orthogonal_workspace_bytes(p, items, 1)
    ws = torch.full((need + 4096,), 33, dtype=torch.uint8, device="cuda")
    _lib.check(_lib.orthogonal_update(p, items, 1, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream), "update")
    torch.cuda.synchronize()
    assert (ws[need:] == 33).all()
    for t, fill in ((g, 0), (m, 7), (w, 7), (q, 7)):
        assert (t[:pad] == fill).all() and (t[pad + n:] == fill).all()
    ref = 1.0 - 0.1 * ob.direction(f64(g[inner].view(shape)), 5, *ABC, 1e-7)
    assert np.abs(f64(w[inner].view(shape)) - ref).max() < 1e-4


def test_other_stream_and_graph_replays():
    shapes = [(16, 700), (300, 64), (9, 9), (100, 300)] + [(8, 40)] * 50  # every kind of launch
    grads, momenta, masters, params = group(shapes, "bf16", "bf16")
    twin = [[t.clone() for t in ts] for ts in (momenta, masters, params)]
    opt = train.OrthogonalUpdate(masters, params, momenta)
    ref = train.OrthogonalUpdate(twin[1], twin[2], twin[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step(grads, 0.02)
    torch.cuda.current_stream().wait_stream(side)
    ref.step(grads, 0.02)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(grads, 0.01)
    for k in range(3):
        for g in grads:
            g.mul_(-0.7)
        graph.replay()
        torch.cuda.synchronize()
        ref.step(grads, 0.01)
        for got, want in zip((momenta, masters, params), twin):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x = torch.randn(8, 40, device="cuda")
    assert train.orthogonalize([]) == []
    assert train.orthogonalize(x[:0]).shape == (0, 40)
    with pytest.raises(ValueError, match="matrix 0"):
        train.orthogonalize(x[0])
    with pytest.raises(ValueError, match="contiguous"):
        train.orthogonalize(x.t())
    with pytest.raises(ValueError, match="on the GPU"):
        train.orthogonalize(x.cpu())
    with pytest.raises(TypeError):
        train.orthogonalize(x.half())
    with pytest.raises(ValueError, match="invalid"):
        train.orthogonalize(torch.zeros(129, 200, device="cuda"))
    with pytest.raises(ValueError, match="invalid"):
        train.orthogonalize(x, steps=0)
    with pytest.raises(ValueError, match="invalid"):
        train.orthogonalize(x, steps=11)  # 3.4445^22 is above 2^38
    with pytest.raises(ValueError, match="no matrices"):
        train.OrthogonalUpdate([])
    with pytest.raises(ValueError, match="master 0"):
        train.OrthogonalUpdate([x.bfloat16()])
    with pytest.raises(ValueError, match="param 0"):
        train.OrthogonalUpdate([x], [x[:4]])
    opt = train.OrthogonalUpdate([x])
    with pytest.raises(ValueError, match="gradient"):
        opt.step([x[:4].clone()], 0.1)
    with pytest.raises(ValueError, match="gradient: expected 1"):
        opt.step([], 0.1)
    with pytest.raises(_lib.LorsError, match="ALIAS"):
        opt.step([x], 0.1)  # the master itself
    with pytest.raises(_lib.LorsError, match="SHAPE"):
        opt.step([x.clone()], float("inf"))
    y = torch.randn(8, 40, device="cuda")
    twice = train.OrthogonalUpdate([y, y], momenta=[torch.zeros_like(y), torch.zeros_like(y)])
    with pytest.raises(_lib.LorsError, match="ALIAS"):
        twice.step([x.clone(), x.clone()], 0.1)
