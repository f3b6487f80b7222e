"""Steps of the orthogonalised updates whose tensors change between them, on the GPU."""
import numpy as np
import pytest
import torch

from paper_2501_08582_amd import ops, train

pytestmark = pytest.mark.gpu

SHAPES = [(16, 700), (300, 20), (100, 300)]


def tensors(seed=0):
    rng = np.random.default_rng(seed)

    def randn(scale):
        return [torch.from_numpy((scale * rng.standard_normal(s)).astype(np.float32)).cuda() for s in SHAPES]

    grads, momenta, masters = randn(1e-3), randn(1e-3), randn(0.05)
    return grads, momenta, masters, [w.bfloat16() for w in masters]


def test_replaced_tensors_take_the_step_and_the_old_ones_keep_their_values():
    """A restored momentum, a parameter's and a master's new storage: the step of an object made from
    them, bit for bit; what they replaced is left alone."""
    grads, momenta, masters, params = tensors()
    opt = train.OrthogonalUpdate(masters, params, momenta)
    opt.step(grads, 0.02)
    old = [momenta[0], params[1].detach(), masters[2].detach()]
    kept = [t.clone() for t in old]
    opt.momenta[0] = torch.ones_like(old[0]) * 1e-3
    params[1].data = params[1].data.clone()
    masters[2].data = 2.0 * masters[2].data
    twins = [[t.clone() for t in ts] for ts in (opt.masters, opt.params, opt.momenta)]
    opt.step(grads, 0.02)
    train.OrthogonalUpdate(*twins).step(grads, 0.02)
    for got, want in zip((opt.masters, opt.params, opt.momenta), twins):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(old, kept))


def test_a_graph_from_before_a_step_is_refused_after_it():
    """The layer saves its adapters; their step must not give its second backward other ones."""
    W = torch.randn(64, 32, device="cuda").bfloat16()
    M = ops.mask_pack(torch.ones(64, 32, dtype=torch.bool, device="cuda"))
    B, A = (torch.randn(s, device="cuda").bfloat16().requires_grad_(True) for s in ((64, 4), (4, 32)))
    X = torch.randn(8, 32, device="cuda").bfloat16()
    opt = train.OrthogonalUpdate([t.detach().float() for t in (B, A)], [t.detach() for t in (B, A)])
    for call in (lambda: ops.lors_linear(X, W, M, B, A, 2.0), lambda: ops.lors_gated(X, (W, M, B, A), (W, M, B, A), 2.0)):
        out = call().float().sum()
        grads = torch.autograd.grad(out, [B, A], retain_graph=True)
        opt.step(grads, 0.02)
        with pytest.raises(RuntimeError, match="inplace operation"):
            torch.autograd.grad(out, [B, A])
        torch.autograd.grad(call().float().sum(), [B, A])  # a new pass is fine
