"""Edges of the operators around the layer on the GPU, against their fp64 oracle.
Bounds are those of ``test_gpu_train_ops.check``."""
import numpy as np
import pytest
import torch

from oracle import train as ot
from paper_2501_08582_amd import train
from test_gpu_train_ops import DT, check, f64

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
