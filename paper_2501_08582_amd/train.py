"""PyTorch-facing calls of the operators around the layer in a fine-tuning step.

``dropout``     from a counter-based generator, its mask never stored, fused with
                the residual it is added to
``norm``        residual + dropout(x) and its layer norm or root-mean-square norm
``embedding``   the scaled lookup of token rows
``preference``  log-probabilities of target tokens and the paired preference loss
``orthogonal``  update directions of adapters by Newton-Schulz steps, and the
                optimiser that steps along them
``sample``      tokens drawn from logits: temperature, top-k, top-p, min-p

As in ``ops``, PyTorch supplies device memory and the current HIP stream and
every step runs in ``liblors.so``.  Tensors must live on a ROCm device, be
contiguous (logits: in their last dimension) and be bf16 or fp32; any width is
accepted.  Each operator comes as plain calls (``*_forward``, ``*_backward``) and
as an autograd op.

Dropout masks are a function of ``seed`` and ``offset`` (64-bit integers): calls
that need different masks take different offsets.  ``rng_state``, an int64
tensor of two on the device, is added to both when the kernel runs, so that a
captured graph can advance its masks.
"""
from __future__ import annotations

import ctypes
import math
from operator import attrgetter
from typing import List, Optional, Sequence, Tuple, Union

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from . import _lib
from .ops import _dev, _dt, _ptr

LAYER = "layer"
RMS = "rms"

_KIND = {LAYER: _lib.NORM_LAYER, RMS: _lib.NORM_RMS}
_INDEX = {torch.int64: _lib.INDEX_I64, torch.int32: _lib.INDEX_I32}
_U64 = 2**64 - 1
_INVALID = 2**64 - 1
_current = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


def _call(dev: torch.device, where: str, fn, *args) -> None:
    """``ops._call`` for calls whose kernels take a few microseconds: the caller's
    tensors are on the GPU, so its runtime is up."""
    index = dev.index
    if _current() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(index))
    if status:
        _lib.check(status, where)


def _place(X: torch.Tensor, *ts: Optional[torch.Tensor]) -> torch.device:
    """The device of X, on which the others have to be as well, all contiguous."""
    index = X.get_device()
    fine = index >= 0 and X.is_contiguous()
    for t in ts:
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            fine = False
    return X.device if fine else _dev(X, *ts)  # which says what is wrong


def _kind(kind) -> int:
    try:
        return _KIND[kind]
    except KeyError:
        raise ValueError(f"kind must be {LAYER!r} or {RMS!r}, got {kind!r}")


def _index(t: torch.Tensor, what: str) -> int:
    try:
        return _INDEX[t.dtype]
    except KeyError:
        raise TypeError(f"{what} must be int64 or int32, got {t.dtype}")


def _like(X: torch.Tensor, what: str, *ts: Optional[torch.Tensor]) -> None:
    """Tensors that must have X's shape and dtype."""
    for t in ts:
        if t is not None and (t.shape != X.shape or t.dtype != X.dtype):
            raise ValueError(f"{what}: expected {tuple(X.shape)} of {X.dtype}, got {tuple(t.shape)} of {t.dtype}")


def _vector(X: torch.Tensor, what: str, t: Optional[torch.Tensor], dtype=None) -> None:
    """A vector as long as X's rows."""
    if t is not None and (t.dim() != 1 or t.shape[0] != X.shape[-1] or t.dtype != (dtype or X.dtype)):
        raise ValueError(f"{what}: expected ({X.shape[-1]},) of {dtype or X.dtype}, got {tuple(t.shape)} of {t.dtype}")


def _extents(X: torch.Tensor) -> Tuple[int, int]:
    """Rows and columns of X with its leading dimensions flattened to one."""
    if X.dim() == 0 or X.shape[-1] == 0:
        raise ValueError("expected a last dimension of at least one element")
    cols = X.shape[-1]
    return X.numel() // cols, cols


def _drops(p: float) -> bool:
    """Whether p, rounded to 2^-16 as the library does, drops anything."""
    return not p * 65536.0 + 0.5 < 1.0


_NO_RNG = _lib.Rng(0, 0, None)  # a descriptor takes a copy


def _rng(p: float, seed: int, offset: int, state: Optional[torch.Tensor]) -> _lib.Rng:
    if p == 0.0:
        return _NO_RNG
    if state is not None and (state.dtype != torch.int64 or state.numel() != 2):
        raise ValueError("rng_state must be two int64")
    return _lib.Rng(int(seed) & _U64, int(offset) & _U64, _ptr(state))


def _workspace(need: int, dev: torch.device) -> Optional[torch.Tensor]:
    if need == _INVALID:
        raise ValueError("invalid problem")
    return torch.empty(need, dtype=torch.uint8, device=dev) if need else None


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
def dropout(X: torch.Tensor, p: float, seed: int, offset: int = 0, residual: Optional[torch.Tensor] = None,
            rng_state: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dropout(X) (+ residual).  ``p`` is applied as the nearest multiple of 2^-16,
    and kept elements are divided by 1 minus that.  The gradient of X is the same call on
    dY without the residual (``dropout_add`` does that under autograd)."""
    dev = _place(X, residual, rng_state, out)
    rows, cols = _extents(X)
    _like(X, "residual", residual)
    _like(X, "out", out)
    d = _lib.Dropout(rows, cols, p, _rng(p, seed, offset, rng_state), _dt(X), 0)
    if out is None:
        out = torch.empty_like(X)
    _call(dev, "lors_dropout", _lib.dropout, d, X.data_ptr(), _ptr(residual), out.data_ptr())
    return out


class DropoutAddFn(torch.autograd.Function):
    """residual + dropout(X); saves nothing but the seed."""

    @staticmethod
    def forward(ctx, X, residual, p, seed, offset, rng_state):
        ctx.args = (p, seed, offset)
        ctx.save_for_backward(rng_state)
        return dropout(X, p, seed, offset, residual, rng_state)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        p, seed, offset = ctx.args
        (rng_state,) = ctx.saved_tensors
        dX = dropout(dY.contiguous(), p, seed, offset, rng_state=rng_state) if ctx.needs_input_grad[0] else None
        return dX, dY if ctx.needs_input_grad[1] else None, None, None, None, None


def dropout_add(X, p, seed, offset=0, residual=None, rng_state=None):
    """dropout(X) (+ residual) with autograd."""
    return DropoutAddFn.apply(X, residual, p, seed, offset, rng_state)


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
def norm_forward(X: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, kind: str = LAYER, residual: Optional[torch.Tensor] = None, p: float = 0.0,
                 seed: int = 0, offset: int = 0, rng_state: Optional[torch.Tensor] = None, need_stats: bool = True):
    """(Y, Z, mean, rstd): Z = residual + dropout(X) in X's dtype (X itself without
    residual and dropout), Y its norm over the last dimension: ``layer``, (Z - mean) rstd
    weight + bias, or ``rms``, Z rstd weight + bias.  mean (None for ``rms``) and rstd are what
    ``norm_backward`` needs; ``need_stats=False`` leaves them out."""
    dev = _place(X, weight, bias, residual, rng_state)
    rows, cols = _extents(X)
    _like(X, "residual", residual)
    _vector(X, "weight", weight)
    _vector(X, "bias", bias)
    k, dt = _kind(kind), _dt(X)
    d = _lib.Norm(rows, cols, eps, p, _rng(p, seed, offset, rng_state), dt, dt, k, 0)
    Y = torch.empty_like(X)
    Z = torch.empty_like(X) if residual is not None or _drops(p) else None
    rstd = torch.empty(X.shape[:-1], dtype=torch.float32, device=dev) if need_stats else None
    mean = torch.empty_like(rstd) if need_stats and k == _lib.NORM_LAYER else None
    _call(dev, "lors_norm_forward", _lib.norm_forward, d, X.data_ptr(), _ptr(residual), _ptr(weight), _ptr(bias),
          Y.data_ptr(), _ptr(Z), _ptr(mean), _ptr(rstd))
    return Y, X if Z is None else Z, mean, rstd


def norm_backward(dY: torch.Tensor, Z: torch.Tensor, weight: Optional[torch.Tensor], mean: Optional[torch.Tensor],
                  rstd: torch.Tensor, kind: str = LAYER, dZ: Optional[torch.Tensor] = None, p: float = 0.0,
                  seed: int = 0, offset: int = 0, rng_state: Optional[torch.Tensor] = None,
                  need_dresidual: bool = False, need_dweight: Optional[bool] = None, need_dbias: bool = False,
                  grad_dtype: Optional[torch.dtype] = None):
    """(dX, dresidual, dweight, dbias) from the gradient of Y and, if Z is used
    elsewhere, its gradient ``dZ`` from there.  dweight (by default where there is a
    weight) and dbias are in ``grad_dtype``, by default Z's.  Without dropout dresidual
    is dX."""
    dev = _place(dY, Z, weight, mean, rstd, dZ, rng_state)
    rows, cols = _extents(Z)
    _like(Z, "dY, dZ", dY, dZ)
    _vector(Z, "weight", weight)
    k, dt = _kind(kind), _dt(Z)
    gdt = grad_dtype or Z.dtype
    if gdt not in (torch.bfloat16, torch.float32):
        raise TypeError(f"dtype {gdt} not supported (bf16 or fp32)")
    for what, t in (("mean", mean if k == _lib.NORM_LAYER else None), ("rstd", rstd)):
        if t is not None and (t.dtype != torch.float32 or t.numel() != rows):
            raise ValueError(f"{what} must be {rows} fp32")
    if k == _lib.NORM_LAYER and mean is None:
        raise ValueError("the layer norm's gradient needs its mean")
    if need_dweight is None:
        need_dweight = weight is not None
    d = _lib.Norm(rows, cols, 0.0, p, _rng(p, seed, offset, rng_state), dt, _lib.DTYPE_BF16 if gdt == torch.bfloat16 else
                  _lib.DTYPE_F32, k, 0)
    dX = torch.empty_like(Z)
    dres = torch.empty_like(Z) if need_dresidual and _drops(p) else None
    dweight = torch.empty(cols, dtype=gdt, device=dev) if need_dweight else None
    dbias = torch.empty(cols, dtype=gdt, device=dev) if need_dbias else None
    need = _lib.norm_workspace_bytes(d) if need_dweight or need_dbias else 0
    ws = _workspace(need, dev)
    _call(dev, "lors_norm_backward", _lib.norm_backward, d, _ptr(dY), _ptr(dZ), _ptr(Z), _ptr(weight), _ptr(mean),
          _ptr(rstd), _ptr(dX), _ptr(dres), _ptr(dweight), _ptr(dbias), _ptr(ws), need)
    return dX, dX if need_dresidual and dres is None else dres, dweight, dbias


class NormFn(torch.autograd.Function):
    """(Y, Z); saves Z and the statistics of its rows, no mask."""

    @staticmethod
    def forward(ctx, X, weight, bias, residual, eps, kind, p, seed, offset, rng_state):
        Y, Z, mean, rstd = norm_forward(X, weight, bias, eps, kind, residual, p, seed, offset, rng_state)
        ctx.args = (kind, p, seed, offset)
        ctx.has_bias = bias is not None
        ctx.own_z = Z is not X
        ctx.save_for_backward(Z, weight, mean, rstd, rng_state)
        ctx.set_materialize_grads(False)
        return Y, Z if ctx.own_z else X.view_as(X)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY, dZ):
        kind, p, seed, offset = ctx.args
        Z, weight, mean, rstd, rng_state = ctx.saved_tensors
        needs = ctx.needs_input_grad
        dY = torch.zeros_like(Z) if dY is None else dY.contiguous()
        dX, dres, dweight, dbias = norm_backward(
            dY, Z, weight, mean, rstd, kind, None if dZ is None else dZ.contiguous(), p, seed, offset, rng_state,
            need_dresidual=needs[3], need_dweight=weight is not None and needs[1], need_dbias=ctx.has_bias and needs[2])
        return dX, dweight, dbias, dres, None, None, None, None, None, None


def norm(X, weight=None, bias=None, eps=1e-5, kind=LAYER, residual=None, p=0.0, seed=0, offset=0, rng_state=None):
    """(Y, Z) of ``norm_forward`` with autograd: Z is the residual stream after the
    sum, Y the norm of it that the next projection reads."""
    return NormFn.apply(X, weight, bias, residual, eps, kind, p, seed, offset, rng_state)


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def _embedding(ids, vocab, cols, scale, dtype, grad_dtype) -> _lib.Embedding:
    return _lib.Embedding(ids.numel(), vocab, cols, scale, dtype, grad_dtype, _index(ids, "ids"), 0)


def embedding_forward(ids: torch.Tensor, E: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """scale * E[ids], with a trailing dimension of E's width.  Ids outside the table
    (padding, e.g. -1) give rows of zeros."""
    dev = _place(ids, E)
    if E.dim() != 2:
        raise ValueError("the table must be vocab x width")
    vocab, cols = E.shape
    dt = _dt(E)
    d = _embedding(ids, vocab, cols, scale, dt, dt)
    Y = E.new_empty((*ids.shape, cols))
    _call(dev, "lors_embedding_forward", _lib.embedding_forward, d, _ptr(ids), _ptr(E), _ptr(Y))
    return Y


def embedding_backward(dY: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0,
                       grad_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The gradient of the whole table (vocab x width) in ``grad_dtype``, by default
    dY's: sums in fp32 over the tokens in their order, rounded once."""
    dev = _place(dY, ids)
    rows, cols = _extents(dY)
    if rows != ids.numel():
        raise ValueError(f"dY has {rows} rows for {ids.numel()} ids")
    gdt = grad_dtype or dY.dtype
    if gdt not in (torch.bfloat16, torch.float32):
        raise TypeError(f"dtype {gdt} not supported (bf16 or fp32)")
    d = _embedding(ids, vocab, cols, scale, _dt(dY), _lib.DTYPE_BF16 if gdt == torch.bfloat16 else _lib.DTYPE_F32)
    need = _lib.embedding_workspace_bytes(d)
    ws = _workspace(need, dev)
    dE = torch.empty((vocab, cols), dtype=gdt, device=dev)
    _call(dev, "lors_embedding_backward", _lib.embedding_backward, d, _ptr(ids), _ptr(dY), _ptr(dE), _ptr(ws), need)
    return dE


class EmbeddingFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, E, scale):
        ctx.vocab, ctx.scale = E.shape[0], scale
        ctx.save_for_backward(ids)
        return embedding_forward(ids, E, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        (ids,) = ctx.saved_tensors
        return None, embedding_backward(dY.contiguous(), ids, ctx.vocab, ctx.scale), None


def embedding(ids, E, scale=1.0):
    """``embedding_forward`` with autograd."""
    return EmbeddingFn.apply(ids, E, scale)


# ---------------------------------------------------------------------------
# preference
# ---------------------------------------------------------------------------
def _logits(logits: torch.Tensor, targets: torch.Tensor):
    """Descriptor and device of logits (batch x length x vocab, or rows x vocab) whose last
    dimension is contiguous, with targets of the leading dimensions."""
    if not logits.is_cuda:
        raise ValueError("all tensors must be on the GPU")
    if logits.dim() not in (2, 3) or targets.shape != logits.shape[:-1]:
        raise ValueError("logits must be (batch x) length x vocab, targets (batch x) length")
    if logits.stride(-1) != 1 and logits.shape[-1] > 1:
        raise ValueError("logits must be contiguous in their last dimension")
    dev = _place(targets)
    if dev != logits.device:
        raise ValueError("all tensors must be on the same device")
    batch, bs = (1, 0) if logits.dim() == 2 else (logits.shape[0], logits.stride(0))
    return _lib.Logits(batch, logits.shape[-2], logits.shape[-1], bs, logits.stride(-2), _dt(logits),
                       _index(targets, "targets"), 0), dev


def _fp32(shape, what: str, *ts: Optional[torch.Tensor]) -> None:
    for t in ts:
        if t is not None and (t.shape != shape or t.dtype != torch.float32):
            raise ValueError(f"{what}: expected {tuple(shape)} of fp32, got {tuple(t.shape)} of {t.dtype}")


def logprob_forward(logits: torch.Tensor, targets: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(logp, stats): log softmax(logits) at the targets, fp32 of their shape, and with
    a trailing dimension of two the row's largest logit and its sum of exp(logits - it), which
    ``logprob_backward`` needs.  A target outside the vocabulary (-100) does not count:
    its results are 0 and its logits are not read."""
    d, dev = _logits(logits, targets)
    return _logprob_forward(d, dev, logits, targets)


def _logprob_forward(d: _lib.Logits, dev: torch.device, logits, targets):
    logp = torch.empty(targets.shape, dtype=torch.float32, device=dev)
    stats = logp.new_empty((*targets.shape, 2))
    need = _lib.logprob_workspace_bytes(d)
    ws = _workspace(need, dev)
    _call(dev, "lors_logprob_forward", _lib.logprob_forward, d, _ptr(logits), _ptr(targets), _ptr(logp), _ptr(stats),
          _ptr(ws), need)
    return logp, stats


def logprob_backward(dlogp: torch.Tensor, logits: torch.Tensor, targets: torch.Tensor, stats: torch.Tensor,
                     upstream: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of the logits, contiguous in their dtype, from that of the
    log-probabilities: one for each token (the targets' shape) or one for each sequence
    (batch), times the scalar ``upstream``."""
    d, dev = _logits(logits, targets)
    if _place(dlogp, stats, upstream) != dev:
        raise ValueError("all tensors must be on the same device")
    _fp32((*targets.shape, 2), "stats", stats)
    span = 1
    if dlogp.dim() == targets.dim() - 1 and dlogp.shape == targets.shape[:-1]:
        _fp32(dlogp.shape, "dlogp", dlogp)
        span = max(1, targets.shape[-1])
    else:
        _fp32(targets.shape, "dlogp", dlogp)
    if upstream is not None and (upstream.numel() != 1 or upstream.dtype != torch.float32):
        raise ValueError("upstream must be one fp32")
    return _logprob_backward(d, dev, dlogp, span, upstream, logits, targets, stats)


def _logprob_backward(d: _lib.Logits, dev: torch.device, dlogp, span, upstream, logits, targets, stats):
    dlogits = logits.new_empty(logits.shape)
    _call(dev, "lors_logprob_backward", _lib.logprob_backward, d, _ptr(dlogp), span, _ptr(upstream), _ptr(logits),
          _ptr(targets), _ptr(stats), _ptr(dlogits))
    return dlogits


class TokenLogprobsFn(torch.autograd.Function):
    """Saves the logits and two fp32 a token."""

    @staticmethod
    def forward(ctx, logits, targets):
        logp, stats = logprob_forward(logits, targets)
        ctx.save_for_backward(logits, targets, stats)
        return logp

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp):
        logits, targets, stats = ctx.saved_tensors
        return logprob_backward(dlogp.contiguous(), logits, targets, stats), None


def token_logprobs(logits, targets):
    """Log-probabilities of the targets, with autograd."""
    return TokenLogprobsFn.apply(logits, targets)


def preference_forward(logp: torch.Tensor, targets: torch.Tensor, vocab: int, ref: Optional[torch.Tensor] = None,
                       beta: float = 0.1, smoothing: float = 0.0):
    """(loss, reward, dseq) of 2 P sequences of log-probabilities, the P preferred
    ones first: reward = beta * sum over counted tokens of (logp - ref), loss the mean over pairs
    of -(1 - smoothing) log sigmoid(m) - smoothing log sigmoid(-m) with m the pair's difference of
    rewards, dseq the loss's gradient by each sequence's summed log-probability."""
    return _preference_forward(logp, targets, vocab, ref, beta, smoothing, shared=True)


def _preference_forward(logp, targets, vocab, ref, beta, smoothing, shared: bool):
    """``shared``: the results are views of one allocation.  Autograd takes none of those
    for the outputs of an op that a program may change in place."""
    dev = _place(logp, targets, ref)
    if logp.dim() != 2 or logp.shape[0] % 2 != 0:
        raise ValueError("expected 2 P x length: the preferred sequences, then the rejected ones")
    _fp32(targets.shape, "logp, ref", logp, ref)
    P = logp.shape[0] // 2
    d = _lib.Preference(P, logp.shape[1], vocab, beta, smoothing, _index(targets, "targets"), 0)
    if shared:
        out = torch.empty(4 * P + 1, dtype=torch.float32, device=dev)
        reward, dseq, loss = out.split((2 * P, 2 * P, 1))
        loss, at = loss.view(()), out.data_ptr()
        places = at + 16 * P, at, at + 8 * P
    else:
        loss, reward, dseq = (torch.empty(n, dtype=torch.float32, device=dev) for n in ((), 2 * P, 2 * P))
        places = _ptr(loss), _ptr(reward), _ptr(dseq)
    _call(dev, "lors_preference", _lib.preference, d, _ptr(logp), _ptr(ref), _ptr(targets), *places)
    return loss, reward, dseq


def preference_step(logits: torch.Tensor, targets: torch.Tensor, ref: Optional[torch.Tensor] = None,
                    beta: float = 0.1, smoothing: float = 0.0):
    """(loss, reward, logp, dlogits) of one training step's loss on logits 2 P x length
    x vocab: forward and gradient together, for loops without autograd."""
    d, dev = _logits(logits, targets)
    logp, stats = _logprob_forward(d, dev, logits, targets)
    loss, reward, dseq = preference_forward(logp, targets, logits.shape[-1], ref, beta, smoothing)
    span = max(1, logits.shape[-2])
    return loss, reward, logp, _logprob_backward(d, dev, dseq, span, None, logits, targets, stats)


class PreferenceLossFn(torch.autograd.Function):
    """(loss, reward, logp); saves the logits, two fp32 a token and one a sequence."""

    @staticmethod
    def forward(ctx, logits, targets, ref, beta, smoothing):
        logp, stats = logprob_forward(logits, targets)
        loss, reward, dseq = _preference_forward(logp, targets, logits.shape[-1], ref, beta, smoothing, shared=False)
        ctx.save_for_backward(logits, targets, stats, dseq)
        ctx.mark_non_differentiable(reward, logp)
        return loss, reward, logp

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss, _dreward, _dlogp):
        logits, targets, stats, dseq = ctx.saved_tensors
        return logprob_backward(dseq, logits, targets, stats, dloss.contiguous()), None, None, None, None


def preference_loss(logits, targets, ref=None, beta=0.1, smoothing=0.0):
    """(loss, reward, logp) with autograd: gradients flow from the loss alone."""
    return PreferenceLossFn.apply(logits, targets, ref, beta, smoothing)


# ---------------------------------------------------------------------------
# orthogonalised updates
# ---------------------------------------------------------------------------
COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # of the steps: singular values of 0.002 to 1 end between 0.7 and 1.2


def _update(momentum, nesterov, coefficients, steps, eps, grad, param) -> _lib.Update:
    a, b, c = coefficients
    return _lib.Update(momentum, eps, a, b, c, steps, int(bool(nesterov)), _dt(grad), _dt(param), 0)


_shape, _dtype = attrgetter("shape"), attrgetter("dtype")


def _matrices(what: str, ts: Sequence[torch.Tensor], shapes: Optional[Sequence[torch.Size]] = None,
              dtype: Optional[torch.dtype] = None) -> None:
    """Contiguous matrices of one device and type, of the given shapes."""
    if shapes is not None and len(ts) != len(shapes):
        raise ValueError(f"{what}: expected {len(shapes)} matrices, got {len(ts)}")
    dtype = dtype or ts[0].dtype
    index = ts[0].get_device()
    # all at once, 0.4 us a matrix where the loop below takes 0.9
    if (index >= 0 and (all(n == 2 for n in map(torch.Tensor.dim, ts)) if shapes is None else list(map(_shape, ts)) == shapes)
            and set(map(_dtype, ts)) == {dtype} and set(map(torch.Tensor.get_device, ts)) == {index}
            and all(map(torch.Tensor.is_contiguous, ts))):
        return
    for i, t in enumerate(ts):
        if t.dim() != 2 or t.dtype != dtype or (shapes is not None and t.shape != shapes[i]):
            shape = tuple(shapes[i]) if shapes is not None else "a matrix"
            raise ValueError(f"{what} {i}: expected {shape} of {dtype}, got {tuple(t.shape)} of {t.dtype}")
        if t.get_device() != index or index < 0 or not t.is_contiguous():
            _dev(ts[0], t)  # which says what is wrong


def _addresses(ts: Sequence[torch.Tensor]) -> List[int]:
    return list(map(torch.Tensor.data_ptr, ts))


def _run_update(p: _lib.Update, items, count: int, ws: Optional[torch.Tensor], dev: torch.device) -> None:
    _call(dev, "lors_orthogonal_update", _lib.orthogonal_update, p, items, count, _ptr(ws), 0 if ws is None else ws.numel())


def orthogonalize(X: Union[torch.Tensor, Sequence[torch.Tensor]], steps: int = 5,
                  coefficients: Tuple[float, float, float] = COEFFICIENTS, eps: float = 1e-7):
    """The Newton-Schulz direction of a matrix, or of each of a list (as a list): x = X / (|X| + eps), then
    ``steps`` times x <- a x + (b S + c S^2) x with S = x x^T on the shorter side, of at
    most 128.  With the default steps every singular value above a fivehundredth of |X| comes near 1.
    X's dtype; 64-bit steps, one rounding."""
    one = isinstance(X, torch.Tensor)
    Xs = [X] if one else list(X)
    if not Xs:
        return []
    _matrices("matrix", Xs)
    dev = _dev(Xs[0])
    out = [torch.empty_like(t) for t in Xs]
    p = _update(0.0, False, coefficients, steps, eps, Xs[0], Xs[0])
    items = (_lib.UpdateItem * len(Xs))(*((*t.shape, t.data_ptr(), None, None, o.data_ptr(), 1.0, 0.0) for t, o in zip(Xs, out)))
    live = [i for i, t in enumerate(Xs) if t.numel()]
    if len(live) < len(Xs):  # matrices of no elements have nothing to do
        items = (_lib.UpdateItem * len(live))(*(items[i] for i in live))
    if live:
        ws = _workspace(_lib.orthogonal_workspace_bytes(p, items, len(live)), dev)
        _run_update(p, items, len(live), ws, dev)
    return out[0] if one else out


class OrthogonalUpdate:
    """An optimiser of matrices with a short side (adapters: R x r, r x C; the shorter side is at most 128).  Of each matrix,

        m      <- momentum . m + (1 - momentum) . grad
        v       = momentum . m + (1 - momentum) . grad  (Nesterov), or m
        master <- (1 - lr . weight_decay) . master - lr . sqrt(max(1, rows / cols)) . direction(v)
        param   = master in the parameter's type

    with the direction of ``orthogonalize``.  ``masters`` and ``momenta`` are fp32 (momenta: zeros if
    not given) and changed in place, for autograd too; ``params``, of one type, receive the masters' values and may be
    left out, or be the masters themselves where they are fp32.  The three lists are the object's to read and
    the caller's to change: a step works on the tensors that they hold then, wherever those
    stand by then (a restored momentum, ``p.data = ...``), of the shapes and types of the first.
    A step is one call, whatever the count: its launches are a few for each size of the
    short side (up to 16, 32, 48, 64, 96, 128).  ``step`` may be captured into a graph, with the lr and the
    tensors of that call; its scratch memory belongs to the object, which the graph must not outlive, and steps of
    one object must not overlap."""

    def __init__(self, masters: Sequence[torch.Tensor], params: Optional[Sequence[torch.Tensor]] = None,
                 momenta: Optional[Sequence[torch.Tensor]] = None, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, steps: int = 5, coefficients: Tuple[float, float, float] = COEFFICIENTS,
                 eps: float = 1e-7):
        self.masters: List[torch.Tensor] = list(masters)
        if not self.masters:
            raise ValueError("no matrices")
        self.momenta = [torch.zeros_like(t) for t in self.masters] if momenta is None else list(momenta)
        self.params = None if params is None else list(params)
        self.weight_decay = float(weight_decay)
        self._rule = (momentum, nesterov, coefficients, steps, eps)
        _matrices("master", self.masters, dtype=torch.float32)
        self._shapes = [t.shape for t in self.masters]
        self._device = _dev(self.masters[0])
        self._param_dtype = torch.float32 if not self.params else self.params[0].dtype
        self._items = (_lib.UpdateItem * len(self.masters))()
        self._grads = np.ndarray((len(self.masters),), np.uint64, self._items, _lib.UpdateItem.grad.offset,
                                 (ctypes.sizeof(_lib.UpdateItem),))  # their grad fields, all of which a step sets
        self._bind()
        p = self._descriptor(self.masters[0])
        self._ws = _workspace(_lib.orthogonal_workspace_bytes(p, self._items, len(self.masters)), self._device)
        self._stream = _raw_stream(self._device.index)  # whose memory the workspace is
        self._shape_rate = [math.sqrt(max(1.0, rows / cols)) for rows, cols in self._shapes]
        self._rates: Optional[Tuple[float, float]] = None  # the lr and weight decay that the items hold

    def _kept(self) -> List[torch.Tensor]:
        return [*self.masters, *self.momenta, *(self.params or ())]

    def _bind(self) -> None:
        """Takes the addresses of the tensors that the lists hold now."""
        _matrices("master", self.masters, self._shapes, torch.float32)
        _matrices("momentum", self.momenta, self._shapes, torch.float32)
        if self.params is not None:
            _matrices("param", self.params, self._shapes, self._param_dtype)
        kept, n = self._kept(), len(self.masters)
        at = _addresses(kept)
        for t, where in zip(kept, at):
            if t.device != self._device:
                raise ValueError("all tensors must be on the same device")
            if where == 0 and t.numel():
                raise ValueError("a tensor's storage has been released")
        for i, (item, (rows, cols), w, m) in enumerate(zip(self._items, self._shapes, at, at[n:])):
            q = at[2 * n + i] if self.params is not None else 0
            if q == w and self._param_dtype == torch.float32:  # an fp32 parameter may be its own master
                q = 0
            item.rows, item.cols, item.m, item.master, item.param = rows, cols, m, w, q or None
            item.grad = w  # (of the workspace query; step sets it)
        # what stands at these addresses stays there until others are taken, so that an address that
        # is still the same is the same memory
        self._held, self._at = [t.detach() for t in kept], at

    def _descriptor(self, grad: torch.Tensor) -> _lib.Update:
        return _update(*self._rule, grad, self.masters[0] if self.params is None else self.params[0])

    def step(self, grads: Sequence[torch.Tensor], lr: float) -> None:
        """One step along the gradients (of the masters' shapes; all bf16 or all fp32), at the lr and the
        ``weight_decay`` of the moment."""
        grads = list(grads)
        _matrices("gradient", grads, self._shapes)
        if grads[0].device != self._device:
            raise ValueError("all tensors must be on the same device")
        if _addresses(self._kept()) != self._at:
            self._bind()
        items = self._items
        rates = (float(lr), float(self.weight_decay))
        if rates != self._rates:
            lr, decay = rates[0], rates[0] * rates[1]
            for item, rate in zip(items, self._shape_rate):
                item.rate, item.decay = lr * rate, decay
            self._rates = rates
        self._grads[:] = _addresses(grads)
        if _raw_stream(self._device.index) != self._stream and not torch.cuda.is_current_stream_capturing():
            self._ws.record_stream(torch.cuda.current_stream(self._device))
        _run_update(self._descriptor(grads[0]), items, len(grads), self._ws, self._device)
        # autograd has to know: a graph that saved one of them must not be passed again
        torch.autograd.graph.increment_version(self._kept())


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def _per_row(value, what: str, shape, dtype: torch.dtype, dev: torch.device):
    """(scalar, tensor or None) of a parameter that is one number or one a row."""
    if not isinstance(value, torch.Tensor):
        return value, None
    if value.shape != shape or value.dtype != dtype:
        raise ValueError(f"{what}: expected {tuple(shape)} of {dtype}, got {tuple(value.shape)} of {value.dtype}")
    if _dev(value) != dev:
        raise ValueError("all tensors must be on the same device")
    return 0, value


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: Union[float, torch.Tensor] = 1.0,
           top_k: Union[int, torch.Tensor] = 0, top_p: Union[float, torch.Tensor] = 1.0,
           min_p: Union[float, torch.Tensor] = 0.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """(token, logp): a token of each row of logits (... x vocab, contiguous in the last dimension;
    rows of a matrix may be strided), int64, and the log of its probability among what is kept, fp32.
    Entries are ordered by logit, equal ones by index.  top_k keeps the first top_k of them (0: all), top_p the
    shortest run of those that holds top_p of their probability (1: all), min_p those of at least
    min_p times the largest probability; the first is always kept.  The token is the first kept one, by
    index, at which the running sum of probabilities exceeds u (fp32 in [0, 1), one a row) times their
    whole.  temperature 0: the first.  Each parameter may be a tensor of one value a row (fp32; top_k
    int32).  A row with a NaN or +Inf, or of -Inf alone, gives token -1 and logp NaN."""
    if not logits.is_cuda:
        raise ValueError("all tensors must be on the GPU")
    if logits.dim() == 0 or logits.shape[-1] == 0:
        raise ValueError("expected a last dimension of at least one element")
    shape, vocab = logits.shape[:-1], logits.shape[-1]
    if logits.stride(-1) != 1 and vocab > 1:
        raise ValueError("logits must be contiguous in their last dimension")
    if logits.dim() == 2:
        stride = logits.stride(0)
    elif logits.is_contiguous():
        stride = vocab
    else:
        raise ValueError("logits must be contiguous, or a matrix with strided rows")
    _fp32(shape, "u", u)
    dev = _place(u)
    if dev != logits.device:
        raise ValueError("all tensors must be on the same device")
    T, Ts = _per_row(temperature, "temperature", shape, torch.float32, dev)
    k, ks = _per_row(top_k, "top_k", shape, torch.int32, dev)
    p, ps = _per_row(top_p, "top_p", shape, torch.float32, dev)
    low, lows = _per_row(min_p, "min_p", shape, torch.float32, dev)
    d = _lib.Sample(u.numel(), vocab, stride, T, k, p, low, _dt(logits), 0)
    token = torch.empty(shape, dtype=torch.int64, device=dev)
    logp = torch.empty(shape, dtype=torch.float32, device=dev)
    need = _lib.sample_workspace_bytes(d)
    ws = _workspace(need, dev)
    _call(dev, "lors_sample", _lib.sample, d, logits.data_ptr(), u.data_ptr(), _ptr(Ts), _ptr(ks), _ptr(ps), _ptr(lows),
          token.data_ptr(), logp.data_ptr(), _ptr(ws), need)
    return token, logp
