"""PyTorch-facing calls of the operators around the layer in a fine-tuning step.

``dropout``     from a counter-based generator, its mask never stored, fused with
                the residual it is added to
``norm``        residual + dropout(x) and its layer norm or root-mean-square norm
``embedding``   the scaled lookup of token rows
``preference``  log-probabilities of target tokens and the paired preference loss

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

from typing import Optional, Tuple

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
