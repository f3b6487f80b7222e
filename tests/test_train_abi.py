"""CPU tests of the C ABI of the operators around the layer: exports, workspace
queries, and refusals in the documented order.  No call here launches device work:
each is refused on the host (the addresses are made up)."""
import os
import re

import pytest

from paper_2501_08582_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lors_train.h")
BASE, GAP = 1 << 40, 1 << 36
BAD = 2**64 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("liblors.so is not built (python -m paper_2501_08582_amd.build)")
    return _lib.lib()


def ptrs(n):
    return [BASE + i * GAP for i in range(n)]


def make(cls, base, kw):
    d = dict(base)
    d.update(kw)
    rng = d.pop("rng", None)
    p = cls(**d)
    if rng is not None:
        p.rng = rng
    return p


def dropout(**kw):
    return make(_lib.Dropout, dict(rows=8, cols=16, p=0.1, dtype=_lib.DTYPE_BF16), kw)


def norm(**kw):
    return make(_lib.Norm, dict(rows=8, cols=16, eps=1e-5, p=0.1, dtype=_lib.DTYPE_BF16, grad_dtype=_lib.DTYPE_BF16), kw)


def embedding(**kw):
    return make(_lib.Embedding, dict(tokens=8, vocab=100, cols=16, scale=1.0), kw)


def logits(**kw):
    return make(_lib.Logits, dict(batch=2, length=8, vocab=100, batch_stride=800, row_stride=100), kw)


def preference(**kw):
    return make(_lib.Preference, dict(pairs=2, length=8, vocab=100, beta=0.1, smoothing=0.0), kw)


# each entry point with every pointer given; `a` are its pointers in order
def call_dropout(p, a):
    return _lib.dropout(p, *a, None)


def call_norm_forward(p, a):
    return _lib.norm_forward(p, *a, None)


def call_norm_backward(p, a, ws=BASE + 30 * GAP, size=1 << 30):
    return _lib.norm_backward(p, *a, ws, size, None)


def call_embedding_forward(p, a):
    return _lib.embedding_forward(p, *a, None)


def call_embedding_backward(p, a, ws=BASE + 30 * GAP, size=1 << 30):
    return _lib.embedding_backward(p, *a, ws, size, None)


def call_logprob_forward(p, a, ws=BASE + 30 * GAP, size=1 << 30):
    return _lib.logprob_forward(p, *a, ws, size, None)


def call_logprob_backward(p, a, span=1):
    dlogp, up, x, t, stats, out = a
    return _lib.logprob_backward(p, dlogp, span, up, x, t, stats, out, None)


def call_preference(p, a):
    return _lib.preference(p, *a, None)


# (call, descriptor, pointers, the required ones, input and output pairs that must not overlap)
ENTRIES = {
    "dropout": (call_dropout, dropout, 3, [0, 2], [(0, 2), (1, 2)]),
    "norm_forward": (call_norm_forward, norm, 8, [0, 4, 5], [(0, 4), (1, 5), (2, 4), (4, 5), (5, 6), (6, 7)]),
    "norm_backward": (call_norm_backward, norm, 10, [0, 2, 4, 5, 6], [(0, 6), (1, 7), (2, 6), (3, 8), (6, 7), (8, 9)]),
    "embedding_forward": (call_embedding_forward, embedding, 3, [0, 1, 2], [(0, 2), (1, 2)]),
    "embedding_backward": (call_embedding_backward, embedding, 3, [0, 1, 2], [(0, 2), (1, 2)]),
    "logprob_forward": (call_logprob_forward, logits, 4, [0, 1, 2], [(0, 2), (1, 3), (2, 3)]),
    "logprob_backward": (call_logprob_backward, logits, 6, [0, 2, 3, 4, 5], [(0, 5), (1, 5), (2, 5), (3, 5), (4, 5)]),
    "preference": (call_preference, preference, 6, [0, 2, 3, 4, 5], [(0, 3), (1, 4), (2, 5), (3, 4), (4, 5)]),
}


def test_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(lors_[a-z0-9_]+)\s*\(", text))
    assert names == set(_lib.EXPORTED_TRAIN)
    for n in names:
        assert hasattr(lib, n), n
    assert lib.lors_train_version() == 10000


@pytest.mark.parametrize("name", ENTRIES)
def test_null_comes_first(lib, name):
    call, make_p, n, required, _ = ENTRIES[name]
    for k in required:
        a = ptrs(n)
        a[k] = None
        p = make_p()
        if hasattr(p, "dtype"):
            p.dtype = 9
        assert call(p, a) == _lib.ERR_NULL, k


def test_no_descriptor(lib):
    a = ptrs(10)
    assert lib.lors_dropout(None, *a[:3], None) == _lib.ERR_NULL
    assert lib.lors_norm_forward(None, *a[:8], None) == _lib.ERR_NULL
    assert lib.lors_norm_backward(None, *a, None, 0, None) == _lib.ERR_NULL
    assert lib.lors_embedding_forward(None, *a[:3], None) == _lib.ERR_NULL
    assert lib.lors_embedding_backward(None, *a[:3], None, 0, None) == _lib.ERR_NULL
    assert lib.lors_logprob_forward(None, *a[:4], None, 0, None) == _lib.ERR_NULL
    assert lib.lors_logprob_backward(None, a[0], 1, *a[1:6], None) == _lib.ERR_NULL
    assert lib.lors_preference(None, *a[:6], None) == _lib.ERR_NULL
    for query in (lib.lors_norm_workspace_bytes, lib.lors_embedding_workspace_bytes, lib.lors_logprob_workspace_bytes):
        assert query(None) == BAD


@pytest.mark.parametrize("name", ENTRIES)
def test_dtype_before_shape(lib, name):
    call, make_p, n, _, _ = ENTRIES[name]
    p = make_p()
    for field in ("dtype", "grad_dtype", "index_dtype"):
        if hasattr(p, field):
            q = make_p(**{field: 2, "flags": 1})
            assert call(q, ptrs(n)) == _lib.ERR_DTYPE, field
    assert call(make_p(flags=1), ptrs(n)) == _lib.ERR_UNSUPPORTED


@pytest.mark.parametrize("name", ENTRIES)
def test_alignment_and_alias(lib, name):
    call, make_p, n, required, pairs = ENTRIES[name]
    for k in range(n):
        a = ptrs(n)
        a[k] += 1
        assert call(make_p(), a) == _lib.ERR_ALIGN, k
    for i, o in pairs:
        a = ptrs(n)
        a[o] = a[i]
        assert call(make_p(), a) == _lib.ERR_ALIAS, (i, o)


SHAPES = {
    "dropout": [dict(rows=-1), dict(rows=2**31), dict(cols=0), dict(cols=2**31), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")),
                dict(p=1.0 - 2.0**-18), dict(rows=2**31 - 1, cols=2**31 - 1, dtype=_lib.DTYPE_F32)],
    "norm_forward": [dict(rows=-1), dict(rows=2**31), dict(cols=0), dict(cols=32769), dict(eps=-1.0), dict(eps=float("inf")),
                     dict(p=1.5)],
    "embedding_forward": [dict(tokens=-1), dict(tokens=2**31), dict(vocab=0), dict(vocab=2**31), dict(cols=0), dict(cols=2**31),
                          dict(scale=float("nan")), dict(vocab=2**31 - 1, cols=2**31 - 1)],
    "logprob_forward": [dict(batch=-1), dict(length=-1), dict(batch=2**16, length=2**15), dict(vocab=0), dict(vocab=2**31),
                        dict(row_stride=-1), dict(batch_stride=-1), dict(batch_stride=2**60), dict(row_stride=2**62)],
    "preference": [dict(pairs=0), dict(pairs=2**30), dict(length=-1), dict(pairs=2**20, length=2**10), dict(vocab=0),
                   dict(beta=float("inf")), dict(smoothing=-0.1), dict(smoothing=0.6), dict(smoothing=float("nan"))],
}
SHAPES["norm_backward"] = SHAPES["norm_forward"]
SHAPES["embedding_backward"] = SHAPES["embedding_forward"]
SHAPES["logprob_backward"] = SHAPES["logprob_forward"]


@pytest.mark.parametrize("name", ENTRIES)
def test_shapes(lib, name):
    call, make_p, n, _, _ = ENTRIES[name]
    for kw in SHAPES[name]:
        assert call(make_p(**kw), ptrs(n)) == _lib.ERR_SHAPE, kw


def test_other_refusals(lib):
    a = ptrs(8)
    assert call_norm_forward(norm(kind=2), a) == _lib.ERR_UNSUPPORTED
    assert call_norm_backward(norm(kind=-1), ptrs(10)) == _lib.ERR_UNSUPPORTED
    X, res, w, b, Y, Z, mean, rstd = a
    # Z where there is nothing to sum, none where there is
    assert _lib.norm_forward(norm(p=0.0), X, None, w, b, Y, Z, mean, rstd, None) == _lib.ERR_UNSUPPORTED
    assert _lib.norm_forward(norm(p=0.0), X, res, w, b, Y, None, mean, rstd, None) == _lib.ERR_NULL
    # the rms norm has no mean: it may be anything
    dY, dZ, Z, w, mean, rstd, dX, dres, dw, db = ptrs(10)
    assert _lib.norm_backward(norm(kind=1), dY, dZ, Z, w, dX, rstd, dX + 1, dres, dw, db, BASE + 30 * GAP, 1 << 30, None) == \
        _lib.ERR_ALIGN
    assert _lib.norm_backward(norm(), dY, dZ, Z, w, None, rstd, dX, dres, dw, db, BASE + 30 * GAP, 1 << 30, None) == _lib.ERR_NULL
    state = norm(rng=_lib.Rng(1, 2, BASE + 20 * GAP + 4))
    assert call_norm_forward(state, a) == _lib.ERR_ALIGN
    over = dropout(rng=_lib.Rng(1, 2, a[2]))
    assert call_dropout(over, a[:3]) == _lib.ERR_ALIAS
    # the statistics of a row are pairs
    x, t, logp, stats = ptrs(4)
    assert call_logprob_forward(logits(), [x, t, logp, stats + 4]) == _lib.ERR_ALIGN
    # spans that do not divide the tokens
    for span in (0, -1, 3, 9, 16):
        assert call_logprob_backward(logits(), ptrs(6), span) == _lib.ERR_SHAPE
    # more work than the grids can count
    assert call_embedding_backward(embedding(vocab=2**31 - 1, cols=2**16, dtype=0, grad_dtype=0), ptrs(3)) == _lib.ERR_UNSUPPORTED
    assert call_logprob_forward(logits(batch=1, length=2**30, vocab=2**15, row_stride=2**15), ptrs(4)) == _lib.ERR_UNSUPPORTED


def test_workspace(lib):
    # the norm: a partial row of dweight and of dbias per workgroup
    for rows, groups in ((0, 0), (3, 3), (100000, None)):
        n = _lib.norm_workspace_bytes(norm(rows=rows, cols=4096))
        assert n % (8 * 4096) == 0 and (groups is None or n == 8 * 4096 * groups)
        assert n <= 8 * 4096 * 4096
    assert _lib.norm_workspace_bytes(norm(cols=0)) == BAD
    a = ptrs(10)
    need = _lib.norm_workspace_bytes(norm())
    assert call_norm_backward(norm(), a, None, 0) == _lib.ERR_WORKSPACE
    assert call_norm_backward(norm(), a, BASE + 30 * GAP, need - 1) == _lib.ERR_WORKSPACE
    assert call_norm_backward(norm(), a, BASE + 30 * GAP + 8, need) == _lib.ERR_ALIGN
    assert call_norm_backward(norm(), a, a[0], need) == _lib.ERR_ALIAS
    # the embedding: none for a few tokens, then 8 bytes each, an fp32 row for every 32, more beyond what is counted
    assert _lib.embedding_workspace_bytes(embedding(tokens=0)) == 0
    assert _lib.embedding_workspace_bytes(embedding(tokens=256)) == 0
    assert _lib.embedding_workspace_bytes(embedding(tokens=320, cols=1000)) == 2560 + -(-10 * 4000 // 256) * 256
    big = _lib.embedding_workspace_bytes(embedding(tokens=1 << 20, cols=4096))
    assert (1 << 20) * (16 + 4 * 4096 // 32) <= big <= (1 << 20) * (18 + 4 * 4096 // 32)
    assert _lib.embedding_workspace_bytes(embedding(cols=0)) == BAD
    assert call_embedding_backward(embedding(tokens=1000), ptrs(3), None, 0) == _lib.ERR_WORKSPACE
    assert call_embedding_backward(embedding(tokens=1000), ptrs(3), BASE + 2 * GAP, 1 << 20) == _lib.ERR_ALIAS
    # log-probabilities: none where the rows fill the chip
    assert _lib.logprob_workspace_bytes(logits(batch=2, length=4096, vocab=100000, batch_stride=0, row_stride=100000)) == 0
    assert _lib.logprob_workspace_bytes(logits(batch=0)) == 0
    few = logits(batch=1, length=4, vocab=300000, row_stride=300000)
    need = _lib.logprob_workspace_bytes(few)
    assert need > 0 and need % 8 == 0
    assert call_logprob_forward(few, ptrs(4), BASE + 30 * GAP, need - 1) == _lib.ERR_WORKSPACE
    assert call_logprob_forward(few, ptrs(4), BASE + 2 * GAP, need) == _lib.ERR_ALIAS
    assert _lib.logprob_workspace_bytes(logits(vocab=0)) == BAD
