"""CPU tests of the C ABI of the gated block, the orthogonalised updates and the
sampling: exports, workspace queries, and refusals in the documented order.  No call
here launches device work: each is refused on the host (the addresses are made up), or
has nothing to do."""
import os
import re

import pytest

from paper_2501_08582_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lors_block.h")
BASE, GAP = 1 << 40, 1 << 36
BAD = 2**64 - 1
WS = BASE + 100 * GAP
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("liblors.so is not built (python -m paper_2501_08582_amd.build)")
    return _lib.lib()


def at(i):
    return BASE + i * GAP


def test_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(lors_[a-z0-9_]+)\s*\(", text))
    assert names == set(_lib.EXPORTED_BLOCK)
    for n in names:
        assert hasattr(lib, n), n
    assert lib.lors_block_version() == 10000


# ---------------------------------------------------------------------------
# gated
# ---------------------------------------------------------------------------
def problem(R=64, C=32, L=8, r=4, scale=2.0, dtype=_lib.DTYPE_BF16, fmt=_lib.MASK_BITMAP, flags=0):
    p = _lib.problem(R, C, L, r, scale, dtype, fmt)
    p.flags = flags
    return p


class Gated:
    """Arguments of both calls, by name; None drops one."""

    def __init__(self, **over):
        self.v = {n: at(i) for i, n in enumerate(
            ("X", "Wg", "Mg", "Bg", "Ag", "Wu", "Mu", "Bu", "Au", "G", "U", "H", "dH", "dX", "dBg", "dAg", "dBu", "dAu"))}
        self.v.update(ws=WS, size=1 << 40)
        self.v.update(over)

    def forward(self, p, act=0):
        v = self.v
        return _lib.gated_forward(p, act, v["X"], _lib.Projection(v["Wg"], v["Mg"], v["Bg"], v["Ag"]),
                                  _lib.Projection(v["Wu"], v["Mu"], v["Bu"], v["Au"]), v["G"], v["U"], v["H"], v["ws"], v["size"], None)

    def backward(self, p, act=0):
        v = self.v
        return _lib.gated_backward(p, act, v["dH"], v["X"], _lib.Projection(v["Wg"], v["Mg"], v["Bg"], v["Ag"]),
                                   _lib.Projection(v["Wu"], v["Mu"], v["Bu"], v["Au"]), v["G"], v["U"], v["dX"], v["dBg"], v["dAg"],
                                   v["dBu"], v["dAu"], v["ws"], v["size"], None)


FORWARD_IN = ("X", "Wg", "Mg", "Bg", "Ag", "Wu", "Mu", "Bu", "Au")
BACKWARD_IN = FORWARD_IN + ("dH", "G", "U")
BACKWARD_OUT = ("dX", "dBg", "dAg", "dBu", "dAu")


def test_gated_null_comes_first():
    broken = problem(dtype=7, R=-1)
    for n in FORWARD_IN + ("H", "G", "U"):  # G and U: both or neither
        assert Gated(**{n: None}).forward(broken) == _lib.ERR_NULL, n
    for n in BACKWARD_IN + BACKWARD_OUT[1:]:
        assert Gated(**{n: None}).backward(broken) == _lib.ERR_NULL, n
    for n in ("G", "U", "dX"):
        assert Gated(**({"G": None, "U": None} if n != "dX" else {n: None})).forward(broken) == _lib.ERR_DTYPE
    assert Gated(dX=None).backward(broken) == _lib.ERR_DTYPE


@pytest.mark.parametrize("call", ["forward", "backward"])
def test_gated_refusals_in_order(call):
    g = Gated(X=at(0) + 8)  # misaligned too: every range comes before it

    def run(act=0, **kw):
        return getattr(g, call)(problem(**kw), act)

    assert run(dtype=2, fmt=9, R=-1) == _lib.ERR_DTYPE
    assert run(fmt=9, R=-1) == _lib.ERR_MASK_FORMAT
    assert run(act=2, R=-1) == _lib.ERR_UNSUPPORTED
    assert run(act=-1, R=-1) == _lib.ERR_UNSUPPORTED
    for wrong in (dict(R=0), dict(C=0), dict(L=-1), dict(r=0), dict(r=129), dict(R=1 << 31), dict(scale=NAN), dict(scale=INF),
                  dict(R=(1 << 31) - 8, C=8, L=(1 << 31) - 1)):
        assert run(**wrong) == _lib.ERR_SHAPE, wrong
    for wrong in (dict(R=60), dict(C=36), dict(flags=_lib.FLAG_BWD_STE), dict(flags=1 << 20)):
        assert run(**wrong) == _lib.ERR_UNSUPPORTED, wrong
    assert run(flags=_lib.FLAG_REUSE_MASK_T) == (_lib.ERR_UNSUPPORTED if call == "forward" else _lib.ERR_ALIGN)
    assert run() == _lib.ERR_ALIGN
    # 2^30 tiles of a projection are 2^31 of both together
    assert run(R=(1 << 31) - 256, C=129 * 256, L=1) == _lib.ERR_UNSUPPORTED
    assert run(R=(1 << 31) - 256, C=64, L=129 * 256) == _lib.ERR_UNSUPPORTED


def test_gated_alignment_of_every_pointer():
    for n in FORWARD_IN + ("G", "U", "H"):
        assert Gated(**{n: at(40) + 8}).forward(problem()) == _lib.ERR_ALIGN, n
    for n in BACKWARD_IN + BACKWARD_OUT + ("ws",):
        assert Gated(**{n: at(40) + 8}).backward(problem()) == _lib.ERR_ALIGN, n


def test_gated_aliases():
    p = problem()
    for out in ("G", "U", "H"):
        for other in FORWARD_IN + ("G", "U", "H"):
            if other != out:
                g = Gated()
                g.v[out] = g.v[other]
                assert g.forward(p) == _lib.ERR_ALIAS, (out, other)
    for out in BACKWARD_OUT + ("ws",):
        for other in BACKWARD_IN + BACKWARD_OUT:
            if other != out:
                g = Gated()
                g.v[out] = g.v[other]
                assert g.backward(p) == _lib.ERR_ALIAS, (out, other)
    # the last byte of an output, the first past it
    g = Gated()
    g.v["H"] = g.v["X"] + 8 * 32 * 2 - 16
    assert g.forward(p) == _lib.ERR_ALIAS


def test_gated_workspace():
    for r in (4, 8, 17, 64, 65, 128):
        for L, R, C in ((8, 64, 32), (300, 1000, 520), (4096, 1024, 5120)):
            p = problem(R=R, C=C, L=L, r=r)
            assert _lib.gated_workspace_bytes(p, False) == 0
            need = _lib.gated_workspace_bytes(p, True)
            least = 2 * (2 * L * R + 4 * C * ((R + 31) // 32))
            assert least <= need <= least + 2 * (2 * R * 128) + (64 << 20) + 6 * 256
            assert Gated(size=need - 1).backward(p) == _lib.ERR_WORKSPACE
            assert Gated(ws=None).backward(p) == _lib.ERR_WORKSPACE
    f32 = problem(dtype=_lib.DTYPE_F32)
    need = _lib.gated_workspace_bytes(f32, False)
    assert need >= 2 * 8 * 64 * 4
    assert Gated(G=None, U=None, size=need - 1).forward(f32) == _lib.ERR_WORKSPACE
    for bad in (dict(r=0), dict(dtype=9), dict(flags=_lib.FLAG_SPLIT_LAST_WAVE)):
        assert _lib.gated_workspace_bytes(problem(**bad), True) == BAD
    assert _lib.gated_workspace_bytes(problem(flags=_lib.FLAG_REUSE_MASK_T), False) == BAD
    assert _lib.gated_workspace_bytes(problem(flags=_lib.FLAG_REUSE_MASK_T), True) != BAD


def test_gated_without_tokens():
    g = Gated(X=None, H=None, G=None, U=None, ws=None, size=0)
    assert g.forward(problem(L=0)) == _lib.OK
    assert Gated(X=None, H=None, Bg=None).forward(problem(L=0)) == _lib.ERR_NULL


# ---------------------------------------------------------------------------
# update
# ---------------------------------------------------------------------------
def rule(**kw):
    d = dict(momentum=0.9, eps=1e-7, a=3.4445, b=-4.775, c=2.0315, steps=5, nesterov=1, grad_dtype=_lib.DTYPE_BF16,
             param_dtype=_lib.DTYPE_BF16, flags=0)
    d.update(kw)
    return _lib.Update(**d)


def item(i=0, **kw):
    d = dict(rows=16, cols=100, grad=at(4 * i), m=at(4 * i + 1), master=at(4 * i + 2), param=at(4 * i + 3), rate=0.1, decay=0.0)
    d.update(kw)
    return _lib.UpdateItem(**d)


def update(p, items, ws=WS, size=1 << 40, count=None):
    a = (_lib.UpdateItem * max(1, len(items)))(*items)
    return _lib.orthogonal_update(p, a, len(items) if count is None else count, ws, size, None)


def test_update_null_comes_first():
    broken = rule(grad_dtype=9, steps=0)
    assert update(broken, [item(grad=None)]) == _lib.ERR_NULL
    assert update(broken, [item(), item(1, master=None, param=None)]) == _lib.ERR_NULL
    assert _lib.orthogonal_update(broken, None, 1, WS, 1 << 40, None) == _lib.ERR_NULL
    for one in (dict(m=None), dict(param=None), dict(master=None)):
        assert update(broken, [item(**one)]) == _lib.ERR_DTYPE


def test_update_refusals_in_order():
    odd = item(grad=at(0) + 1)  # misaligned: every range comes before it
    assert update(rule(grad_dtype=5, steps=0), [odd]) == _lib.ERR_DTYPE
    assert update(rule(param_dtype=-1, steps=0), [odd]) == _lib.ERR_DTYPE
    for wrong in (dict(momentum=-0.1), dict(momentum=1.1), dict(momentum=NAN), dict(eps=-1.0), dict(eps=INF), dict(a=NAN),
                  dict(b=INF), dict(c=NAN), dict(steps=0), dict(steps=33), dict(nesterov=2)):
        assert update(rule(flags=1, **wrong), [odd]) == _lib.ERR_SHAPE, wrong
    for wrong in (dict(rows=0), dict(cols=0), dict(rows=-4), dict(cols=1 << 31), dict(rows=1 << 20, cols=1 << 20), dict(rate=NAN),
                  dict(decay=INF)):
        assert update(rule(flags=1), [item(1), item(grad=at(0) + 1, **wrong)]) == _lib.ERR_SHAPE, wrong
    assert update(rule(), [odd], count=65536) == _lib.ERR_SHAPE
    assert update(rule(), [odd], count=-1) == _lib.ERR_SHAPE
    assert update(rule(flags=1), [odd]) == _lib.ERR_UNSUPPORTED
    assert update(rule(steps=11), [odd]) == _lib.ERR_UNSUPPORTED  # a^22 is above 2^38
    assert update(rule(steps=32, a=1.5, b=-0.5, c=0.0), [odd]) == _lib.ERR_ALIGN  # 1.5^64 is below
    assert update(rule(), [item(1, rows=129, cols=129), odd]) == _lib.ERR_UNSUPPORTED
    for n in ("m", "master"):
        assert update(rule(), [item(**{n: at(9) + 2})]) == _lib.ERR_ALIGN
    assert update(rule(), [item(param=at(9) + 1)]) == _lib.ERR_ALIGN
    assert update(rule(param_dtype=_lib.DTYPE_F32), [item(param=at(9) + 2)]) == _lib.ERR_ALIGN
    assert update(rule(), [item()], ws=WS + 8) == _lib.ERR_ALIGN


def test_update_aliases():
    for out in ("m", "master", "param"):
        for other in ("grad", "m", "master", "param"):
            if other != out:
                assert update(rule(), [item(**{out: getattr(item(), other)})]) == _lib.ERR_ALIAS, (out, other)
            # across items, by one element
            assert update(rule(), [item(), item(1, **{out: getattr(item(), other) + 1600})]) == _lib.ERR_ALIAS, (out, other)
        assert update(rule(), [item(**{out: WS + 16})]) == _lib.ERR_ALIAS
    assert update(rule(), [item(), item()]) == _lib.ERR_ALIAS
    # one gradient in two items is an input twice; arrays that only touch
    last = item(1, grad=at(0), m=at(1) + 6400, master=at(2) + 6400, param=at(3) + 3200)
    assert update(rule(), [item(), last], size=0) == _lib.ERR_WORKSPACE
    # a long output that lies behind a short one in it
    assert update(rule(), [item(), item(1, m=at(1) + 4), item(2, m=at(1) + 6396)]) == _lib.ERR_ALIAS


def test_update_workspace():
    def need(items, p=None):
        return _lib.orthogonal_workspace_bytes(p or rule(), (_lib.UpdateItem * len(items))(*items), len(items))

    one = need([item()])
    assert 0 < one < 1 << 20
    assert update(rule(), [item()], size=one - 1) == _lib.ERR_WORKSPACE and update(rule(), [item()], ws=None) == _lib.ERR_WORKSPACE
    many = [item(i) for i in range(100)]
    total = need(many)
    assert total >= 100 * one and update(rule(), many, ws=BASE + 500 * GAP, size=total - 1) == _lib.ERR_WORKSPACE
    # a matrix and its transpose take the same
    assert need([item(rows=100, cols=16)]) == one
    for bad in (item(rows=0), item(rows=200, cols=300), item(grad=None)):
        assert need([bad]) == BAD
    assert need([item()], rule(flags=2)) == BAD
    assert update(rule(), [], ws=None, size=0) == _lib.OK


# ---------------------------------------------------------------------------
# sample
# ---------------------------------------------------------------------------
def rows(**kw):
    d = dict(rows=4, vocab=100, row_stride=100, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, dtype=_lib.DTYPE_BF16, flags=0)
    d.update(kw)
    return _lib.Sample(**d)


NAMES = ("logits", "u", "temperature", "top_k", "top_p", "min_p", "token", "logp")


def sample(p, **over):
    v = {n: at(i) for i, n in enumerate(NAMES)}
    v.update(over)
    return _lib.sample(p, *(v[n] for n in NAMES), None, 0, None)


def test_sample_refusals_in_order():
    for n in ("logits", "u", "token"):
        assert sample(rows(dtype=9, rows=4), **{n: None}) == _lib.ERR_NULL
    assert sample(rows(dtype=9), logp=None, temperature=None, top_k=None, top_p=None, min_p=None) == _lib.ERR_DTYPE
    for wrong in (dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(row_stride=-1),
                  dict(row_stride=(1 << 62)), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(top_p=-0.1),
                  dict(top_p=NAN), dict(min_p=-0.5), dict(min_p=NAN), dict(min_p=INF), dict(rows=(1 << 31) - 1, vocab=1 << 27)):
        assert sample(rows(flags=1, **wrong), u=at(1) + 2) == _lib.ERR_SHAPE, wrong
        assert _lib.sample_workspace_bytes(rows(**wrong)) == BAD
    assert sample(rows(flags=1), u=at(1) + 2) == _lib.ERR_UNSUPPORTED
    assert _lib.sample_workspace_bytes(rows(flags=1)) == BAD
    for n, off in (("logits", 1), ("u", 2), ("temperature", 2), ("top_k", 2), ("top_p", 1), ("min_p", 3), ("token", 4), ("logp", 2)):
        assert sample(rows(), **{n: at(30) + off}) == _lib.ERR_ALIGN, n
    assert sample(rows(dtype=_lib.DTYPE_F32), logits=at(0) + 2) == _lib.ERR_ALIGN
    for out in ("token", "logp"):
        for other in NAMES:
            if other != out:
                assert sample(rows(), **{out: at(NAMES.index(other))}) == _lib.ERR_ALIAS, (out, other)
    # the last entry of the last strided row
    assert sample(rows(row_stride=1000), token=at(0) + (3 * 1000 + 96) * 2) == _lib.ERR_ALIAS


def test_sample_without_rows():
    assert _lib.sample(rows(rows=0), *(None,) * 8, None, 0, None) == _lib.OK
