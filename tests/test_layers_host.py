"""Refusals and host arithmetic of the embedding and the orthogonalised update: argument errors come back before any launch,
so no call here has a device behind its pointers."""
import ctypes as C
import math
import os

import pytest

from paper_1811_08596_amd import fftsp

A = 1 << 20           # fake addresses, far apart: never dereferenced on these paths
B, D, E, F, W = (A + i * (1 << 30) for i in range(1, 6))
OK, EINVAL, EWORKSPACE, EUNSUPPORTED = fftsp.OK, fftsp.EINVAL, fftsp.EWORKSPACE, fftsp.EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fftsp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return fftsp.load()


def test_embedding_refusals(lib):
    def call(**k):
        return lib.fftsp_embedding(k.get("table", A), k.get("tt", 0), k.get("rows", 10), k.get("width", 4), k.get("ts", 4),
                                   k.get("tokens", B), k.get("bits", 64), k.get("n", 3), k.get("scale", 1.0), k.get("out", D),
                                   k.get("ot", 1), k.get("os", 4), None)
    for bad in (dict(table=None), dict(tokens=None), dict(out=None), dict(tt=3), dict(tt=-1), dict(ot=7), dict(bits=16),
                dict(rows=0), dict(rows=(1 << 30) + 1), dict(width=0), dict(width=(1 << 20) + 1, ts=1 << 21, os=1 << 21),
                dict(ts=3), dict(os=3), dict(ts=(1 << 40) + 1), dict(scale=math.inf), dict(scale=math.nan), dict(n=(1 << 30) + 1),
                dict(table=A + 2), dict(out=D + 1), dict(tokens=B + 4), dict(tokens=B + 2, bits=32),
                dict(out=A + 8), dict(out=B), dict(out=A + 4 * 39, ot=0)):
        assert call(**bad) == EINVAL, bad
    assert call(n=0) == OK and call(n=0, table=A, tokens=None, out=None) == OK
    assert call(n=0, tt=9) == EINVAL


def test_embedding_gradient_refusals(lib):
    need = fftsp.workspace_bytes_embedding(10, 4, 3)
    assert need > 0
    assert fftsp.workspace_bytes_embedding(0, 4, 3) == 0 and fftsp.workspace_bytes_embedding(10, 0, 3) == 0
    assert fftsp.workspace_bytes_embedding(10, 4, (1 << 24) + 1) == 0
    assert fftsp.workspace_bytes_embedding((1 << 30) + 1, 4, 3) == 0
    assert fftsp.workspace_bytes_embedding(1 << 30, 1 << 20, 1 << 24) > 0

    def call(**k):
        return lib.fftsp_embedding_gradient(k.get("grad", A), k.get("gt", 1), k.get("gs", 4), k.get("tokens", B), k.get("bits", 64),
                                            k.get("n", 3), k.get("scale", 1.0), k.get("base", None), k.get("out", D), k.get("ot", 0),
                                            k.get("rows", 10), k.get("width", 4), k.get("os", 4), k.get("ws", W), k.get("wsb", need),
                                            None)
    for bad in (dict(grad=None), dict(tokens=None), dict(out=None), dict(gt=3), dict(ot=3), dict(bits=8), dict(rows=0),
                dict(width=0), dict(gs=3), dict(os=3), dict(scale=math.nan), dict(grad=A + 1), dict(out=D + 2), dict(base=E + 2),
                dict(base=D + 16), dict(base=D - 16), dict(out=A), dict(out=B), dict(ws=None), dict(ws=W + 8)):
        assert call(**bad) == EINVAL, bad
    assert call(wsb=need - 1) == EWORKSPACE
    assert call(n=(1 << 24) + 1) == EUNSUPPORTED


def matrices(*ms):
    return (fftsp.Matrix * len(ms))(*[fftsp.Matrix(*m) for m in ms]), len(ms)


def test_lists_of_matrices(lib):
    def need(*ms):
        return lib.fftsp_workspace_bytes_orthogonal(*matrices(*ms))
    assert need((0, 4, 5), (20, 3, 3)) > 0
    assert lib.fftsp_workspace_bytes_orthogonal(None, 0) == 0             # nothing to do, nothing needed
    assert lib.fftsp_workspace_bytes_orthogonal(None, 1) == 0
    assert need((0, 0, 5)) == 0 and need((0, 5, 0)) == 0
    assert need((0, 4, 5, 4)) == 0                                       # stride below the columns
    assert need((0, 4, 5), (19, 3, 3)) == 0                              # one element shared
    assert need((20, 3, 3), (0, 4, 5)) > 0                               # any order
    assert need((0, 4, 5), (0, 4, 5)) == 0                               # the same one twice
    assert need((0, 4, 3, 10), (3, 4, 7, 10)) > 0                        # columns of one array
    assert need((0, 4, 3, 10), (2, 4, 7, 10)) == 0
    assert need((0, 4, 3, 10), (4, 4, 7, 10)) == 0                       # its last column is the first one's next row
    assert need((0, 4, 3, 10), (5, 2, 2, 9)) == 0                        # other strides: refused where they meet
    assert need((0, 100, 3, 10), (3, 2, 7, 10), (43, 3, 7, 10), (990, 1, 5), (995, 4, 4)) == 0
    assert need((0, 100, 3, 10), (3, 2, 7, 10), (43, 3, 7, 10), (993, 1, 5), (998, 4, 4)) > 0
    assert need((0, 16385, 16385)) == 0 and need((0, 1, (1 << 20) + 1)) == 0 and need((0, 1, 1 << 20)) > 0
    assert need((0, 4, 5, 5, math.nan)) == 0


def test_orthogonal_refusals(lib):
    ms, n = matrices((0, 4, 5), (20, 3, 3))
    need = lib.fftsp_workspace_bytes_orthogonal(ms, n)
    co = (C.c_float * 6)(1, 2, 3, 4, 5, 6)

    def call(**k):
        return lib.fftsp_orthogonal(k.get("x", A), k.get("xt", 0), k.get("out", B), k.get("ot", 0), k.get("ms", ms), k.get("n", n),
                                    k.get("co", None), k.get("steps", 0), k.get("eps", 1e-7), k.get("ws", W), k.get("wsb", need), None)
    bad_co = (C.c_float * 3)(1, math.inf, 0)
    for bad in (dict(x=None), dict(out=None), dict(xt=3), dict(ot=-1), dict(ms=None), dict(n=-1), dict(co=co, steps=0),
                dict(co=co, steps=17), dict(co=bad_co, steps=1), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf),
                dict(ws=None), dict(ws=W + 4), dict(x=A + 2), dict(out=B + 1, ot=1), dict(out=A, ot=1), dict(out=A + 4),
                dict(ms=matrices((0, 4, 5), (3, 3, 3))[0])):
        assert call(**bad) == EINVAL, bad
    assert call(wsb=need - 1) == EWORKSPACE
    for steps in ([5000, 0, 0], [4, 0, 0] * 7, [20, 0, 0] * 3):                      # singular values or products past 4096
        assert call(co=(C.c_float * len(steps))(*steps), steps=len(steps) // 3) == EUNSUPPORTED, steps
    assert call(ms=matrices((0, 20000, 20000))[0], n=1) == EUNSUPPORTED
    assert call(n=0) == OK and call(ms=None, n=0, x=None, out=None, ws=None) == OK


def test_step_refusals(lib):
    ms, n = matrices((0, 4, 5), (20, 3, 3))
    need = lib.fftsp_workspace_bytes_orthogonal(ms, n)

    def call(step=None, **k):
        s = fftsp.Step(0.1, 0.9, 0.0, 1e-7, 1, 0, None)
        for name, v in (step or {}).items():
            setattr(s, name, v)
        return lib.fftsp_orthogonal_step(k.get("g", A), k.get("gt", 0), k.get("m", B), k.get("mo", B), k.get("w", D), k.get("wo", D),
                                         k.get("wt", 0), k.get("ms", ms), k.get("n", n), None if k.get("none") else C.byref(s),
                                         k.get("ws", W), k.get("wsb", need), None)
    for bad in (dict(none=True), dict(g=None), dict(m=None), dict(mo=None), dict(w=None), dict(wo=None), dict(gt=3), dict(wt=3),
                dict(step=dict(lr=math.nan)), dict(step=dict(beta=-0.1)), dict(step=dict(beta=1.5)), dict(step=dict(weight_decay=math.inf)),
                dict(step=dict(lr=3e38, weight_decay=3e38)), dict(step=dict(eps=-1.0)), dict(ws=None), dict(m=B + 2), dict(wo=D + 2),
                dict(mo=B + 4), dict(wo=D + 4), dict(mo=A), dict(wo=A), dict(wo=B), dict(mo=D, wo=E), dict(mo=E, wo=E)):
        assert call(**bad) == EINVAL, bad
    assert call(wsb=need - 1) == EWORKSPACE
    assert call(n=0) == OK


def test_the_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    t = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        fftsp.embedding(t, torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4))     # not on a GPU
    with pytest.raises(ValueError):
        fftsp._rows(t.t()[:, :3], 3)                                                # columns are not consecutive
    with pytest.raises(ValueError):
        fftsp._rows(torch.zeros(2, 3, 4).transpose(0, 1), 4)
    assert fftsp._rows(torch.zeros(2, 3, 4), 4)[1:] == (6, 4)
    assert fftsp._rows(torch.zeros(5, 8)[:, 2:5], 3)[1:] == (5, 8)
    assert fftsp._rows(torch.zeros(1, 8)[:, 2:5], 3)[1:] == (1, 8)
    with pytest.raises(TypeError):
        fftsp._tokens(torch.zeros(2, dtype=torch.int16), 2)
    with pytest.raises(ValueError):
        fftsp._tokens(torch.zeros(4, dtype=torch.int64)[::2], 2)
    with pytest.raises(TypeError):
        fftsp._type(torch.zeros(1, dtype=torch.float64))
    listing = fftsp.matrices([fftsp.Matrix(3, 4, 5, 7)])
    assert listing.end == 3 + 3 * 7 + 5 and fftsp.workspace_bytes_orthogonal(listing) > 0
    with pytest.raises(ValueError):
        fftsp._flat(torch.zeros(28), listing, "x")
    assert fftsp._flat(torch.zeros(29), listing, "x")
    with pytest.raises(ValueError):
        fftsp._coefficients([(1.0, 2.0)])
