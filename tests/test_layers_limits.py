"""Which calls of the embedding and the orthogonalised update are accepted: limits that do not go by how a list is taken.
A call that is accepted stops at a workspace of too few bytes, so no call here has a device behind its pointers."""
import ctypes as C
import os

import pytest

from paper_1811_08596_amd import fftsp

A = 1 << 20           # fake addresses, far apart: never dereferenced on these paths
B, W = A + (1 << 40), A + (1 << 41)
OK, EINVAL, EWORKSPACE, EUNSUPPORTED = fftsp.OK, fftsp.EINVAL, fftsp.EWORKSPACE, fftsp.EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fftsp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return fftsp.load()


def refusal(lib, shapes, coefficients, out_type=0):
    """What the call returns that has one byte less of workspace than it needs"""
    at, listing = 0, []
    for rows, cols in shapes:
        listing.append(fftsp.Matrix(at, rows, cols))
        at += rows * cols
    ms = (fftsp.Matrix * len(listing))(*listing)
    need = lib.fftsp_workspace_bytes_orthogonal(ms, len(listing))
    assert need > 0
    flat = [v for abc in coefficients for v in abc]
    return lib.fftsp_orthogonal(A, 0, B, out_type, ms, len(listing), (C.c_float * len(flat))(*flat), len(coefficients), 1e-7, W,
                                need - 1, None)


SHAPES = [[(64, 768)], [(65, 65)], [(300, 20000)], [(512, 20000)], [(1024, 1024)], [(2048, 2048)], [(1024, 4096)] * 4, [(768, 4100)],
          [(16, 27), (512, 20000)]]


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: "%d of %dx%d" % (len(s), *s[-1]))
@pytest.mark.parametrize("out_type", [0, 1, 2])
@pytest.mark.parametrize("coefficients", [[(.01, 0, 0)] * 2 + [(100, 0, 0)] * 2 + [(.01, 0, 0)],
                                          [(.01, 0, 0), (1, 0, 0), (1000, 0, 0), (5, 0, 0), (1, 0, 0)],
                                          [(.001, 0, 0), (1, 0, 0), (60, 0, 0), (60, 0, 0), (60, 0, 0)]])
def test_products_over_several_steps_refuse_nothing(lib, shapes, out_type, coefficients):
    """the steps' polynomials grow past 4096 together, in one place or another, while singular values do not"""
    assert refusal(lib, shapes, coefficients, out_type) == EWORKSPACE
