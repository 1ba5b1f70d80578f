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


USUAL = [(3.4445, -4.7750, 2.0315)] * 5
NEAR_ONE = USUAL + [(1.875, -1.25, 0.375)] * 4      # singular values from 1/256 on are at one, smaller ones anywhere below


def test_singular_values_between_any_samples_count(lib):
    """x (1 + 40000 x^2 - 40000 x^4) is one at one, and 7436 where x^2 is 0.6"""
    for shapes in ([(96, 200)], [(64, 64)], [(512, 20000)]):
        assert refusal(lib, shapes, NEAR_ONE + [(1.0, 40000.0, -40000.0)]) == EUNSUPPORTED
        assert refusal(lib, shapes, NEAR_ONE + [(1.0, 40.0, -40.0)]) == EWORKSPACE
        assert refusal(lib, shapes, [(1.0, 0.0, 0.0), (0.0, 0.0, 0.0)] + USUAL) == EWORKSPACE
        assert refusal(lib, shapes, [(0.0, 0.0, 4000.0)]) == EWORKSPACE
        assert refusal(lib, shapes, [(0.0, 0.0, 4100.0)]) == EUNSUPPORTED
        assert refusal(lib, shapes, [(0.0, 16000.0, -16000.0)]) == EWORKSPACE      # s p(s^2) is 2974 at s^2 = 0.6, p(s^2) 4000 at 0.5
        assert refusal(lib, shapes, [(0.0, 16500.0, -16500.0)]) == EUNSUPPORTED    # 4125 at 0.5


@pytest.mark.parametrize("coefficients", [[(100.0, 0, 0), (.01, 0, 0)], [(4000.0, 0, 0), (.001, 0, 0), (1, 0, 0)], [(4000.0, 0, 0), (1, 0, 0), (1, 0, 0)],
                                          [(4000.0, 0, 0), (2e-4, 6e-11, 0)]])
def test_singular_values_up_to_4096_are_accepted(lib, coefficients):
    for shapes in ([(64, 768)], [(512, 20000)], [(1024, 1024)]):
        for out_type in (0, 1):
            assert refusal(lib, shapes, coefficients, out_type) == EWORKSPACE
            assert refusal(lib, shapes, [(4097.0, 0, 0)] + coefficients[1:], out_type) == EUNSUPPORTED
            assert refusal(lib, shapes, [(-4097.0, 0, 0)] + coefficients[1:], out_type) == EUNSUPPORTED
            assert refusal(lib, shapes, [(4000.0, 0, 0), (2.0, 0, 0)], out_type) == EUNSUPPORTED


def listing_of(count, rows, cols):
    """count matrices behind each other"""
    import numpy as np
    kind = np.dtype([("offset", "<u8"), ("stride", "<u8"), ("rows", "<u4"), ("cols", "<u4"), ("gain", "<f4"), ("reserved", "<u4")])
    m = np.zeros(count, kind)
    m["offset"] = np.arange(count, dtype=np.uint64) * np.uint64(rows * cols)
    m["stride"], m["rows"], m["cols"], m["gain"] = cols, rows, cols, 1
    return m, m.ctypes.data_as(C.POINTER(fftsp.Matrix))


def test_the_largest_lists(lib):
    m, p = listing_of(1, 16384, 1 << 20)                   # both limits at once
    assert lib.fftsp_workspace_bytes_orthogonal(p, 1) > 4 * 4 << 34
    assert lib.fftsp_orthogonal(A, 1, B, 1, p, 1, None, 0, 1e-7, A + (1 << 50), 1 << 20, None) == EWORKSPACE
    m, p = listing_of(2, 16384, 1 << 20)
    assert lib.fftsp_workspace_bytes_orthogonal(p, 2) == 0
    assert lib.fftsp_orthogonal(A, 1, A + (1 << 50), 1, p, 2, None, 0, 1e-7, A + (1 << 52), 1 << 62, None) == EUNSUPPORTED
    m, p = listing_of((1 << 22) + 1, 1, 1)                  # small ones, a workgroup each
    assert lib.fftsp_workspace_bytes_orthogonal(p, 1 << 22) > 0
    assert lib.fftsp_workspace_bytes_orthogonal(p, (1 << 22) + 1) == 0
    assert lib.fftsp_orthogonal(A, 0, B, 0, p, 1 << 22, None, 0, 1e-7, W, 1 << 20, None) == EWORKSPACE
    assert lib.fftsp_orthogonal(A, 0, B, 0, p, (1 << 22) + 1, None, 0, 1e-7, W, 1 << 40, None) == EUNSUPPORTED


def test_overlaps_of_rows_that_are_far_apart(lib):
    """distances whose product passes 64 bits: the table's second row is beyond any memory, its first one still meets `out`"""
    def lookup(rows, stride, out, count=2, out_stride=4):
        return lib.fftsp_embedding(A, 0, rows, 4, stride, B, 64, count, 1.0, out, 0, out_stride, None)

    def gradient(rows, stride, out, count=2, out_stride=4):
        return lib.fftsp_embedding_gradient(A, 0, out_stride, B, 64, count, 1.0, None, out, 0, rows, 4, stride, W, 1 << 40, None)
    far = 1 << 40
    assert lookup((1 << 24) + 1, far, A + 16) == EINVAL and lookup(1 << 30, far, W) == EINVAL
    assert lookup(1 << 10, far, W) == EINVAL and lookup(10, 4, W, 1 << 24, far) == EINVAL
    assert gradient((1 << 24) + 1, far, W) == EINVAL and gradient(10, 4, W, (1 << 24) - 1, far) == EINVAL
    assert lib.fftsp_embedding_gradient(A, 0, 4, B, 64, 2, 1.0, None, W, 0, 1 << 8, 4, far, W + (1 << 60), 0, None) == EWORKSPACE


def test_the_binding_takes_no_size_modulo_a_fields_range():
    torch = pytest.importorskip("torch")
    for bad in ((0, (1 << 32) + 4, 1), (0, 1, (1 << 32) + 4), (-1, 4, 4), (0, -4, 4), (0, 4, -4), (1 << 64, 4, 4), (0, 4, 4, (1 << 64) + 4), (0, 4, 4, -1)):
        with pytest.raises(ValueError):
            fftsp.Matrix(*bad)
    m = fftsp.Matrix(5, (1 << 32) - 1, 7, 9, 2.0)
    assert (m.offset, m.stride, m.rows, m.cols, m.gain, m.reserved) == (5, 9, (1 << 32) - 1, 7, 2.0, 0)
    wide = torch.empty(2, (1 << 32) + 4, device="meta", dtype=torch.float16)
    with pytest.raises(ValueError):
        fftsp._rows(wide, wide.shape[-1])
    assert fftsp.workspace_bytes_embedding(10, (1 << 32) + 4, 3) == 0
