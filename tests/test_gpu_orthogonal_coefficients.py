"""Orthogonalisation under coefficients other than the usual ones: what the header accepts is right."""
import pytest

from tests.gpu_harness import Device
from tests.newton_schulz_model import iterate, predicted
from tests.test_gpu_orthogonal import view

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Device()


def flat_list(f, shapes):
    at, ms = 0, []
    for rows, cols in shapes:
        ms.append(f.Matrix(at, rows, cols))
        at += rows * cols
    return f.matrices(ms), ms


@pytest.mark.parametrize("shapes", [[(512, 20000)], [(64, 768)], [(130, 70), (20, 2000)]], ids=lambda s: "%dx%d" % s[0])
@pytest.mark.parametrize("factors", [(.01, 1, 1000, 5, 1), (.01, 1, 2000, 3, .5), (.01, .01, 100, 100, .01), (.001, 1, 60, 60, 60)])
def test_linear_steps_scale(dev, shapes, factors):
    """X <- a X only.  A product of planes is off by 2^-23 of itself for either operand, 2^-22 for the part left out and three
    roundings of a sum that has one term, X stored by 2^-23: under 2^-20.  Five steps have at most ten products."""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(7)
    listing, ms = flat_list(f, shapes)
    x = torch.randn(listing.end, device="cuda", generator=gen)
    got = torch.full_like(x, float("nan"))
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal(x, got, listing, ws, coefficients=[(a, 0.0, 0.0) for a in factors], eps=0.0)
    size = 1.0
    for a in factors:
        size *= float(torch.tensor(a, dtype=torch.float32))
    for m in ms:
        g = view(torch, x, m).double()
        want = g * (size / float(torch.linalg.vector_norm(g)))
        err = float(torch.linalg.vector_norm(view(torch, got, m).double() - want))
        assert err <= 10 * 2.0 ** -20 * size, (m.rows, m.cols, err / size)


@pytest.mark.parametrize("shape", [(96, 200), (64, 200), (200, 40), (520, 3000)], ids=lambda s: "%dx%d" % s)
@pytest.mark.parametrize("out", ["float32", "float16"])
def test_steps_that_are_largest_at_small_singular_values(dev, shape, out):
    """Nine steps take all singular values from 1/256 on to one, where the last step's polynomial is one; a smaller one meets
    its largest, eleven.  Allowed: three times what the arithmetic's model is off, over one and two steps a phase, and half
    a step of the result's type."""
    torch, f = dev.torch, dev.f
    co = [(3.4445, -4.7750, 2.0315)] * 5 + [(1.875, -1.25, 0.375)] * 4 + [(1.0, 40.0, -40.0)]
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = min(shape)
    left = torch.linalg.qr(torch.randn(shape[0], n, device="cuda", generator=gen, dtype=torch.float64))[0]
    right = torch.linalg.qr(torch.randn(shape[1], n, device="cuda", generator=gen, dtype=torch.float64))[0]
    g = ((left * torch.logspace(0, -5, n, device="cuda", dtype=torch.float64)) @ right.t().contiguous()).float()
    before = torch.linalg.svdvals(iterate(torch, g, co[:-1], 0.0))
    assert float((1 + 40 * before ** 2 - 40 * before ** 4).max()) > 8    # the matrix has such a singular value
    listing = f.matrices([f.Matrix(0, *shape)])
    got = torch.full(shape, float("nan"), device="cuda", dtype=getattr(torch, out))
    f.orthogonal(g.view(-1), got.view(-1), listing, dev.workspace(f.workspace_bytes_orthogonal(listing)), coefficients=co, eps=0.0)
    off = 0.0
    for phase in (1, 2):
        want, more = predicted(torch, g, co, 0.0, phase=phase, roundings=3)
        off = max(off, more)
    size = float(torch.linalg.vector_norm(want))
    err = float(torch.linalg.vector_norm(got.double() - want))
    assert err <= 3 * off + torch.finfo(got.dtype).eps / 2 * 1.001 * size, (err, off, size)


@pytest.mark.parametrize("shape", [(64, 300), (70, 300), (520, 1500)], ids=lambda s: "%dx%d" % s)
@pytest.mark.parametrize("coefficients", [[(100, 0, 0), (.01, 0, 0)], [(3000, 0, 0), (1, -1.5e-7, 1e-14), (.5, 0, 0)],
                                          [(40, 0, 0), (60, 0, 0), (1.6, -2e-7, 1e-14), (1, 0, 0), (1e-3, 0, 0)]])
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_singular_values_of_thousands(dev, shape, coefficients, out):
    """Allowed: as above"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(6)
    g = torch.randn(shape, device="cuda", generator=gen) @ torch.diag(torch.logspace(0, -2, shape[1], device="cuda"))
    listing = f.matrices([f.Matrix(0, *shape)])
    got = torch.full(shape, float("nan"), device="cuda", dtype=getattr(torch, out))
    f.orthogonal(g.view(-1), got.view(-1), listing, dev.workspace(f.workspace_bytes_orthogonal(listing)), coefficients=coefficients, eps=0.0)
    off = 0.0
    for phase in (1, 2):
        want, more = predicted(torch, g, coefficients, 0.0, phase=phase, roundings=3)
        off = max(off, more)
    size = float(torch.linalg.vector_norm(want))
    err = float(torch.linalg.vector_norm(got.double() - want))
    assert err <= 3 * off + torch.finfo(got.dtype).eps / 2 * 1.001 * size, (err, off, size)
