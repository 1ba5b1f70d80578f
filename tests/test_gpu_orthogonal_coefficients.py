"""Orthogonalisation under coefficients other than the usual ones: what the header accepts is right."""
import pytest

from tests.gpu_harness import Device
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
