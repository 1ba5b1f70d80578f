"""How many bits the orthogonalised update has: results against the exact ones, with what a model of the arithmetic allows
(newton_schulz_model, which says where its figures come from).  Matrices under 512 rows have phases of one step whatever else is
in the list, others of up to two; a result in 16 bits is the one in 32, rounded."""
import pytest

from tests.gpu_harness import Device
from tests.newton_schulz_model import allowed, share_allowed
from tests.test_gpu_orthogonal import DEFAULT, LARGE, SHAPES, lay, matrix_like, view

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Device()


def falling(torch, gen, h, w):
    """a few outer products of falling size, and noise"""
    r = max(1, min(h, w) // 8)
    size = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -0.7
    return (torch.randn(h, r, device="cuda", generator=gen) * size) @ torch.randn(r, w, device="cuda", generator=gen) \
        + 0.5 * torch.randn(h, w, device="cuda", generator=gen)


def one_large(torch, gen, h, w):
    """one singular value far above the others"""
    return torch.randn(h, w, device="cuda", generator=gen) \
        + 30 * torch.randn(h, 1, device="cuda", generator=gen) @ torch.randn(1, w, device="cuda", generator=gen)


def low(m):
    return min(m.rows, m.cols) < 512


@pytest.mark.parametrize("name", list(SHAPES) + list(LARGE))
def test_results_in_32_bits(dev, name):
    torch, f = dev.torch, dev.f
    shapes = SHAPES.get(name) or LARGE[name]
    gen = torch.Generator(device="cuda").manual_seed(31)
    listing, total, ms = lay(torch, f, shapes, [1.0] * len(shapes))
    x = torch.zeros(total, device="cuda")
    for m in ms:
        view(torch, x, m).copy_(matrix_like(torch, gen, m.rows, m.cols))
    got = torch.full_like(x, -7.0)
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal(x, got, listing, ws)
    again = torch.full_like(x, -7.0)
    ws.fill_(0x5A)
    f.orthogonal(x, again, listing, ws)
    assert torch.equal(again, got)                      # every matrix, the last one's end and what is behind it
    for m in ms[:1] if len(set(shapes)) == 1 else ms:
        # tiles of 256 add the cross terms to the same sum
        want, off = allowed(torch, view(torch, x, m), DEFAULT, phases=(1,) if low(m) else (1, 2), roundings=3 if max(min(s) for s in shapes) > 256 else 1)
        err = float(torch.linalg.vector_norm(view(torch, got, m).double() - want))
        assert err <= off, (m.rows, m.cols, err / float(torch.linalg.vector_norm(want)), off / float(torch.linalg.vector_norm(want)))


@pytest.mark.parametrize("kind", ["falling", "one_large"])
@pytest.mark.parametrize("shapes", [[(100, 8000)], [(8000, 100)], [(256, 4608)], [(64, 769)], [(64, 768)], [(193, 317)] * 2, [(1024, 4096)],
                                    [(1024, 4096), (100, 4700)], [(100, 4700), (1024, 4096), (16, 300)],
                                    [(1024, 4096), (100, 4600)], [(16, 2000), (520, 9000), (60, 60), (3000, 60), (2000, 600)], [(513, 20000)]],
                         ids=lambda s: "%d of %dx%d" % (len(s), *s[0]))
@pytest.mark.parametrize("kept", ["float16", "bfloat16"])
def test_results_in_16_bits(dev, kind, shapes, kept):
    """Nearly all of them are the nearest numbers to the exact result: as many as binary32 arithmetic gives"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(32)
    make = falling if kind == "falling" else one_large
    listing, total, ms = lay(torch, f, shapes, [1.25] * len(shapes))
    x = torch.zeros(total, device="cuda", dtype=getattr(torch, kept))
    for m in ms:
        view(torch, x, m).copy_(make(torch, gen, m.rows, m.cols))
    got = torch.full_like(x, -7.0)
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal(x, got, listing, ws)
    wide = torch.full((total,), -7.0, device="cuda")
    f.orthogonal(x, wide, listing, ws)
    assert torch.equal(wide.to(x.dtype), got)
    for m in ms:
        near, share = share_allowed(torch, view(torch, x, m), DEFAULT, x.dtype, phases=(1,) if low(m) else (1, 2),
                                    roundings=3 if max(min(s) for s in shapes) > 256 else 1, gain=m.gain)
        other = float((view(torch, got, m) != near).double().mean())
        assert other <= share, (m.rows, m.cols, other, share)
