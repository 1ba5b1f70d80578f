"""Newton-Schulz orthogonalisation and the momentum step against the definition in 64 bits.

Tolerance (2-norm of a matrix's error): the iteration's map has, as a function of the singular values, a slope of at most
L = |a| (a rise of three and a half at zero for the default), so an error made in step i reaches the result at most L^(steps - 1 - i) times as
large.  A step makes, relative to the 2-norms of its terms, an error of e = 2^-24 (3 + 2 sqrt(K / 16)) a product: two operands
of 2^-24 each, the part of the product that is left out, and 3 K / 16 roundings of the running sum, which add up like random
ones.  a X has none of them, b A X two products, c A A X three; storing X adds 2^-24 of it."""
import numpy as np
import pytest

from tests.gpu_harness import Device

pytestmark = pytest.mark.gpu

DEFAULT = [(3.4445, -4.7750, 2.0315)] * 5


@pytest.fixture(scope="module")
def dev():
    return Device()


def largest(torch, gram):
    """its largest eigenvalue: exactly for small matrices, else by forty products with a vector, and a tenth more"""
    if float(gram.abs().max()) == 0:
        return 0.0
    if gram.shape[0] <= 400:
        return float(torch.linalg.matrix_norm(gram, 2))
    v = torch.ones(gram.shape[0], 1, dtype=gram.dtype, device=gram.device)
    for i in range(40):
        v = gram @ v
        size = float(torch.linalg.vector_norm(v))
        v = v / size
    return 1.1 * size


def exact(torch, g, coefficients=DEFAULT, eps=1e-7):
    """(orthogonalised g in 64 bits, bound of the error's 2-norm)"""
    u = 2.0 ** -24
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    norm = float(torch.linalg.vector_norm(x)) + float(np.float32(eps))
    x = x / norm if norm > 0 else x * 0
    bound = u * float(torch.linalg.vector_norm(x))
    e = u * (3 + 2 * np.sqrt(max(x.shape) / 16))
    for a, b, c in [[float(np.float32(v)) for v in abc] for abc in coefficients]:
        gram = x @ x.t()
        top = largest(torch, gram)
        size = float(torch.linalg.vector_norm(x))
        x = a * x + (b * gram + c * (gram @ gram)) @ x
        bound = bound * max(abs(a), 1.0) + e * size * (abs(a) + 2 * abs(b) * top + 3 * abs(c) * top * top) + u * float(torch.linalg.vector_norm(x))
    return (x.t() if tall else x), bound


def matrix_like(torch, gen, h, w, rank=None):
    r = rank if rank is not None else max(1, min(h, w) // 4)
    g = torch.randn(h, r, device="cuda", generator=gen) @ torch.randn(r, w, device="cuda", generator=gen)
    return (g + (0.3 if rank is None else 0.0) * torch.randn(h, w, device="cuda", generator=gen)) * 1e-3


def lay(torch, f, shapes, gains, spread=False):
    """matrices one behind the other, odd gaps and strides between them where `spread`"""
    at, got = 3 if spread else 0, []
    for i, (h, w) in enumerate(shapes):
        stride = w + (i % 3 if spread else 0)
        got.append(f.Matrix(at, h, w, stride, gains[i]))
        at += h * stride + (i % 2 if spread else 0)
    return f.matrices(got), at + 5, got


def view(torch, flat, m):
    return torch.as_strided(flat, (m.rows, m.cols), (m.stride, 1), flat.storage_offset() + m.offset)


SHAPES = {
    "one": [(1, 1)],
    "row": [(1, 300), (300, 1)],
    "small": [(16, 27), (10, 64), (64, 10), (33, 33)],
    "tile": [(128, 128)],
    "around": [(127, 129), (129, 127), (128, 130), (257, 255)],
    "wide": [(48, 1500), (1500, 48)],
    "long": [(5, 20011), (20011, 5)],
    "middle": [(384, 640), (640, 384)],
    "many": [(7 + 5 * i, 90 - i) for i in range(70)],
    "small wide": [(64, 768), (768, 64), (32, 768), (767, 31), (33, 577), (513, 49), (1, 768), (17, 256)],
    "small wider": [(64, 769), (64, 64)],
    "small many": [(1 + i % 64, 1 + 37 * i % 768) for i in range(150)],
}


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("source,out", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"),
                                        ("float32", "float16")])
def test_orthogonal(dev, name, source, out):
    torch, f = dev.torch, dev.f
    shapes = SHAPES[name]
    gen = torch.Generator(device="cuda").manual_seed(len(name) + len(shapes))
    gains = [1.0 + 0.25 * (i % 4) for i in range(len(shapes))]
    listing, total, ms = lay(torch, f, shapes, gains, spread=True)
    x = torch.full((total,), float("nan"), device="cuda", dtype=getattr(torch, source))
    for m in ms:
        view(torch, x, m).copy_(matrix_like(torch, gen, m.rows, m.cols) * 300)
    got = torch.full((total,), -7.0, device="cuda", dtype=getattr(torch, out))
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal(x, got, listing, ws)
    dev.sync()
    half = torch.finfo(got.dtype).eps / 2
    rest = torch.ones(total, dtype=torch.bool, device="cuda")
    for m in ms:
        want, bound = exact(torch, view(torch, x, m))
        want, bound = want * m.gain, bound * m.gain
        err = float(torch.linalg.vector_norm(view(torch, got, m).double() - want))
        assert err <= bound + half * 1.001 * float(torch.linalg.vector_norm(want)) + 1e-7, (m.rows, m.cols, err, bound)
        view(torch, rest, m).fill_(False)
    assert bool((got[rest] == -7).all())
    # the same bits over a workspace that holds other things, and in place where the types agree
    ws.fill_(0x5A)
    again = torch.full_like(got, 3.0)
    f.orthogonal(x, again, listing, ws)
    assert torch.equal(again[~rest], got[~rest])
    if source == out:
        place = x.clone()
        f.orthogonal(place, place, listing, ws)
        assert torch.equal(place[~rest], got[~rest])


# tiles of 256 of every kind of product; rows so long that their sums are taken in slices; wide products in slices; many of one size
LARGE = {
    "four": [(2560, 2600)] * 4,
    "two": [(4100, 2570), (2560, 2600)],
    "long": [(300, 20000), (20003, 190)],
    "deep": [(1024, 1030)],
    "eight": [(1024, 1024)] * 8,
}


@pytest.mark.parametrize("name", list(LARGE))
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_large(dev, name, kind):
    torch, f = dev.torch, dev.f
    shapes = LARGE[name]
    gen = torch.Generator(device="cuda").manual_seed(11)
    listing, total, ms = lay(torch, f, shapes, [1.0] * len(shapes))
    x = torch.zeros(total, device="cuda", dtype=getattr(torch, kind))
    for m in ms:
        view(torch, x, m).copy_(matrix_like(torch, gen, m.rows, m.cols))
    got = torch.full((total,), float("nan"), device="cuda", dtype=x.dtype)
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    f.orthogonal(x, got, listing, ws)
    half = torch.finfo(got.dtype).eps / 2
    for m in ms:
        want, bound = exact(torch, view(torch, x, m))
        size = float(torch.linalg.vector_norm(want))
        err = float(torch.linalg.vector_norm(view(torch, got, m).double() - want))
        assert err <= bound + half * 1.001 * size, (m.rows, m.cols, err, bound)
        # far inside that bound, which adds up the worst of every step: what binary32 products give
        assert err <= (2e-5 + half) * size, (m.rows, m.cols, err / size)
    again = torch.full_like(got, 1.0)
    f.orthogonal(x, again, listing, ws)
    assert torch.equal(again[:ms[-1].offset], got[:ms[-1].offset])


def test_offsets_past_32_bits(dev):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(12)
    at = (1 << 32) + 5
    m = f.Matrix(at, 70, 40, (1 << 20) + 3)
    listing = f.matrices([m])
    x = torch.zeros(listing.end, device="cuda", dtype=torch.bfloat16)
    view(torch, x, m).copy_(torch.randn(70, 40, device="cuda", generator=gen))
    want, bound = exact(torch, view(torch, x, m))
    f.orthogonal(x, x, listing, dev.workspace(f.workspace_bytes_orthogonal(listing)))
    err = float(torch.linalg.vector_norm(view(torch, x, m).double() - want))
    assert err <= bound + 2.0 ** -8 * 1.001 * float(torch.linalg.vector_norm(want))


@pytest.mark.parametrize("stride", [(1 << 23) - 5, (1 << 23) + 5])   # rows from the first byte to past 2^31, and further
def test_rows_far_apart(dev, stride):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.zeros(63 * stride + 40, device="cuda")
    m = f.Matrix(0, 64, 40, stride)
    view(torch, x, m).copy_(matrix_like(torch, gen, 64, 40))
    want, bound = exact(torch, view(torch, x, m))
    listing = f.matrices([m])
    f.orthogonal(x, x, listing, dev.workspace(f.workspace_bytes_orthogonal(listing)))
    assert float(torch.linalg.vector_norm(view(torch, x, m).double() - want)) <= bound + 2.0 ** -24 * 1.001 * float(torch.linalg.vector_norm(want))
    view(torch, x, m).zero_()
    assert not bool(x.any())


def test_ranks_sizes_and_zeros(dev):
    """a matrix of rank one, one of zeros, tiny and huge ones, eps of 0 and one that shrinks"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(2)
    shapes = [(40, 70)] * 5
    listing, total, ms = lay(torch, f, shapes, [1.0] * 5)
    x = torch.zeros(total, device="cuda")
    view(torch, x, ms[0]).copy_(matrix_like(torch, gen, 40, 70, rank=1))
    view(torch, x, ms[2]).copy_(torch.randn(40, 70, device="cuda", generator=gen) * 1e-30)
    view(torch, x, ms[3]).copy_(torch.randn(40, 70, device="cuda", generator=gen) * 1e30)
    view(torch, x, ms[4]).copy_(torch.randn(40, 70, device="cuda", generator=gen))
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    for eps in (0.0, 1e-7, 10.0):
        got = torch.full((total,), float("nan"), device="cuda")
        f.orthogonal(x, got, listing, ws, eps=eps)
        for i, m in enumerate(ms):
            want, bound = exact(torch, view(torch, x, m), eps=eps)
            err = float(torch.linalg.vector_norm(view(torch, got, m).double() - want))
            assert err <= bound + 1e-6 * float(torch.linalg.vector_norm(want)) + 1e-9, (eps, i, err, bound)
        assert bool((view(torch, got, ms[1]) == 0).all())


@pytest.mark.parametrize("coefficients", [[(1.5, -0.5, 0.0)], [(2.0, -1.5, 0.5)] * 3, [(3.4445, -4.7750, 2.0315)] * 2,
                                          [(4.0, -6.0, 3.0)] + [(1.875, -1.25, 0.375)] * 11, [(0.0, 0.0, 0.0)]])
def test_other_coefficients(dev, coefficients):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(3)
    listing, total, ms = lay(torch, f, [(96, 200), (150, 150), (140, 30)], [1.0, 2.0, 0.5])
    x = torch.empty(total, device="cuda")
    for m in ms:
        view(torch, x, m).copy_(matrix_like(torch, gen, m.rows, m.cols))
    got = torch.full((total,), float("nan"), device="cuda")
    f.orthogonal(x, got, listing, dev.workspace(f.workspace_bytes_orthogonal(listing)), coefficients=coefficients)
    for m in ms:
        want, bound = exact(torch, view(torch, x, m), coefficients)
        err = float(torch.linalg.vector_norm(view(torch, got, m).double() - m.gain * want))
        assert err <= m.gain * bound + 2.0 ** -23 * float(torch.linalg.vector_norm(want)) + 1e-9


def test_columns_of_one_array(dev):
    """two matrices whose rows alternate in memory"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(4)
    ms = [f.Matrix(0, 50, 30, 72), f.Matrix(30, 50, 42, 72)]
    listing = f.matrices(ms)
    x = torch.randn(50 * 72, device="cuda", generator=gen)
    got = torch.empty_like(x)
    f.orthogonal(x, got, listing, dev.workspace(f.workspace_bytes_orthogonal(listing)))
    for m in ms:
        want, bound = exact(torch, view(torch, x, m))
        assert float(torch.linalg.vector_norm(view(torch, got, m).double() - want)) <= bound + 1e-6


def test_a_matrix_that_is_not_finite_leaves_the_others(dev):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(6)
    listing, total, ms = lay(torch, f, [(60, 60)] * 3, [1.0] * 3)
    x = torch.randn(total, device="cuda", generator=gen)
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    want = torch.empty_like(x)
    f.orthogonal(x, want, listing, ws)
    view(torch, x, ms[1])[3, 4] = float("nan")
    got = torch.empty_like(x)
    f.orthogonal(x, got, listing, ws)
    for m in (ms[0], ms[2]):
        assert torch.equal(view(torch, got, m), view(torch, want, m))


@pytest.mark.parametrize("weight", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shapes", [[(16, 27), (130, 70), (64, 576), (1, 40), (200, 200)],
                                    [(16, 27), (64, 70), (64, 576), (1, 40), (700, 50), (10, 64)]], ids=["mixed", "small"])
def test_step(dev, weight, grad, nesterov, shapes):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(8)
    gains = [max(1.0, h / w) ** 0.5 for h, w in shapes]
    listing, total, ms = lay(torch, f, shapes, gains, spread=True)
    g = torch.randn(total, device="cuda", generator=gen).to(getattr(torch, grad))
    mom = torch.randn(total, device="cuda", generator=gen)
    w = (torch.randn(total, device="cuda", generator=gen) * 0.05).to(getattr(torch, weight))
    lr, beta, decay = 0.02, 0.9, 0.1
    ws = dev.workspace(f.workspace_bytes_orthogonal(listing))
    mom_in, w_in = mom.clone(), w.clone()
    mo, wo = torch.full_like(mom, -7.0), torch.full_like(w, -7.0)
    f.orthogonal_step(g, mom, w, listing, ws, lr, beta, decay, nesterov, momentum_out=mo, weights_out=wo)
    assert torch.equal(mom, mom_in) and torch.equal(w, w_in)
    lr32, beta32 = float(np.float32(lr)), float(np.float32(beta))
    keep = 1.0 - lr32 * float(np.float32(decay))
    rest = torch.ones(total, dtype=torch.bool, device="cuda")
    for m in ms:
        view(torch, rest, m).fill_(False)
        want_m = beta32 * view(torch, mom, m).double() + view(torch, g, m).double()
        assert bool(((view(torch, mo, m).double() - want_m).abs() <= 2.0 ** -24 * 1.01 * want_m.abs()).all())
        got_m = view(torch, mo, m).double()                   # as stored: its rounding is in the momentum
        u = view(torch, g, m).double() + beta32 * got_m if nesterov else got_m
        want, bound = exact(torch, u.float())
        want = keep * view(torch, w, m).double() - lr32 * m.gain * want
        err = float(torch.linalg.vector_norm(view(torch, wo, m).double() - want))
        half = torch.finfo(w.dtype).eps / 2
        assert err <= lr * m.gain * bound + (half + 2.0 ** -22) * float(torch.linalg.vector_norm(want)) + 1e-9, (m.rows, m.cols)
    assert bool((mo[rest] == -7).all()) and bool((wo[rest] == -7).all())
    f.orthogonal_step(g, mom, w, listing, ws, lr, beta, decay, nesterov)       # in place
    assert torch.equal(mom[~rest], mo[~rest]) and torch.equal(w[~rest], wo[~rest])
    assert torch.equal(mom[rest], mom_in[rest]) and torch.equal(w[rest], w_in[rest])


def test_no_matrices(dev):
    torch, f = dev.torch, dev.f
    listing = f.matrices([])
    x = torch.ones(4, device="cuda")
    f.orthogonal(x, x, listing, dev.workspace(16))
    assert bool((x == 1).all())
