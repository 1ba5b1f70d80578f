"""Embedding lookup and its gradient against the definition in 64 bits.

Tolerances: a product or sum in binary32 is off by at most half a step (2^-24 of it), the last rounding by half a step of
the output's type (and half its smallest number).  A sum of k terms in any order is off by at most k 2^-24 of the sum of
their magnitudes."""
import numpy as np
import pytest

from tests.gpu_harness import Device

pytestmark = pytest.mark.gpu

TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


@pytest.fixture(scope="module")
def dev():
    return Device()


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def draw_tokens(torch, gen, count, rows, index, outside=0.2, skew=True):
    u = torch.rand(count, device="cuda", generator=gen, dtype=torch.float64)
    t = (u * np.log(rows + 1)).exp().long() - 1 if skew else (u * rows).long()
    t.clamp_(0, rows - 1)
    o = torch.rand(count, device="cuda", generator=gen)
    t[o < outside / 2] = -1
    t[(o >= outside / 2) & (o < outside * 0.75)] = rows
    t[(o >= outside * 0.75) & (o < outside)] = 2 ** 31 - 1 if index == 32 else 2 ** 40 + 1
    return t.to(torch.int32 if index == 32 else torch.int64)


def strided(torch, rows, width, stride, dtype, gen=None, offset=0):
    """a [rows, width] view of a buffer that begins `offset` elements in, filled with a mark"""
    buf = torch.full((offset + rows * stride + 8,), -7.0, device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * stride].view(rows, stride)[:, :width]
    if gen is not None:
        view.copy_(torch.randn(rows, width, device="cuda", generator=gen))
    return buf, view


@pytest.mark.parametrize("rows,width,count,stride,offset", [
    (1, 1, 1, 1, 0), (7, 3, 5, 3, 1), (1000, 64, 257, 64, 0), (333, 771, 1025, 777, 3), (50, 8192, 3, 8192, 0),
    (129, 513, 64, 600, 5), (4000, 2048, 300, 2048, 0), (20, 9001, 11, 9001, 1)])
@pytest.mark.parametrize("source,out", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "bfloat16"),
                                        ("float16", "float32"), ("float32", "float16"), ("bfloat16", "float16")])
@pytest.mark.parametrize("index", [32, 64])
def test_lookup(dev, rows, width, count, stride, offset, source, out, index):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(rows * 31 + width)
    ti, to = getattr(torch, source), getattr(torch, out)
    tokens = draw_tokens(torch, gen, count, rows, index)
    _, table = strided(torch, rows, width, stride, ti, gen, offset)
    buf, got = strided(torch, count, width, stride + 2, to, None, offset)
    scale = 1.7
    f.embedding(table, tokens, got, scale)
    dev.sync()
    inside = (tokens >= 0) & (tokens < rows)
    want = table.double()[torch.where(inside, tokens, 0).long()] * float(np.float32(scale))
    want[~inside] = 0
    err = (got.double() - want).abs()
    assert bool((err <= want.abs() * (half_step(torch, to) + 2.0 ** -24) * 1.001 + TINY[out]).all())
    assert bool((got[~inside] == 0).all())
    rest = buf[offset:offset + count * (stride + 2)].view(count, stride + 2)[:, width:]
    assert bool((rest == -7).all()) and bool((buf[:offset] == -7).all()) and bool((buf[offset + count * (stride + 2):] == -7).all())


def want_gradient(torch, grad, tokens, rows, scale, base):
    """(the definition in 64 bits, sum of magnitudes, terms) on the host's order"""
    inside = (tokens >= 0) & (tokens < rows)
    at = tokens[inside].long()
    g = grad.double()[inside]
    total = torch.zeros(rows, grad.shape[1], dtype=torch.float64, device="cuda")
    size, terms = torch.zeros_like(total), torch.zeros(rows, dtype=torch.float64, device="cuda")
    total.index_add_(0, at, g)
    size.index_add_(0, at, g.abs())
    terms.index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    scale = float(np.float32(scale))
    want = total * scale + (base.double() if base is not None else 0)
    return want, size * abs(scale), terms


CASES = [(1, 1, 1), (5, 3, 7), (1000, 64, 257), (100, 771, 4099), (9, 513, 5000), (3000, 257, 700), (2, 40, 9000),
         (70000, 128, 20000), (600, 2050, 4096), (1, 96, 12345), (300000, 8, 20000), ((1 << 27) + 5, 1, 9000), (5, 2, 1 << 20)]


# where the ways of summing and sorting change, and one place to either side
EDGES = [(700, 72, n) for n in (63, 64, 65, 255, 257, 1023, 1024, 1025, 8191, 8192, 8193, 10240, 65537)]


@pytest.mark.parametrize("rows,width,count", CASES + EDGES)
@pytest.mark.parametrize("source,out", [("float32", "float32"), ("bfloat16", "float32"), ("float16", "bfloat16"),
                                        ("bfloat16", "bfloat16"), ("float32", "float16")])
@pytest.mark.parametrize("base", ["none", "apart", "place"])
def test_gradient(dev, rows, width, count, source, out, base):
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + width + count)
    ti, to = getattr(torch, source), getattr(torch, out)
    tokens = draw_tokens(torch, gen, count, rows, 64 if count % 2 else 32)
    _, grad = strided(torch, count, width, width + 1, ti, gen, 1)
    buf, got = strided(torch, rows, width, width + 3, to, None, 3)
    _, other = strided(torch, rows, width, width + 3, to, gen, 2)
    ws = dev.workspace(f.workspace_bytes_embedding(rows, width, count))
    scale = 0.37
    start = None
    if base == "apart":
        start = other
    elif base == "place":
        got.copy_(other)
        start = got
    want, size, terms = want_gradient(torch, grad, tokens, rows, scale, None if start is None else other)
    f.embedding_gradient(grad, tokens, got, ws, scale, base=start)
    dev.sync()
    err = (got.double() - want).abs()
    u = 2.0 ** -24
    allowed = (size * (terms[:, None] + 2) * u + want.abs() * u) * (1 + half_step(torch, to)) + want.abs() * half_step(torch, to) * 1.001 + TINY[out]
    assert bool((err <= allowed).all()), float((err / allowed).max())
    none = (terms == 0)[:, None]
    assert bool((~none | (got == (0 if start is None else other))).all())
    rest = buf[3:3 + rows * (width + 3)].view(rows, width + 3)[:, width:]
    assert bool((rest == -7).all()) and bool((buf[:3] == -7).all())
    # the same bits again, over a workspace and an output that hold other things
    if base != "place":
        again = torch.full_like(got, float("nan"))
        ws.fill_(0x5A)
        buf2, got2 = strided(torch, rows, width, width + 3, to, None, 3)
        f.embedding_gradient(grad, tokens, got2, ws, scale, base=start)
        assert torch.equal(got2, got)


def test_gradient_agrees_with_differences(dev):
    """<lookup(table + h D) - lookup(table - h D), W> / 2h is <gradient(W), D>: both sides are linear, so h is 1"""
    torch, f = dev.torch, dev.f
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, width, count, scale = 57, 130, 900, 2.5
    tokens = draw_tokens(torch, gen, count, rows, 64)
    table, d = (torch.randn(rows, width, device="cuda", generator=gen) for _ in range(2))
    w = torch.randn(count, width, device="cuda", generator=gen)
    up, down = torch.empty_like(w), torch.empty_like(w)
    f.embedding(table + d, tokens, up, scale)
    f.embedding(table - d, tokens, down, scale)
    grad = torch.empty_like(table)
    f.embedding_gradient(w, tokens, grad, dev.workspace(f.workspace_bytes_embedding(rows, width, count)), scale)
    a = ((up.double() - down.double()) * w.double()).sum() / 2
    b = (grad.double() * d.double()).sum()
    # rounding of every value by 2^-23 of magnitudes of up to 12 and terms of up to 40: random, 117 000 of them
    assert abs(float(a - b)) <= 2.0 ** -23 * 500 * np.sqrt(rows * width + count * width)


def test_rows_of_tokens_far_apart(dev):
    """element offsets past 2^32: a table of 2^21 + 5 rows that are 2^11 apart"""
    torch, f = dev.torch, dev.f
    rows, width, stride = (1 << 21) + 5, 16, 1 << 11
    buf = torch.zeros(rows * stride, device="cuda", dtype=torch.float16)
    table = buf.view(rows, stride)[:, :width]
    tokens = torch.tensor([rows - 1, 0, rows - 2, -1, rows - 1], device="cuda")
    table[rows - 1] = 3.0
    table[rows - 2] = 5.0
    table[0] = 7.0
    out = torch.full((5, width), 9.0, device="cuda")
    f.embedding(table, tokens, out, 2.0)
    assert out[:, 0].tolist() == [6.0, 14.0, 10.0, 0.0, 6.0] and bool((out == out[:, :1]).all())
    ws = dev.workspace(f.workspace_bytes_embedding(rows, width, 5))
    g = torch.arange(1, 6, device="cuda", dtype=torch.float32)[:, None].expand(5, width).contiguous()
    f.embedding_gradient(g, tokens, table, ws, 1.0, base=table)
    assert table[[rows - 1, 0, rows - 2, 1], width - 1].tolist() == [9.0, 9.0, 8.0, 0.0]


def test_no_tokens(dev):
    torch, f = dev.torch, dev.f
    tokens = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones(4, 8, device="cuda")
    f.embedding(table, tokens, torch.empty(0, 8, device="cuda"))
    grad = torch.full((4, 8), 5.0, device="cuda")
    none = torch.empty(0, 8, device="cuda")
    ws = dev.workspace(16)
    f.embedding_gradient(none, tokens, grad, ws, base=grad)
    assert bool((grad == 5).all())
    f.embedding_gradient(none, tokens, grad, ws, base=table)
    assert bool((grad == 1).all())
    f.embedding_gradient(none, tokens, grad, ws)
    assert bool((grad == 0).all())


def test_infinities_stay_in_their_rows(dev):
    torch, f = dev.torch, dev.f
    g = torch.ones(6, 5, device="cuda")
    g[1] = float("inf")
    g[2] = float("nan")
    g[4] = float("nan")
    tokens = torch.tensor([0, 1, 2, 3, -1, 1], device="cuda")
    out = torch.full((5, 5), -3.0, device="cuda")
    f.embedding_gradient(g, tokens, out, dev.workspace(f.workspace_bytes_embedding(5, 5, 6)))
    assert bool((out[0] == 1).all()) and bool(torch.isinf(out[1]).all()) and bool(torch.isnan(out[2]).all())
    assert bool((out[3] == 1).all()) and bool((out[4] == 0).all())
