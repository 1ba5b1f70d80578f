"""The embedding's gradient over as many places as a call takes: sums of whole numbers, which binary32 adds exactly."""
import pytest

from tests.gpu_harness import Device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Device()


def draw(torch, count, rows, width, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = ((torch.rand(count, device="cuda", generator=gen) ** 3) * (rows + 2)).long() - 1      # some outside, low ones often
    return tokens.int(), torch.randint(-1, 2, (count, width), device="cuda", generator=gen).bfloat16()


@pytest.mark.parametrize("count,rows", [(1 << 19, 700), ((1 << 19) + 1, 700), ((1 << 20) + 77, 50000), (3 << 20, 3), ((1 << 22) + 131071, 1 << 20),
                                        (1 << 24, 1000), (1 << 24, 300000)])
def test_sums_over_many_places(dev, count, rows):
    torch, f = dev.torch, dev.f
    width = 3
    tokens, grad = draw(torch, count, rows, width, count % 1000)
    inside = (tokens >= 0) & (tokens < rows)
    want = torch.zeros(rows, width, dtype=torch.float64, device="cuda")
    want.index_add_(0, tokens[inside].long(), grad[inside].double())
    assert float(want.abs().max()) < 2 ** 23
    ws = dev.workspace(f.workspace_bytes_embedding(rows, width, count))
    got = torch.full((rows, width), float("nan"), device="cuda")
    f.embedding_gradient(grad, tokens, got, ws)
    assert torch.equal(got.double(), want)
    f.embedding_gradient(grad, tokens, got, ws, 2.0, base=got)
    assert torch.equal(got.double(), 3 * want)


def test_sorting_takes_time_by_the_place(dev):
    """2^24 places may take three times as long a place as 2^21 (by reading every block's counts in every workgroup: eight)"""
    torch, f = dev.torch, dev.f
    took = []
    for count in (1 << 21, 1 << 24):
        tokens, grad = draw(torch, count, 50000, 1, 5)
        ws = dev.workspace(f.workspace_bytes_embedding(50000, 1, count))
        out = torch.empty(50000, 1, device="cuda")
        f.embedding_gradient(grad, tokens, out, ws)
        torch.cuda.synchronize()
        f.profile_enable(True)
        for _ in range(5):
            f.embedding_gradient(grad, tokens, out, ws)
        report = f.profile_report()
        f.profile_enable(False)
        took.append(sum(ms for name, (_, ms) in report.items() if name.startswith("embedding_sort")) / count)
    assert took[1] <= 3 * took[0], took
