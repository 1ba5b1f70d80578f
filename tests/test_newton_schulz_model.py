"""The model that the GPU tests of the orthogonalised update take their tolerances from sees lost bits."""
import pytest
import torch

from tests.newton_schulz_model import allowed, iterate, share_allowed

USUAL = [(3.4445, -4.7750, 2.0315)] * 5


def matrix(rows, cols, seed=1):
    gen = torch.Generator().manual_seed(seed)
    r = max(1, min(rows, cols) // 4)
    return torch.randn(rows, r, generator=gen) @ torch.randn(r, cols, generator=gen) + 0.3 * torch.randn(rows, cols, generator=gen)


def distance(a, b):
    return float(torch.linalg.vector_norm(a - b))


@pytest.mark.parametrize("shape", [(1, 300), (16, 27), (64, 64), (64, 768), (48, 1500), (128, 128), (193, 317), (384, 640)])
def test_four_lost_bits_are_seen(shape):
    """operands of 18 bits instead of 22, and the model with another seed as it is"""
    g = matrix(*shape)
    want, off = allowed(torch, g, USUAL)
    assert distance(iterate(torch, g, USUAL, gen=torch.Generator().manual_seed(77)), want) <= off
    assert distance(iterate(torch, g, USUAL, gen=torch.Generator().manual_seed(77), bits=18), want) > 1.5 * off
    assert off <= 1.2e-5 * float(torch.linalg.vector_norm(want))


def test_exact_iteration_is_the_definition():
    g = matrix(20, 33)
    x = g.double() / (torch.linalg.vector_norm(g.double()) + float(torch.tensor(1e-7)))
    for a, b, c in torch.tensor(USUAL, dtype=torch.float32).double().tolist():
        gram = x @ x.t()
        x = a * x + (b * gram + c * gram @ gram) @ x
    for phase in (1, 2, 3):
        assert distance(iterate(torch, g, USUAL, phase=phase), x) <= 1e-11
        assert distance(iterate(torch, g.t().contiguous(), USUAL, phase=phase), x.t()) <= 1e-11


def test_three_steps_a_phase_are_seen_where_sums_are_short():
    """in a result of binary16"""
    gen = torch.Generator().manual_seed(5)
    left = torch.randn(60, 7, generator=gen) * torch.arange(1, 8).float() ** -0.7
    g = left @ torch.randn(7, 1500, generator=gen) + 0.5 * torch.randn(60, 1500, generator=gen)
    near, share = share_allowed(torch, g, USUAL, torch.float16)
    drawn = lambda phase: float((iterate(torch, g, USUAL, gen=torch.Generator().manual_seed(9), phase=phase).half() != near).double().mean())
    assert drawn(1) <= share < drawn(3)
