"""The reference that the 8-bit step's gradients are held to: its formulas are the derivatives, roundings to 8 bits are within its bounds, mistakes are not."""
import pytest
import torch

from tests import mlp_ref as M

SIZES = [(64, 256, 256), (33, 528, 784)]


def inputs(T, d, F):
    g = torch.Generator().manual_seed(T)
    draw = lambda std, *s: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).double()
    return draw(1.0, T, d), draw(0.05, 2 * F, d), draw(0.05, d, F), draw(0.01, T, d)


@pytest.mark.parametrize("T,d,F", SIZES)
def test_formulas_are_the_derivatives(T, d, F):
    at = inputs(T, d, F)
    for got, want in zip(M.step(*at, eight=False), M.gradients(*at)):
        assert (got - want).norm() <= 1e-10 * want.norm()


@pytest.mark.parametrize("T,d,F", SIZES)
def test_roundings_are_within_the_bounds(T, d, F):
    at = inputs(T, d, F)
    assert M.check(M.step(*at), *at) == []


@pytest.mark.parametrize("T,d,F", SIZES)
@pytest.mark.parametrize("mistake,found", [("no mlp", "dX"), ("rmsnorm", "dX along x"), ("silu'", "dWup, gates"), ("gates", "dWup, gates"), ("half the tokens", "dWdown")])
def test_mistakes_are_not(T, d, F, mistake, found):
    at = inputs(T, d, F)
    assert any(line.startswith(found) for line in M.check(M.step(*at, mistake=mistake), *at))
