"""Gradients of the step in 8 bits, on the GPU, against automatic differentiation of its loss in 64 bits.  Bounds: mlp_ref."""
import pytest
import torch

from tests import mlp_ref
from tests.test_gpu_scaled import Mlp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,F", [(64, 256, 256), (33, 528, 784), (300, 256, 512)])
def test_gradients_of_the_step(T, d, F):
    m = Mlp(T, d, F)
    m.step()
    torch.cuda.synchronize()
    at = [t.cpu().double() for t in (m.X, m.Wup, m.Wdown, m.dY)]
    assert mlp_ref.check([t.cpu().double() for t in (m.dX, m.dWup, m.dWdown)], *at) == []
