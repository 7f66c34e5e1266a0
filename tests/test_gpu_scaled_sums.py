"""How exact the sums of the products of 8-bit operands with block scales are: within 2e-5 of the result's 2-norm whatever K is, on every kind of kernel, on the GPU.

Products and scales are exact, so this is the instructions' adding up alone: measured 0.9e-5 to 1.6e-5, by how the codes are spread; 2e-5 leaves a quarter.  A block
of the contraction that is lost or counted twice is off by 1 / sqrt(K / 128) of the 2-norm, 0.09 for the longest here."""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests.test_gpu_scaled_large import OnDevice

pytestmark = pytest.mark.gpu


# few rows, 128 x 256 tiles, partials, 256 x 256 tiles
@pytest.mark.parametrize("M,N,K,ws", [(8, 512, 384, False), (8, 512, 8192, False), (300, 784, 384, False), (300, 784, 16384, False), (300, 784, 2064, True),
                                      (33, 528, 3088, True), (2304, 4096, 640, False), (2064, 4112, 2064, False)])
@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("std,lo,hi", [(1.0, 118, 132), (0.3, 122, 128), (60.0, 120, 120)])
def test_sums(M, N, K, ws, trans, std, lo, hi):
    o = OnDevice(M, N, K, trans, M + K, std, lo, hi)
    w = o.workspace() if ws else None
    assert (w is not None) == ws
    D = torch.empty(M, N, device="cuda")
    o.run([coda.store(D, f32=True)], workspace=w)
    assert (D.cpu().double() - o.product()).norm() <= 2e-5 * o.product().norm()
