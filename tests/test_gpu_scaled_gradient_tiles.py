"""Weight gradients from 8-bit checkpoints on the GPU: whole 256 x 256 tiles, and one round of 128 x 128 tiles.  The test and its bounds are those of the other gradients
(test_gpu_scaled_large)."""
import pytest

from tests import test_gpu_scaled_large as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 320), (4096, 4096, 257), (1024, 8192, 333)])
@pytest.mark.parametrize("b8", [True, False])
def test_gradient(M, N, K, b8):
    L.test_gradient_in_large_tiles(M, N, K, b8)
