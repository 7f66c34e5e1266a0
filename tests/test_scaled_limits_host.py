"""Sizes past what one launch takes (2^32 work items) are refused before anything is launched."""
import ctypes

import pytest

from paper_2605_19269_amd import coda
from tests.test_abi_host import P, _mat

F8 = coda.CODA_F8E4M3


# rows, columns, square blocks: workgroups of 64 rows x 128 columns (square: 128) and 256 threads
@pytest.mark.parametrize("rows,cols,square", [(1 << 30, 8, 0), ((1 << 30) - 63, 128, 0), (1 << 29, 136, 0), (1 << 20, 1 << 17, 0), ((1 << 31) - 112, 8, 1), (1 << 30, 256, 1)])
def test_quantize(rows, cols, square):
    ld, pitch = (cols + 15) // 16 * 16, (rows + 15) // 16 * 16
    X = _mat(coda, P, rows, cols, ld=ld)
    assert coda._lib.coda_quantize(None, ctypes.byref(X), square, P, ld, P, pitch, None, 0) == coda.CODA_ERR_SHAPE


# workgroups of 32 rows x 128 columns
@pytest.mark.parametrize("rows,cols", [(1 << 29, 8), ((1 << 29) - 31, 128), (1 << 28, 136), (1 << 19, 1 << 17)])
def test_dequantize(rows, cols):
    ld = (cols + 15) // 16 * 16
    Q = _mat(coda, P, rows, cols, ld=ld, dtype=F8)
    assert coda._lib.coda_dequantize(None, ctypes.byref(Q), P, (rows + 15) // 16 * 16, P, ld) == coda.CODA_ERR_SHAPE


def test_products_and_gradients():
    M, N, K = 1 << 29, 1 << 12, 16
    A, B = _mat(coda, P, M, K, dtype=F8), _mat(coda, P, N, K, trans=1, dtype=F8)
    ops, n = coda._prog([coda.coda_epi_op(kind=coda.CODA_EPI_STORE, out=P, ld_out=N)])
    assert coda._lib.coda_gemm_scaled(None, M, N, K, ctypes.byref(A), P, M, ctypes.byref(B), P, N, ops, n, None, 0) == coda.CODA_ERR_SHAPE
    N = 1 << 20
    A, B = _mat(coda, P, K, N, trans=1, dtype=F8), _mat(coda, P, K, N, dtype=F8)
    assert coda._lib.coda_grad_scaled(None, N, N, K, ctypes.byref(A), P, 16, ctypes.byref(B), P, 16, P, N, None, 0) == coda.CODA_ERR_SHAPE
