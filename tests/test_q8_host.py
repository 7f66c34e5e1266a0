"""The entry points for 8 bits with block scales without a GPU: refusals (before anything is launched), the program grammar, the plans, and
the reference that the GPU tests use."""
import ctypes
import re

import pytest
import torch

from paper_2605_19269_amd import coda
from tests import q8_ref as R
from tests.test_abi_host import P, ROOT, _mat, _op

F8 = coda.CODA_F8E4M3


def gemm(M, N, K, A=None, B=None, ops=(), sa=P, lsa=64, sb=P, lsb=64, ws=None, nbytes=0):
    A = A or _mat(coda, P, M, K, dtype=F8)
    B = B or _mat(coda, P, N, K, trans=1, dtype=F8)
    arr, n = coda._prog(list(ops))
    return coda._lib.coda_gemm_scaled(None, M, N, K, ctypes.byref(A), sa, lsa, ctypes.byref(B), sb, lsb, arr, n, ws, nbytes)


def store(ld=64, out=P):
    return _op(coda, coda.CODA_EPI_STORE, out=out, ld_out=ld)


def store_q8(ld=64, pitch=64, out=P, scales=P, flags=0):
    return _op(coda, coda.CODA_EPI_STORE_Q8, flags=flags, out=out, ld_out=ld, out2=scales, i0=pitch)


def fwd_q8(**k):
    return _op(coda, coda.CODA_EPI_SWIGLU_FWD_Q8, **k)


def bwd_q8(**k):
    k = dict(dict(in_=P, ld_in=128, in2=P, i0=64), **k)
    return _op(coda, coda.CODA_EPI_SWIGLU_BWD_Q8, **k)


def test_enums_mirror_the_header():
    text = open(ROOT + "/include/coda.h").read()
    for name in ("CODA_EPI_STORE_Q8", "CODA_EPI_SWIGLU_FWD_Q8", "CODA_EPI_SWIGLU_BWD_Q8"):
        assert int(re.search(r"\b%s\s*=\s*(\d+)" % name, text).group(1)) == getattr(coda, name)


def test_product_refuses_bad_arguments():
    st = [store()]
    assert gemm(0, 64, 32, ops=st) == coda.CODA_OK and gemm(64, 0, 32, B=_mat(coda, P, 0, 32, trans=1, dtype=F8), ops=st) == coda.CODA_OK
    assert gemm(64, 64, 40, ops=st) == coda.CODA_ERR_ALIGN                                              # pitch of 40 bytes
    assert gemm(64, 64, 24, A=_mat(coda, P, 64, 24, ld=32, dtype=F8), B=_mat(coda, P, 64, 24, ld=32, trans=1, dtype=F8), ops=st) == coda.CODA_ERR_SHAPE
    assert gemm(64, 72, 32, B=_mat(coda, P, 72, 32, trans=1, dtype=F8), ops=[store(72)], lsb=80) == coda.CODA_ERR_SHAPE
    assert gemm(64, 64, 32, A=_mat(coda, P, 32, 64, trans=1, dtype=F8), ops=st) == coda.CODA_ERR_SHAPE  # A^T is coda_grad_scaled
    assert gemm(64, 64, 32, A=_mat(coda, P, 64, 32), ops=st) == coda.CODA_ERR_DTYPE
    assert gemm(64, 64, 32, B=_mat(coda, P, 64, 32, trans=1), ops=st) == coda.CODA_ERR_DTYPE
    assert gemm(-1, 64, 32, ops=st) == coda.CODA_ERR_SHAPE
    assert gemm(64, 64, 32, ops=st, sa=None) == coda.CODA_ERR_NULL and gemm(64, 64, 32, ops=st, sb=None) == coda.CODA_ERR_NULL
    assert gemm(64, 64, 32, ops=st, lsa=48) == coda.CODA_ERR_SHAPE and gemm(64, 64, 32, ops=st, lsb=48) == coda.CODA_ERR_SHAPE
    assert gemm(64, 64, 32, ops=st, lsa=72) == coda.CODA_ERR_ALIGN and gemm(64, 64, 32, ops=st, sa=P + 4) == coda.CODA_ERR_ALIGN
    assert gemm(64, 64, 32, ops=st, lsb=1 << 31) == coda.CODA_ERR_SHAPE
    assert gemm(64, 64, 32, ops=[]) == coda.CODA_ERR_PROGRAM
    need = coda.coda_gemm_scaled_workspace_bytes(64, 64, 4096)
    big = dict(A=_mat(coda, P, 64, 4096, dtype=F8), B=_mat(coda, P, 64, 4096, trans=1, dtype=F8), ops=st)
    assert need > 0 and gemm(64, 64, 4096, ws=P, nbytes=need - 1, **big) == coda.CODA_ERR_WORKSPACE
    assert gemm(64, 64, 4096, ws=P + 4, nbytes=need, **big) == coda.CODA_ERR_ALIGN


def test_programs_of_the_product():
    g = lambda ops, N=64: gemm(0, N, 32, A=_mat(coda, P, 0, 32, dtype=F8), B=_mat(coda, P, N, 32, trans=1, dtype=F8), ops=ops)
    OK, BAD, SHAPE, NULL, ALIGN = coda.CODA_OK, coda.CODA_ERR_PROGRAM, coda.CODA_ERR_SHAPE, coda.CODA_ERR_NULL, coda.CODA_ERR_ALIGN
    rs = _op(coda, coda.CODA_EPI_ROW_SCALE, in_=P)
    add = _op(coda, coda.CODA_EPI_ADD_TILE, in_=P, ld_in=64)
    z = fwd_q8(out=P, ld_out=64, out2=P, i0=64)
    assert g([store()]) == OK and g([rs, add, store()]) == OK
    assert g([store_q8()]) == OK and g([rs, store_q8()]) == OK
    assert g([fwd_q8(), store_q8()]) == OK and g([rs, z, store_q8()]) == OK
    assert g([bwd_q8(), store_q8(128)]) == OK and g([bwd_q8(out2=P, flags=1), store_q8(128)]) == OK
    assert g([add, store_q8()]) == BAD and g([store_q8(), rs]) == BAD and g([store_q8(flags=2)]) == BAD
    assert g([z]) == BAD and g([z, store()]) == BAD and g([z, rs, store_q8()]) == BAD and g([fwd_q8(flags=1), store_q8()]) == BAD
    assert g([rs, bwd_q8(), store_q8(128)]) == BAD and g([bwd_q8(), store(128)]) == BAD and g([bwd_q8(flags=2), store_q8(128)]) == BAD
    assert g([_op(coda, coda.CODA_EPI_SWIGLU_FWD), store_q8()]) == BAD
    assert g([_op(coda, coda.CODA_EPI_ACCUM_F32, out=P, ld_out=64)]) == BAD
    assert g([fwd_q8(), store_q8()], N=48) == SHAPE                                                      # 24 codes a row
    assert g([store_q8(48)]) == SHAPE and g([store_q8(72)]) == ALIGN and g([store_q8(pitch=72)]) == ALIGN
    assert g([store_q8(out=None)]) == NULL and g([store_q8(scales=None)]) == NULL and g([store_q8(out=P + 8)]) == ALIGN
    assert g([bwd_q8(in2=None), store_q8(128)]) == NULL and g([bwd_q8(ld_in=64), store_q8(128)]) == SHAPE and g([bwd_q8(), store_q8(64)]) == SHAPE
    assert g([fwd_q8(out=P, ld_out=64, out2=None, i0=64), store_q8()]) == NULL
    # these ops are not coda_gemm's
    A, B = _mat(coda, P, 0, 32), _mat(coda, P, 32, 64)
    for ops in ([store_q8()], [fwd_q8(), store_q8()], [bwd_q8(), store_q8(128)]):
        assert coda.coda_gemm_raw(None, 0, 64, 32, A, B, ops) == BAD


def test_scale_pitch_covers_the_rows():
    assert gemm(64, 64, 32, ops=[store_q8(pitch=48)]) == coda.CODA_ERR_SHAPE                             # 64 rows


def test_quantize_and_dequantize_refuse_bad_arguments():
    L = coda._lib

    def q(rows=4, cols=16, ld=None, ptr=P, dtype=0, trans=0, square=0, codes=P, ldc=16, s=P, lds=16, st=None, ldst=0):
        m = _mat(coda, ptr, rows, cols, ld=ld, trans=trans, dtype=dtype)
        return L.coda_quantize(None, ctypes.byref(m), square, codes, ldc, s, lds, st, ldst)

    def d(rows=4, cols=16, ld=16, ptr=P, dtype=F8, trans=0, s=P, lds=16, out=P, ldo=16):
        m = _mat(coda, ptr, rows, cols, ld=ld, trans=trans, dtype=dtype)
        return L.coda_dequantize(None, ctypes.byref(m), s, lds, out, ldo)

    E = coda
    for f in (q, d):
        assert f(rows=0) == E.CODA_OK and f(cols=0) == E.CODA_OK
        assert f(cols=12) == E.CODA_ERR_SHAPE and f(trans=1) == E.CODA_ERR_SHAPE and f(rows=-1) == E.CODA_ERR_SHAPE
        assert f(dtype=1) == E.CODA_ERR_DTYPE and f(ptr=None) == E.CODA_ERR_NULL and f(ptr=P + 8) == E.CODA_ERR_ALIGN
        assert f(s=None) == E.CODA_ERR_NULL and f(s=P + 8) == E.CODA_ERR_ALIGN and f(lds=24) == E.CODA_ERR_ALIGN and f(rows=17) == E.CODA_ERR_SHAPE
    assert q(dtype=F8) == E.CODA_ERR_DTYPE and d(dtype=0) == E.CODA_ERR_DTYPE
    assert q(codes=None) == E.CODA_ERR_NULL and q(ldc=8) == E.CODA_ERR_SHAPE and q(ldc=24) == E.CODA_ERR_ALIGN
    assert q(st=P, ldst=16) == E.CODA_ERR_SHAPE                                                          # not without square blocks
    assert q(square=1, st=P, ldst=0) == E.CODA_ERR_SHAPE and q(square=1, st=P + 1, ldst=16) == E.CODA_ERR_ALIGN
    assert d(out=None) == E.CODA_ERR_NULL and d(ldo=8) == E.CODA_ERR_SHAPE and d(ldo=20) == E.CODA_ERR_ALIGN
    assert L.coda_quantize(None, None, 0, P, 16, P, 16, None, 0) == E.CODA_ERR_NULL and L.coda_dequantize(None, None, P, 16, P, 16) == E.CODA_ERR_NULL


def test_gradient_refuses_bad_arguments():
    def grad(M=32, N=32, K=8, A=None, B=None, sa=P, lsa=16, sb=P, lsb=16, G=P, ldg=None, ws=None, nbytes=0, b8=True):
        A = A or _mat(coda, P, K, M, trans=1, dtype=F8)
        B = B or _mat(coda, P, K, N, dtype=F8 if b8 else 0)
        return coda._lib.coda_grad_scaled(None, M, N, K, ctypes.byref(A), sa, lsa, ctypes.byref(B), sb, lsb, G, ldg or max(N, 4), ws, nbytes)

    E = coda
    assert grad(M=0, A=_mat(coda, P, 8, 0, ld=16, trans=1, dtype=F8)) == E.CODA_OK
    assert grad(A=_mat(coda, P, 32, 8, ld=16, dtype=F8)) == E.CODA_ERR_SHAPE                             # not transposed
    assert grad(B=_mat(coda, P, 32, 8, ld=16, trans=1, dtype=F8)) == E.CODA_ERR_SHAPE
    assert grad(M=24, A=_mat(coda, P, 8, 24, ld=32, trans=1, dtype=F8)) == E.CODA_ERR_SHAPE
    assert grad(N=24, B=_mat(coda, P, 8, 24, ld=32, dtype=F8)) == E.CODA_ERR_SHAPE
    assert grad(N=20, b8=False, sb=None, B=_mat(coda, P, 8, 20, ld=24)) == E.CODA_ERR_SHAPE
    assert grad(A=_mat(coda, P, 8, 32, trans=1)) == E.CODA_ERR_DTYPE and grad(b8=False) == E.CODA_ERR_DTYPE       # scales of a bf16 operand
    assert grad(sa=None) == E.CODA_ERR_NULL and grad(sb=None) == E.CODA_ERR_NULL and grad(G=None) == E.CODA_ERR_NULL
    assert grad(K=20, A=_mat(coda, P, 20, 32, trans=1, dtype=F8), B=_mat(coda, P, 20, 32, dtype=F8)) == E.CODA_ERR_SHAPE   # 16 scales, 20 tokens
    assert grad(ldg=16) == E.CODA_ERR_SHAPE and grad(ldg=34) == E.CODA_ERR_ALIGN and grad(G=P + 4) == E.CODA_ERR_ALIGN
    need = coda.coda_grad_scaled_workspace_bytes(32, 32, 4096)
    k = dict(K=4096, A=_mat(coda, P, 4096, 32, trans=1, dtype=F8), B=_mat(coda, P, 4096, 32, dtype=F8), lsa=4096, lsb=4096)
    assert need > 0 and grad(ws=P, nbytes=need - 1, **k) == E.CODA_ERR_WORKSPACE and grad(ws=P + 8, nbytes=need, **k) == E.CODA_ERR_ALIGN


def test_workspaces_of_no_work_are_empty():
    for f in (coda.coda_gemm_scaled_workspace_bytes, coda.coda_grad_scaled_workspace_bytes):
        assert f(0, 64, 64) == 0 and f(64, 0, 64) == 0 and f(-1, 64, 64) == 0 and f(64, 64, 0) == 0


def test_binding_refuses_tensors_of_the_wrong_kind():
    u = lambda *s: torch.zeros(s, dtype=torch.uint8)
    X = torch.zeros(4, 256, dtype=torch.bfloat16)
    for call in (lambda: coda.coda_quantize(X, u(4, 256), u(1, 16), stream=0),                           # one block of scales for two
                 lambda: coda.coda_quantize(X, u(4, 128), u(2, 16), stream=0),
                 lambda: coda.coda_quantize(X, u(4, 256), u(2, 3), stream=0),
                 lambda: coda.coda_quantize(X, torch.zeros(4, 256), u(2, 16), stream=0),
                 lambda: coda.coda_dequantize(u(4, 256), u(2, 16), torch.zeros(4, 256), stream=0),
                 lambda: coda.store_q8(u(4, 256), torch.zeros(2, 16)),
                 lambda: coda.store_q8(u(4, 256), u(2, 16).t()),
                 lambda: coda.swiglu_bwd_q8(u(4, 256), u(1, 16)),
                 lambda: coda.coda_gemm_scaled(u(4, 256), u(1, 16), u(16, 256), u(2, 16), [], transB=True, stream=0),
                 lambda: coda.coda_gemm_scaled(u(4, 256), u(2, 16), u(256, 32), u(2, 16), [], stream=0),
                 lambda: coda.coda_grad_scaled(u(16, 32), u(1, 16), u(16, 32), u(1, 16), torch.zeros(32, 16), stream=0)):
        with pytest.raises(AssertionError):
            call()


def test_a_program_keeps_its_tensors():
    import weakref
    t, s = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(1, 16, dtype=torch.uint8)
    refs = [weakref.ref(t), weakref.ref(s)]
    op = coda.store_q8(t, s)
    assert (op.out, op.ld_out, op.out2, op.i0) == (t.data_ptr(), 128, s.data_ptr(), 16)
    del t, s
    assert all(r() is not None for r in refs)


def test_the_reference_knows_the_format():
    codes = torch.arange(256, dtype=torch.uint8)
    v = R.decode(codes)
    assert torch.equal(torch.nan_to_num(v, 999.0), torch.nan_to_num(codes.view(torch.float8_e4m3fn).double(), 999.0))
    finite = v[torch.isfinite(v)]
    assert torch.equal(R.round_e4m3(finite), finite) and torch.equal(R.decode(R.codes_of(finite)), finite)
    amax = torch.tensor([0.0, 448.0, 449.0, 224.0, 1.0, 2.0 ** -118, 2.0 ** -150, 3.38e38], dtype=torch.float64)
    byte = R.scale_byte(amax)
    assert byte.tolist()[:4] == [1, 127, 128, 126] and (amax <= 448 * R.scale(byte)).all()
    assert ((byte == 1) | (amax > 448 * R.scale(byte - 1))).all()
    x = torch.tensor([17.0, 18.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10], dtype=torch.float64)
    assert R.round_e4m3(x).tolist() == [16.0, 18.0, 20.0, 0.0, 2.0 ** -8]                                # ties to even, subnormals too


def test_kernels_fit_their_registers_and_lds():
    """What the compiler reported: nothing spills in the whole-tile kernels, the small ones and the gradients; two registers in the ragged 256 x 256 instances of
    SwiGLU backward into 8 bits."""
    import os
    import re
    from paper_2605_19269_amd import build as B
    if not os.path.exists(B.RESOURCES):
        B.build(force=True)
    seen = {}
    for line in open(B.RESOURCES):
        name, vgpr, agpr, scratch, spill, lds = line.split()
        m = re.match(r"_ZN4coda\d+(gemm_scaled_\w+?|grad_scaled_kernel|epi_rows_q8_kernel|quantize_\w+?_kernel|dequantize_kernel)(I|EP)(.*)", name)
        if not m:
            continue
        seen[m.group(1)] = seen.get(m.group(1), 0) + 1
        ragged_backward = re.match(r"gemm_scaled_largeILb[01]ELi2ELb1ELb1E", m.group(1) + m.group(2) + m.group(3))
        assert int(spill) <= (4 if ragged_backward else 0) and int(agpr) == 0 and int(vgpr) <= 256 and int(lds) <= 160 * 1024, line
    assert seen == {"gemm_scaled_few": 8, "gemm_scaled_large": 28, "gemm_scaled_tile": 12, "gemm_scaled_partial": 6, "grad_scaled_kernel": 4, "epi_rows_q8_kernel": 3,
                    "quantize_rows_kernel": 2, "quantize_square_kernel": 1, "dequantize_kernel": 1}, seen
