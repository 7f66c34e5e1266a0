"""Infinities and NaN among the values of a block that is rounded to 8 bits behind a product: they become the code NaN, and the block's scale and other codes are
those of its finite values.  On every kind of kernel, on the GPU."""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import q8_ref as R
from tests.test_gpu_q8 import guarded
from tests.test_gpu_scaled import Operands

pytestmark = pytest.mark.gpu

INF, NAN = 70, 9                              # columns of D: one that overflows, one that is NaN
# 128 x 256 tiles, 256 x 256 ragged and whole, divided
SHAPES = [(66, 288, 256, False), (2064, 4128, 144, False), (2304, 4096, 128, False), (70, 544, 2064, True)]


def overflowing(M, N, K, trans, ws):
    """Operands whose product has +-inf in column INF (one product of at least 2^128 in each element) and NaN in column NAN, and their product."""
    o = Operands(M, N, K, trans, M + N, std=0.3, lo=122, hi=128)
    k = K - 5
    o.a[:, k] = torch.where(torch.arange(M) % 2 == 0, 0x7E, 0xFE).to(torch.uint8)          # +-448
    o.sa[k // 128, :M] = 127
    b = o.b if trans else o.b.t()
    b[INF] = 0
    b[INF, k] = 0x7E
    b[NAN, 3] = 0x7F
    o.sb[:, INF] = 254
    A = R.decode(o.a) * R.per_element(o.sa, M, K)
    B = (R.decode(o.b) * R.per_element(o.sb, N, K)).t() if trans else R.decode(o.b) * R.per_element_down(o.sb, K, N)
    v = A @ B.contiguous()
    v[:, INF] = torch.where(torch.arange(M) % 2 == 0, float("inf"), -float("inf"))
    o.w = o.workspace() if ws else None
    assert (o.w is not None) == ws
    return o, v


def check(q, s, want, what):
    """As Q8Out.check of test_gpu_scaled, on the finite values; the others are NaN."""
    M, W = want.shape
    fin = torch.isfinite(want)
    got_s = s.cpu().long()
    m = torch.zeros(M, R.blocks(W) * 128, dtype=torch.float64)
    m[:, :W] = R.magnitude(want)
    amax = m.reshape(M, -1, 128).amax(2).t()
    assert ((got_s >= R.scale_byte(amax * 0.999)) & (got_s <= R.scale_byte(amax * 1.001))).all(), what + ": scales"
    per, v = R.per_element(got_s, M, W), R.decode(q.cpu())
    assert torch.equal(torch.isnan(v), ~fin), what + ": NaN"
    finite = torch.where(fin, want, torch.zeros_like(want))
    bound = torch.maximum(finite.abs() * 2.0 ** -4, per * 2.0 ** -10) + 1e-3 * finite.square().mean(1, keepdim=True).sqrt()
    assert ((v * per - want).abs() <= bound)[fin].all(), what


@pytest.fixture(params=[(s, t) for s in SHAPES for t in (True, False)], ids=lambda p: "%dx%dx%d-%s" % (p[0][:3] + ("NK" if p[1] else "KN",)))
def operands(request):
    (M, N, K, ws), trans = request.param
    return overflowing(M, N, K, trans, ws)


def test_the_product_overflows(operands):
    o, v = operands
    D = torch.empty(o.M, o.N, device="cuda")
    o.run([coda.store(D, f32=True)], workspace=o.w)
    D = D.cpu().double()
    assert torch.equal(D[:, INF], v[:, INF]) and torch.isnan(D[:, NAN]).all()
    rest = torch.ones(o.N, dtype=torch.bool)
    rest[[INF, NAN]] = False
    assert torch.isfinite(D[:, rest]).all()


def test_store_q8(operands):
    o, v = operands
    (q, q_ok), (s, s_ok) = guarded(o.M, o.N), guarded(R.blocks(o.N), o.M)
    o.run([coda.store_q8(q, s)], workspace=o.w)
    q_ok(); s_ok()
    check(q, s, v, "store_q8")


def test_swiglu_forward_q8(operands):
    o, v = operands
    (z, z_ok), (zs, zs_ok) = guarded(o.M, o.N), guarded(R.blocks(o.N), o.M)
    (h, h_ok), (hs, hs_ok) = guarded(o.M, o.N // 2), guarded(R.blocks(o.N // 2), o.M)
    o.run([coda.swiglu_fwd_q8(z, zs), coda.store_q8(h, hs)], workspace=o.w)
    for ok in (z_ok, zs_ok, h_ok, hs_ok):
        ok()
    check(z, zs, v, "Z")
    check(h, hs, R.swiglu(v), "H")


def test_swiglu_backward_q8(operands):
    o, v = operands
    M, N = o.M, o.N
    zq, zs = R.random_codes(o.g, (M, 2 * N), 60.0), R.random_scales(o.g, R.blocks(2 * N), M, 118, 122)
    (q, q_ok), (s, s_ok) = guarded(M, 2 * N), guarded(R.blocks(2 * N), M)
    o.run([coda.swiglu_bwd_q8(zq.cuda(), zs.cuda()), coda.store_q8(q, s)], workspace=o.w)
    q_ok(); s_ok()
    check(q, s, R.swiglu_bwd(v, R.decode(zq) * R.per_element(zs, M, 2 * N)), "dZ")
