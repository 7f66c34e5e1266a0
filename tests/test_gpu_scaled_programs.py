"""Every program on products of 8-bit operands with block scales, on every kind of kernel that may run it, on the GPU.  References in 64 bits.  Tolerances: those of
the other tests of these products (test_gpu_scaled)."""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import gpu_util as G
from tests import q8_ref as R
from tests.test_gpu_scaled import Q8Out, assert_near
from tests.test_gpu_scaled_large import OnDevice

pytestmark = pytest.mark.gpu

# Divided, in tiles of 32, 64 and 128 rows: rows and columns that end inside the four rows and the 256 columns of a workgroup of the second kernel, in an odd half
# block of 128 and inside the wave's columns
DIVIDED = [(5, 288, 4096), (33, 288, 3088), (70, 544, 2064), (257, 800, 2576)]

# Undivided: 128 x 256 tiles; 256 x 256 tiles, ragged and whole (instances of their own)
HALF = [(300, 800, 400), (256, 512, 256)]
LARGE = [(2064, 4128, 400), (2304, 4096, 640)]

SHAPES = [s + (True,) for s in DIVIDED] + [s + (False,) for s in HALF + LARGE]


@pytest.fixture(params=[(s, t) for s in SHAPES for t in (True, False)], ids=lambda p: "%dx%dx%d-%s-%s" % (p[0][:3] + ("ws" if p[0][3] else "none", "NK" if p[1] else "KN")))
def operands(request):
    def make(std=1.0, lo=118, hi=132):
        (M, N, K, ws), trans = request.param
        o = OnDevice(M, N, K, trans, M + K, std, lo, hi)
        o.ws = o.workspace() if ws else None
        assert (o.ws is not None) == ws                      # the sizes are divided
        return o
    return make


def test_residual_and_row_sums(operands):
    o = operands()
    M, N = o.M, o.N
    r = torch.rand(M, generator=o.g) + 0.5
    C, gamma = torch.randn(M, N, generator=o.g).to(torch.bfloat16), torch.rand(N, generator=o.g) + 0.5
    part = torch.full((coda.coda_row_partial_blocks(N), M), G.SENTINEL_F32, device="cuda")
    D, side = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16)
    o.run([coda.row_scale(r.cuda()), coda.add_tile(C.cuda()), coda.row_sumsq(part), coda.col_scale_side(gamma.cuda(), side.t), coda.store(D.t)], workspace=o.ws)
    v, noise = o.product() * r.double()[:, None] + C.double(), o.noise() * r.double()[:, None]
    for x in (D, side):
        x.check_guards(); x.written()
    assert_near(D.t, v, noise, "residual")
    assert_near(side.t, v * gamma.double(), noise * gamma.double(), "side")
    G.assert_sumsq_close(part.sum(0).cpu().double().numpy(), (v * v).sum(1).numpy(), "row sums")


def test_rope(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N, v = o.M, o.N, o.product()
    T, hd = 64, 48
    cols = N // 2 // hd * hd
    ang, pos = torch.rand(T, hd // 2, generator=o.g) * 6.28, torch.randint(0, T, (M,), generator=o.g).to(torch.int32)
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.rope(ang.cos().cuda(), ang.sin().cuda(), pos.cuda(), hd, cols), coda.store(D.t)], workspace=o.ws)
    want = v.clone()
    c, s = (f.double()[pos.long()].repeat(1, cols // hd) for f in (ang.cos(), ang.sin()))
    x0, x1 = v[:, 0:cols:2], v[:, 1:cols:2]
    want[:, 0:cols:2], want[:, 1:cols:2] = x0 * c - x1 * s, x0 * s + x1 * c
    D.check_guards(); D.written()
    G.assert_bf16_close(G.host_f64(D.t), want.numpy(), "rope")


def test_log_sum_exp_and_fp32_store(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N, v = o.M, o.N, o.product()
    y = torch.randint(0, N, (M,), generator=o.g).to(torch.int32)
    nblk = coda.coda_row_partial_blocks(N)
    pm, ps, zt, lse = (torch.empty(nblk, M, device="cuda"), torch.empty(nblk, M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"))
    F = G.Guarded(M, N, torch.float32)
    o.run([coda.lse_partial(y.cuda(), pm, ps, zt), coda.store(F.t, f32=True)], workspace=o.ws)
    coda.coda_lse_finalize(pm, ps, M, nblk, ztgt=zt, lse_out=lse)
    F.check_guards(); F.written()
    G.assert_f32_signed_close(G.host_f64(F.t), v.numpy(), "fp32 store")
    G.assert_f32_signed_close(G.host_f64(lse), torch.logsumexp(v, 1).numpy(), "log-sum-exp")
    G.assert_f32_signed_close(G.host_f64(zt), v[torch.arange(M), y.long()].numpy(), "target")


def test_swiglu_forward(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N = o.M, o.N
    r = torch.rand(M, generator=o.g) + 0.5
    Z, H = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N // 2, torch.bfloat16)
    o.run([coda.row_scale(r.cuda()), coda.swiglu_fwd(Z.t), coda.store(H.t)], workspace=o.ws)
    z = o.product() * r.double()[:, None]
    for x in (Z, H):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(Z.t), z.numpy(), "pre-activation")
    G.assert_bf16_close(G.host_f64(H.t), R.swiglu(z).numpy(), "swiglu")


def test_swiglu_backward(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N, v = o.M, o.N, o.product()
    saved = torch.randn(M, 2 * N, generator=o.g).to(torch.bfloat16)
    dZ, act = G.Guarded(M, 2 * N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16)
    stat = torch.empty(coda.coda_row_partial_blocks(N), M, device="cuda")
    o.run([coda.swiglu_bwd(saved.cuda(), act_out=act.t, stat_out=stat), coda.store(dZ.t)], workspace=o.ws)
    want = R.swiglu_bwd(v, saved.double())
    for x in (dZ, act):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(dZ.t), want.numpy(), "swiglu backward")
    G.assert_bf16_close(G.host_f64(act.t), R.swiglu(saved.double()).numpy(), "activation")
    G.assert_f32_signed_close(stat.sum(0).cpu().double().numpy(), (want * saved.double()).sum(1).numpy(), "row statistic")


def test_rmsnorm_backward(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N, v = o.M, o.N, o.product()
    C, res = torch.randn(M, N, generator=o.g).to(torch.bfloat16), torch.randn(M, N, generator=o.g).to(torch.bfloat16)
    r, zz, gamma = torch.rand(M, generator=o.g) + 0.5, torch.randn(M, generator=o.g), torch.rand(N, generator=o.g) + 0.5
    out, cout = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16)
    dgp, dg = torch.empty(coda.coda_col_partial_blocks(M), N, device="cuda"), torch.empty(N, device="cuda")
    o.run([coda.rmsnorm_bwd(C.cuda(), r.cuda(), zz.cuda(), gamma.cuda(), c_out=cout.t, dgamma_out=dgp), coda.add_tile(res.cuda()), coda.store(out.t)], workspace=o.ws)
    coda.coda_col_finalize(dgp, N, dgp.shape[0], dg)
    cn = C.double() * r.double()[:, None]
    for x in (out, cout):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(out.t), (res.double() + (v * gamma.double() - cn * zz.double()[:, None]) * r.double()[:, None]).numpy(), "rmsnorm backward")
    G.assert_bf16_close(G.host_f64(cout.t), (cn * gamma.double()).numpy(), "normalised")
    G.assert_f32_signed_close(G.host_f64(dg), (v * cn).sum(0).numpy(), "dgamma")


def test_store_q8(operands):
    o = operands()
    r = torch.rand(o.M, generator=o.g) + 0.5
    out = Q8Out(o.M, o.N)
    o.run([coda.row_scale(r.cuda()), coda.store_q8(out.q, out.s)], workspace=o.ws)
    out.check(o.product() * r.double()[:, None], "store_q8")


def test_swiglu_forward_q8(operands):
    o = operands(std=0.3, lo=122, hi=128)
    M, N = o.M, o.N
    r = torch.rand(M, generator=o.g) + 0.5
    scale = coda.row_scale(r.cuda())
    H, Z, alone = Q8Out(M, N // 2), Q8Out(M, N), Q8Out(M, N // 2)
    o.run([scale, coda.swiglu_fwd_q8(Z.q, Z.s), coda.store_q8(H.q, H.s)], workspace=o.ws)
    z = o.product() * r.double()[:, None]
    H.check(R.swiglu(z), "H"); Z.check(z, "Z")
    o.run([scale, coda.swiglu_fwd_q8(), coda.store_q8(alone.q, alone.s)], workspace=o.ws)
    assert torch.equal(alone.q, H.q) and torch.equal(alone.s, H.s)


def test_swiglu_backward_q8(operands):
    o = operands()
    M, N = o.M, o.N
    zq, zs = R.random_codes(o.g, (M, 2 * N), 60.0), R.random_scales(o.g, R.blocks(2 * N), M, 118, 122)
    z = R.decode(zq) * R.per_element(zs, M, 2 * N)
    dZ, part = Q8Out(M, 2 * N), torch.zeros(coda.coda_row_partial_blocks(N), M, device="cuda")
    o.run([coda.swiglu_bwd_q8(zq.cuda(), zs.cuda(), stat_out=part), coda.store_q8(dZ.q, dZ.s)], workspace=o.ws)
    want = R.swiglu_bwd(o.product(), z)
    dZ.check(want, "dZ")
    G.assert_f32_signed_close(part.sum(0).cpu().double().numpy(), (want * z).sum(1).numpy(), "row statistic")
