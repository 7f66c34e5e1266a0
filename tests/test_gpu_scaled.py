"""Products of 8-bit operands with block scales, their programs and the weight gradient from checkpoints, on the GPU, against 64 bits.

Tolerances.  Products are exact and scales powers of two, so what is left is the order and width of the sums and the last rounding.  Where
operands have rows and columns of very different size, bf16 outputs are held to half a step, 2^-8 of the value, beside 1e-3 of the root of
the sum of the squared products of the element: for independent products that root is what an element has of the result's 2-norm, and
the sums of the 8-bit instructions are off by 1.3e-5 of that, so 1e-3 is 75 times its expectation.  (The fixed 1e-2 of gpu_util's bound
for bf16 is not for those: with products of up to 2^14 an element near zero is off by more.)  The others, and fp32 sums, are held to the bounds
of the other GEMM tests (gpu_util).  Codes: half a step of
E4M3, 2^-4 of the value or 2^-10 of the scale, beside 1e-3 of the row's rms for the sums; the scale itself may be the neighbour's where the
block's largest value is within 1e-3 of a border.  Gradients (bf16 instructions, K fp32 additions of exact products, and the one to G):
(K + 1) 2^-24 of the sum of magnitudes, and 1e-6 of the 2-norm (sqrt(K) rounding errors of 2^-25 add up to under 1e-6 for K <= 1000).
"""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import gpu_util as G
from tests import q8_ref as R
from tests.test_gpu_q8 import guarded

pytestmark = pytest.mark.gpu


class Operands:
    def __init__(self, M, N, K, trans, seed, std=1.0, lo=118, hi=132):
        g = torch.Generator().manual_seed(seed)
        self.M, self.N, self.K, self.trans = M, N, K, trans
        self.a = R.random_codes(g, (M, K), std)
        self.b = R.random_codes(g, (N, K) if trans else (K, N), std)
        nb = R.blocks(K)
        self.sa, self.sb = R.random_scales(g, nb, M, lo, hi), R.random_scales(g, nb, N, lo, hi)
        self.A = R.decode(self.a) * R.per_element(self.sa, M, K)
        if trans:
            self.B = (R.decode(self.b) * R.per_element(self.sb, N, K)).t().contiguous()
        else:
            self.B = R.decode(self.b) * R.per_element_down(self.sb, K, N)
        self.g = g

    def product(self):
        return self.A @ self.B

    def noise(self):
        """What the sums of an element may be off by (above)."""
        return 1e-3 * (self.A.square() @ self.B.square()).sqrt()

    def run(self, ops, workspace=None, stream=None):
        pad = torch.zeros(self.a.shape[0], self.a.shape[1] + 32, dtype=torch.uint8)
        pad[:, :self.K] = self.a
        self.dev = [pad.cuda()[:, :self.K], self.sa.cuda(), self.b.cuda(), self.sb.cuda()]
        a, sa, b, sb = self.dev
        coda.coda_gemm_scaled(a, sa, b, sb, ops, transB=self.trans, workspace=workspace, stream=stream)
        torch.cuda.synchronize()

    def workspace(self):
        need = coda.coda_gemm_scaled_workspace_bytes(self.M, self.N, self.K)
        return torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None


def assert_near(got, ref, noise, what):
    err = (got.cpu().double() - ref).abs()
    bad = ~(err <= ref.abs() * 2.0 ** -8 + noise * (1 + 2.0 ** -8))
    assert not bad.any(), "%s: %d elements off, the worst by %.3g" % (what, int(bad.sum()), float(err.max()))


# (M, N, K): one row, few rows, ragged everywhere, whole tiles, K of one chunk, one block, several, a short last block
SHAPES = [(1, 16, 16), (1, 272, 4096), (3, 144, 400), (31, 256, 128), (33, 528, 1040), (64, 1024, 2048), (65, 272, 784), (130, 400, 256), (256, 256, 384),
          (257, 512, 1168), (300, 784, 2064), (512, 768, 640), (513, 1040, 144), (1000, 2304, 272)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("ws", [True, False])
def test_plain_store(M, N, K, trans, ws):
    o = Operands(M, N, K, trans, M + N + K)
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.store(D.t)], workspace=o.workspace() if ws else None)
    D.check_guards(); D.written()
    assert_near(D.t, o.product(), o.noise(), "scaled product")


@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("M", [5, 300])
def test_every_block_has_its_scale(M, trans):
    """Ones in one block of 128 of the contraction at a time, scales that name block, row and column: the sums are exact."""
    N, K = 272, 1168
    nb = R.blocks(K)
    one = R.codes_of(torch.ones(1, dtype=torch.float64))
    for blk in (0, 1, 4, nb - 1):
        o = Operands(M, N, K, trans, 3)
        o.a = torch.zeros(M, K, dtype=torch.uint8)
        o.a[:, blk * 128:(blk + 1) * 128] = one
        o.b = one.expand(*o.b.shape).contiguous()
        o.sa[:, :M] = (120 + torch.arange(M) % 5).to(torch.uint8)
        o.sb[:, :N] = (125 + torch.arange(N) % 3).to(torch.uint8)
        o.sa[blk, :M] += 7
        o.sb[blk, :N] += 4
        D = torch.empty(M, N, device="cuda")
        o.run([coda.store(D, f32=True)], workspace=o.workspace())
        n = min(128, K - blk * 128)
        want = n * R.scale(o.sa[blk, :M].long())[:, None] * R.scale(o.sb[blk, :N].long())[None, :]
        assert torch.equal(D.cpu().double(), want)


@pytest.mark.parametrize("lo,hi", [(1, 1), (0, 0), (254, 254)])
def test_extreme_scales(lo, hi):
    """2^-126 and 2^-127 against 2^100, 2^127 against 2^-120: the instruction takes every byte for the power of two that it stands for."""
    o = Operands(40, 32, 256, True, 5)
    o.sa[:, :40] = lo
    o.sb[:, :32] = 227 if lo < 2 else 7
    o.A = R.decode(o.a) * R.per_element(o.sa, 40, 256)
    o.B = (R.decode(o.b) * R.per_element(o.sb, 32, 256)).t().contiguous()
    D = torch.empty(40, 32, device="cuda")
    o.run([coda.store(D, f32=True)])
    G.assert_f32_signed_close(G.host_f64(D), o.product().numpy(), "scale %d" % lo)


def test_nan_scales_and_codes_stay_in_their_row_and_column():
    for ws in (True, False):
        o = Operands(70, 48, 400, True, 6)
        o.sa[1, 7] = 255
        o.sb[2, 9] = 255
        o.a[11, 3] = 0x7F
        D = torch.empty(70, 48, dtype=torch.bfloat16, device="cuda")
        o.run([coda.store(D)], workspace=o.workspace() if ws else None)
        got, want = torch.isnan(D.cpu()), torch.zeros(70, 48, dtype=torch.bool)
        want[7] = want[11] = True
        want[:, 9] = True
        assert torch.equal(got, want)


def test_no_contraction_runs_the_program_on_zero():
    R_ = torch.randn(5, 32, device="cuda").to(torch.bfloat16)
    D = torch.empty(5, 32, dtype=torch.bfloat16, device="cuda")
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    coda.coda_gemm_scaled(u(5, 16)[:, :0], u(1, 16), u(32, 16)[:, :0], u(1, 32), [coda.add_tile(R_), coda.store(D)], transB=True)
    assert torch.equal(D, R_)
    q, s = torch.full((5, 32), 9, dtype=torch.uint8, device="cuda"), u(1, 16)
    coda.coda_gemm_scaled(u(5, 16)[:, :0], u(1, 16), u(32, 16)[:, :0], u(1, 32), [coda.store_q8(q, s)], transB=True)
    assert bool((q == 0).all()) and bool((s[0, :5] == 1).all())


@pytest.mark.parametrize("M,N,K", [(3, 144, 400), (64, 1024, 2048), (300, 784, 400), (513, 1040, 256)])
@pytest.mark.parametrize("ws", [True, False])
def test_linear_program(M, N, K, ws):
    o = Operands(M, N, K, True, 11)
    r = torch.rand(M, generator=o.g) + 0.5
    C = torch.randn(M, N, generator=o.g).to(torch.bfloat16)
    gamma = torch.rand(N, generator=o.g) + 0.5
    nblk = coda.coda_row_partial_blocks(N)
    D, side, part = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16), torch.full((nblk, M), G.SENTINEL_F32, device="cuda")
    keep = [r.cuda(), C.cuda(), gamma.cuda()]
    o.run([coda.row_scale(keep[0]), coda.add_tile(keep[1]), coda.row_sumsq(part), coda.col_scale_side(keep[2], side.t), coda.store(D.t)],
          workspace=o.workspace() if ws else None)
    v = o.product() * r.double()[:, None] + C.double()
    for x in (D, side):
        x.check_guards(); x.written()
    noise = o.noise() * r.double()[:, None]
    assert_near(D.t, v, noise, "residual")
    assert_near(side.t, v * gamma.double(), noise * gamma.double(), "side")
    G.assert_sumsq_close(part.sum(0).cpu().double().numpy(), (v * v).sum(1).numpy(), "row sums")


@pytest.mark.parametrize("M,N,K", [(3, 256, 256), (300, 512, 400)])
@pytest.mark.parametrize("ws", [True, False])
def test_rope_lse_and_fp32_store(M, N, K, ws):
    o = Operands(M, N, K, True, 12, std=0.3, lo=122, hi=128)
    w = o.workspace() if ws else None
    v = o.product()
    T, hd = 64, 64
    ang = torch.rand(T, hd // 2, generator=o.g) * 6.28
    pos = torch.randint(0, T, (M,), generator=o.g).to(torch.int32)
    cos, sin = ang.cos().cuda(), ang.sin().cuda()
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.rope(cos, sin, pos.cuda(), hd, N // 2), coda.store(D.t)], workspace=w)
    want = v.clone()
    c, s = ang.cos().double()[pos.long()].repeat(1, N // 2 // hd), ang.sin().double()[pos.long()].repeat(1, N // 2 // hd)
    x0, x1 = v[:, 0:N // 2:2], v[:, 1:N // 2:2]
    want[:, 0:N // 2:2], want[:, 1:N // 2:2] = x0 * c - x1 * s, x0 * s + x1 * c
    D.check_guards(); D.written()
    G.assert_bf16_close(G.host_f64(D.t), want.numpy(), "rope")
    y = torch.randint(0, N, (M,), generator=o.g).to(torch.int32)
    nblk = coda.coda_row_partial_blocks(N)
    pm, ps, zt, lse = (torch.empty(nblk, M, device="cuda"), torch.empty(nblk, M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"))
    F = G.Guarded(M, N, torch.float32)
    o.run([coda.lse_partial(y.cuda(), pm, ps, zt), coda.store(F.t, f32=True)], workspace=w)
    coda.coda_lse_finalize(pm, ps, M, nblk, ztgt=zt, lse_out=lse)
    F.check_guards(); F.written()
    G.assert_f32_signed_close(G.host_f64(F.t), v.numpy(), "fp32 store")
    G.assert_f32_signed_close(G.host_f64(lse), torch.logsumexp(v, 1).numpy(), "log-sum-exp")
    G.assert_f32_signed_close(G.host_f64(zt), v[torch.arange(M), y.long()].numpy(), "target")


@pytest.mark.parametrize("M,N,K", [(3, 256, 256), (300, 528, 400), (513, 1040, 256)])
@pytest.mark.parametrize("ws", [True, False])
def test_pairwise_and_rmsnorm_programs_in_bf16(M, N, K, ws):
    o = Operands(M, N, K, False, 13, std=0.3, lo=122, hi=128)
    w = o.workspace() if ws else None
    v = o.product()
    r = torch.rand(M, generator=o.g) + 0.5
    Z, H = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N // 2, torch.bfloat16)
    o.run([coda.row_scale(r.cuda()), coda.swiglu_fwd(Z.t), coda.store(H.t)], workspace=w)
    z = v * r.double()[:, None]
    for x in (Z, H):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(Z.t), z.numpy(), "pre-activation")
    G.assert_bf16_close(G.host_f64(H.t), R.swiglu(z).numpy(), "swiglu")
    saved = torch.randn(M, 2 * N, generator=o.g).to(torch.bfloat16)
    dZ, act = G.Guarded(M, 2 * N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16)
    nblk = coda.coda_row_partial_blocks(N)
    stat = torch.empty(nblk, M, device="cuda")
    o.run([coda.swiglu_bwd(saved.cuda(), act_out=act.t, stat_out=stat), coda.store(dZ.t)], workspace=w)
    want = R.swiglu_bwd(v, saved.double())
    for x in (dZ, act):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(dZ.t), want.numpy(), "swiglu backward")
    G.assert_bf16_close(G.host_f64(act.t), R.swiglu(saved.double()).numpy(), "activation")
    G.assert_f32_signed_close(stat.sum(0).cpu().double().numpy(), (want * saved.double()).sum(1).numpy(), "row statistic")
    C, res = torch.randn(M, N, generator=o.g).to(torch.bfloat16), torch.randn(M, N, generator=o.g).to(torch.bfloat16)
    zz, gamma = torch.randn(M, generator=o.g), torch.rand(N, generator=o.g) + 0.5
    out, cout = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16)
    dgp, dg = torch.empty(coda.coda_col_partial_blocks(M), N, device="cuda"), torch.empty(N, device="cuda")
    o.run([coda.rmsnorm_bwd(C.cuda(), r.cuda(), zz.cuda(), gamma.cuda(), c_out=cout.t, dgamma_out=dgp), coda.add_tile(res.cuda()), coda.store(out.t)], workspace=w)
    coda.coda_col_finalize(dgp, N, dgp.shape[0], dg)
    cn = C.double() * r.double()[:, None]
    for x in (out, cout):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(out.t), (res.double() + (v * gamma.double() - cn * zz.double()[:, None]) * r.double()[:, None]).numpy(), "rmsnorm backward")
    G.assert_bf16_close(G.host_f64(cout.t), (cn * gamma.double()).numpy(), "normalised")
    G.assert_f32_signed_close(G.host_f64(dg), (v * cn).sum(0).numpy(), "dgamma")


# ---------------------------------------------------------------- programs that end in 8 bits
class Q8Out:
    def __init__(self, M, W):
        self.M, self.W = M, W
        self.q, self.q_ok = guarded(M, W)
        self.s, self.s_ok = guarded(R.blocks(W), M)

    def check(self, want, what):
        self.q_ok(); self.s_ok()
        got_s = self.s.cpu().long()
        byte, _ = R.along_rows(want)
        if not torch.equal(got_s, byte):
            m = torch.zeros(self.M, R.blocks(self.W) * 128, dtype=torch.float64)
            m[:, :self.W] = want.abs()
            amax = m.reshape(self.M, -1, 128).amax(2).t()
            up, down = R.scale_byte(amax * 1.001), R.scale_byte(amax * 0.999)
            assert ((got_s >= down) & (got_s <= up)).all(), what + ": scales"
        per = R.per_element(got_s, self.M, self.W)
        got = R.decode(self.q.cpu()) * per
        noise = 1e-3 * want.square().mean(1, keepdim=True).sqrt()
        bound = torch.maximum(want.abs() * 2.0 ** -4, per * 2.0 ** -10) + noise
        bad = (got - want).abs() > bound
        assert not bad.any(), "%s: %d codes off, at %s" % (what, int(bad.sum()), bad.nonzero()[:3].tolist())


Q8_SHAPES = [(1, 32, 16), (1, 512, 4096), (5, 288, 400), (64, 1024, 2048), (70, 544, 272), (256, 512, 256), (300, 800, 400), (513, 1056, 256), (770, 4096, 144)]


@pytest.mark.parametrize("M,N,K", Q8_SHAPES)
@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("ws", [True, False])
def test_store_q8(M, N, K, trans, ws):
    o = Operands(M, N, K, trans, 21)
    r = torch.rand(M, generator=o.g) + 0.5
    out = Q8Out(M, N)
    o.run([coda.row_scale(r.cuda()), coda.store_q8(out.q, out.s)], workspace=o.workspace() if ws else None)
    out.check(o.product() * r.double()[:, None], "store_q8")


@pytest.mark.parametrize("M,N,K", Q8_SHAPES)
@pytest.mark.parametrize("save", [True, False])
@pytest.mark.parametrize("ws", [True, False])
def test_swiglu_forward_q8(M, N, K, save, ws):
    o = Operands(M, N, K, True, 22, std=0.3, lo=122, hi=128)
    r = torch.rand(M, generator=o.g) + 0.5
    H, Z = Q8Out(M, N // 2), Q8Out(M, N)
    o.run([coda.row_scale(r.cuda()), coda.swiglu_fwd_q8(Z.q, Z.s) if save else coda.swiglu_fwd_q8(), coda.store_q8(H.q, H.s)],
          workspace=o.workspace() if ws else None)
    z = o.product() * r.double()[:, None]
    H.check(R.swiglu(z), "H")
    if save:
        Z.check(z, "Z")


@pytest.mark.parametrize("M,N,K", Q8_SHAPES)
@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("stat", ["none", "partials", "atomic"])
def test_swiglu_backward_q8(M, N, K, ws, stat):
    o = Operands(M, N, K, False, 23)
    zq, zs = R.random_codes(o.g, (M, 2 * N), 60.0), R.random_scales(o.g, R.blocks(2 * N), M, 118, 122)
    z = R.decode(zq) * R.per_element(zs, M, 2 * N)
    out = Q8Out(M, 2 * N)
    part = torch.zeros(coda.coda_row_partial_blocks(N), M, device="cuda")
    op = coda.swiglu_bwd_q8(zq.cuda(), zs.cuda(), stat_out=None if stat == "none" else part, atomic=stat == "atomic")
    o.run([op, coda.store_q8(out.q, out.s)], workspace=o.workspace() if ws else None)
    want = R.swiglu_bwd(o.product(), z)
    out.check(want, "dZ")
    if stat != "none":
        got = (part.sum(0) if stat == "partials" else part[0]).cpu().double().numpy()
        G.assert_f32_signed_close(got, (want * z).sum(1).numpy(), "row statistic")


def test_infinite_and_nan_values_in_codes():
    """Infinite products and NaN become the code NaN and leave the block's scale to the others."""
    for ws in (True, False):
        o = Operands(66, 256, 128, True, 24)
        r = torch.ones(66)
        r[3] = float("nan")
        o.a[5, 0] = 0x7F
        q, s = torch.empty(66, 256, dtype=torch.uint8, device="cuda"), torch.empty(2, 80, dtype=torch.uint8, device="cuda")
        o.run([coda.row_scale(r.cuda()), coda.store_q8(q, s)], workspace=o.workspace() if ws else None)
        v = R.decode(q.cpu())
        assert torch.isnan(v[3]).all() and torch.isnan(v[5]).all() and torch.isfinite(v[6:]).all()
        assert (s[:, 3] == 1).all() and (s[:, 5] == 1).all()


# ---------------------------------------------------------------- weight gradient from checkpoints
@pytest.mark.parametrize("M,N,K", [(16, 16, 1), (32, 272, 5), (256, 256, 64), (272, 528, 129), (400, 144, 1000), (1024, 256, 333), (2048, 4096, 70)])
@pytest.mark.parametrize("b8", [True, False])
@pytest.mark.parametrize("ws", [True, False])
def test_gradient(M, N, K, b8, ws):
    g = torch.Generator().manual_seed(M + N + K)
    N = N if b8 else N + 8
    a, sa = R.random_codes(g, (K, M)), R.random_scales(g, R.blocks(M), K)
    A = R.decode(a) * R.per_element(sa, K, M)
    if b8:
        b, sb = R.random_codes(g, (K, N)), R.random_scales(g, R.blocks(N), K)
        Bv = R.decode(b) * R.per_element(sb, K, N)
    else:
        b, sb = torch.randn(K, N, generator=g).to(torch.bfloat16), None
        Bv = b.double()
    G0 = torch.randn(M, N, generator=g)
    out = G.Guarded(M, N, torch.float32)
    out.t.copy_(G0)
    need = coda.coda_grad_scaled_workspace_bytes(M, N, K)
    w = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if ws and need else None
    keep = [a.cuda(), sa.cuda(), b.cuda(), None if sb is None else sb.cuda()]
    coda.coda_grad_scaled(keep[0], keep[1], keep[2], keep[3], out.t, workspace=w)
    torch.cuda.synchronize()
    out.check_guards()
    want, size = A.t() @ Bv + G0.double(), A.abs().t() @ Bv.abs() + G0.double().abs()
    err = (out.t.cpu().double() - want).abs()
    assert (err <= (K + 1) * 2.0 ** -24 * size).all()
    assert err.norm() <= 1e-6 * want.norm()


def test_gradient_of_no_tokens_leaves_g():
    out = torch.randn(32, 48, device="cuda")
    before = out.clone()
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    coda.coda_grad_scaled(u(0, 32), u(1, 16), u(0, 48), u(1, 16), out)
    assert torch.equal(out, before)


def test_nan_in_a_checkpoint_reaches_its_rows():
    g = torch.Generator().manual_seed(4)
    a, sa, b = R.random_codes(g, (40, 256)), R.random_scales(g, 2, 40), torch.randn(40, 64, generator=g).to(torch.bfloat16)
    a[7, 9] = 0x7F
    sa[1, 3] = 255
    out = torch.zeros(256, 64, device="cuda")
    coda.coda_grad_scaled(a.cuda(), sa.cuda(), b.cuda(), None, out)
    want = torch.zeros(256, dtype=torch.bool)
    want[9] = True
    want[128:] = True
    assert torch.equal(torch.isnan(out.cpu()).all(1), want) and torch.equal(torch.isnan(out.cpu()).any(1), want)


# ---------------------------------------------------------------- together
class Mlp:
    """The MLP half of a block in 8 bits, forward and backward: what a training step keeps between passes."""

    def __init__(self, T, d, F, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.d, self.F = T, d, F
        u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
        sc = lambda nb, rows: u8(nb, (rows + 15) // 16 * 16)
        b16 = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
        self.X = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
        self.dY = (torch.randn(T, d, generator=g) * 0.01).to(torch.bfloat16).cuda()
        self.Wup = (torch.randn(2 * F, d, generator=g) * 0.05).to(torch.bfloat16).cuda()
        self.Wdown = (torch.randn(d, F, generator=g) * 0.05).to(torch.bfloat16).cuda()
        self.gamma = torch.ones(d, device="cuda")
        nb = R.blocks
        self.x, self.up, self.down = (u8(T, d), sc(nb(d), T)), (u8(2 * F, d), sc(nb(d), 2 * F), sc(nb(2 * F), d)), (u8(d, F), sc(nb(F), d), sc(nb(d), F))
        self.z, self.h, self.dy, self.dz = (u8(T, 2 * F), sc(nb(2 * F), T)), (u8(T, F), sc(nb(F), T)), (u8(T, d), sc(nb(d), T)), (u8(T, 2 * F), sc(nb(2 * F), T))
        self.xn = (u8(T, d), sc(nb(d), T))
        self.Y, self.dX, self.Xn, self.C = b16(T, d), b16(T, d), b16(T, d), b16(T, d)
        f = lambda *s: torch.empty(s, device="cuda")
        self.ss, self.rstd, self.stat, self.part = f(1, T), f(T), f(T), f(coda.coda_row_partial_blocks(F), T)
        self.dWup, self.dWdown = torch.zeros(2 * F, d, device="cuda"), torch.zeros(d, F, device="cuda")
        need = max(coda.coda_gemm_scaled_workspace_bytes(T, 2 * F, d), coda.coda_gemm_scaled_workspace_bytes(T, d, F), coda.coda_gemm_scaled_workspace_bytes(T, F, d),
                   coda.coda_gemm_scaled_workspace_bytes(T, d, 2 * F), coda.coda_grad_scaled_workspace_bytes(2 * F, d, T), coda.coda_grad_scaled_workspace_bytes(d, F, T), 16)
        self.ws = u8(need)

    def step(self):
        T, d, w = self.T, self.d, dict(workspace=self.ws)
        coda.coda_quantize(self.Wup, self.up[0], self.up[1], scales_t=self.up[2], square=True)
        coda.coda_quantize(self.Wdown, self.down[0], self.down[1], scales_t=self.down[2], square=True)
        coda.coda_row_sumsq(self.X, self.ss)
        coda.coda_row_finalize(self.ss, T, 1, rstd_out=self.rstd, d=d, eps=1e-6)
        coda.coda_quantize(self.X, *self.x)
        coda.coda_gemm_scaled(*self.x, self.up[0], self.up[1], [coda.row_scale(self.rstd), coda.swiglu_fwd_q8(*self.z), coda.store_q8(*self.h)], transB=True, **w)
        coda.coda_gemm_scaled(*self.h, self.down[0], self.down[1], [coda.add_tile(self.X), coda.store(self.Y)], transB=True, **w)
        coda.coda_quantize(self.dY, *self.dy)
        coda.coda_gemm_scaled(*self.dy, self.down[0], self.down[2], [coda.swiglu_bwd_q8(*self.z, stat_out=self.part), coda.store_q8(*self.dz)], **w)
        coda.coda_row_finalize(self.part, T, self.part.shape[0], sum_out=self.stat, d=d)
        coda.coda_grad_scaled(*self.dy, *self.h, self.dWdown, **w)
        coda.coda_dequantize(*self.x, self.C)
        coda.coda_gemm_scaled(*self.dz, self.up[0], self.up[2], [coda.rmsnorm_bwd(self.C, self.rstd, self.stat, self.gamma, c_out=self.Xn, z_sum_over=d),
                                                               coda.add_tile(self.dY), coda.store(self.dX)], **w)
        coda.coda_quantize(self.Xn, *self.xn)
        coda.coda_grad_scaled(*self.dz, *self.xn, self.dWup, **w)

    def outputs(self):
        return [self.Y, self.dX, self.dWup, self.dWdown, self.z[0], self.h[0], self.dz[0]]


def value(q, s):
    q, s = q.cpu(), s.cpu()
    return R.decode(q) * R.per_element(s, *q.shape)


@pytest.mark.parametrize("T,d,F", [(300, 256, 512), (33, 528, 784)])
def test_mlp_block_forward_and_backward_stage_by_stage(T, d, F):
    """Each stage against 64 bits on the bytes that the stage before it left."""
    m = Mlp(T, d, F)
    m.step()
    torch.cuda.synchronize()
    x, up, down = value(*m.x), value(m.up[0], m.up[1]), value(m.down[0], m.down[1])
    assert torch.equal(up, R.decode(m.up[0].cpu()) * R.per_element_down(m.up[2].cpu(), 2 * F, d))
    r = m.rstd.cpu().double()[:, None]
    z = (x @ up.t()) * r
    # values against the formula: half a step of E4M3 (2-norm: 2^-4 / sqrt(3) at the most)
    near = lambda got, want: float((got - want).norm() / want.norm()) < 2.0 ** -4 / 3 ** 0.5
    assert near(value(*m.z), z) and near(value(*m.h), R.swiglu(z))
    h = value(*m.h)
    G.assert_bf16_close(G.host_f64(m.Y), (h @ down.t() + m.X.cpu().double()).numpy(), "Y")
    dy = value(*m.dy)
    dz = R.swiglu_bwd(dy @ down, value(*m.z))
    assert near(value(*m.dz), dz)
    dzq = value(*m.dz)
    v = dzq @ up
    cn, st = value(*m.x) * r, m.stat.cpu().double()[:, None] / d
    G.assert_bf16_close(G.host_f64(m.dX), (m.dY.cpu().double() + (v - cn * st) * r).numpy(), "dX")
    for got, want in ((m.dWdown, dy.t() @ h), (m.dWup, dzq.t() @ value(*m.xn))):
        assert (got.cpu().double() - want).norm() <= 1e-6 * want.norm()


def test_gradients_against_differences():
    """The step's gradients against differences of its own loss in 64 bits without rounding to 8 bits: within the rounding of three 8-bit
    tensors along the way (2^-4 / sqrt(3) each, in quadrature under a tenth)."""
    T, d, F = 64, 256, 256
    m = Mlp(T, d, F)
    m.step()
    torch.cuda.synchronize()
    X, dY, Wup, Wdown = (t.cpu().double() for t in (m.X, m.dY, m.Wup, m.Wdown))

    def loss(X, Wup, Wdown):
        r = (X.square().mean(1, keepdim=True) + 1e-6).rsqrt()
        return float(((R.swiglu((X * r) @ Wup.t()) @ Wdown.t() + X) * dY).sum())

    g = torch.Generator().manual_seed(1)
    for got, at in ((m.dX, 0), (m.dWup, 1), (m.dWdown, 2)):
        got = got.cpu().double()
        args = [X, Wup, Wdown]
        for direction in (got, torch.randn(got.shape, generator=g, dtype=torch.float64)):
            direction = direction / direction.norm()
            eps = 1e-3
            plus, minus = [list(args), list(args)]
            plus[at], minus[at] = args[at] + eps * direction, args[at] - eps * direction
            slope = (loss(*plus) - loss(*minus)) / (2 * eps)
            assert abs(slope - float((got * direction).sum())) <= 0.1 * float(got.norm())


def test_two_passes_give_the_same_bits():
    a, b = Mlp(300, 256, 512), Mlp(300, 256, 512)
    b.ws.fill_(0x3C)
    a.step(); b.step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.outputs(), b.outputs()))


def test_captured_step_replays_on_another_stream():
    eager, m = Mlp(200, 256, 512), Mlp(200, 256, 512)
    eager.step()
    once = [t.clone() for t in eager.outputs()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(once, m.outputs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step()
    for k in range(3):
        for t in m.outputs():
            t.zero_()
        m.ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(once, m.outputs()))


def test_an_explicit_stream_is_the_one_that_runs():
    o = Operands(40, 256, 512, True, 9)
    D = torch.empty(40, 256, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    o.run([coda.store(D)], stream=s)
    assert_near(D, o.product(), o.noise(), "stream")
