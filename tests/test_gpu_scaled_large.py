"""Products of 8-bit operands with block scales in 256 x 256 tiles and for few rows, gradients in 256 x 256 tiles, and operands that pass 2^31 bytes, on the
GPU.  References in 64 bits, on the GPU too.  Tolerances: those of the other tests of these products (test_gpu_scaled); bytes and exact sums are compared as
they are."""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import gpu_util as G
from tests import q8_ref as R
from tests.test_gpu_scaled import Operands, Q8Out, assert_near

pytestmark = pytest.mark.gpu


class OnDevice(Operands):
    """The same operands, their 64-bit product on the GPU."""

    def product(self):
        if not hasattr(self, "v"):
            a, b = self.A.cuda(), self.B.cuda()
            self.v, self.n = (a @ b).cpu(), 1e-3 * (a.square() @ b.square()).sqrt().cpu()
        return self.v

    def noise(self):
        self.product()
        return self.n


# more than 256 tiles of 128 x 256: ragged, whole; K of a chunk, one block, two (one pair), three, five, nine, ten and seventeen
LARGE = [(2064, 4112, 16), (2064, 4112, 128), (2064, 4112, 400), (2056, 4368, 1168), (2304, 4096, 256), (2304, 4096, 640), (2304, 4096, 1280), (2304, 4096, 2176),
         (4609, 2064, 2064)]


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("trans", [True, False])
def test_large_tiles_plain_store(M, N, K, trans):
    o = OnDevice(M, N, K, trans, M + K)
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.store(D.t)])
    D.check_guards(); D.written()
    assert_near(D.t, o.product(), o.noise(), "scaled product")


@pytest.mark.parametrize("M,N,K", [(2064, 4112, 400), (2304, 4096, 640)])
@pytest.mark.parametrize("trans", [True, False])
def test_large_tiles_every_block_has_its_scale(M, N, K, trans):
    one = R.codes_of(torch.ones(1, dtype=torch.float64))
    o = Operands(M, N, K, trans, 3)
    nb = R.blocks(K)
    for blk in range(nb):
        o.a = torch.zeros(M, K, dtype=torch.uint8)
        o.a[:, blk * 128:(blk + 1) * 128] = one
        o.b = one.expand(*o.b.shape).contiguous()
        o.sa[:, :M] = (120 + torch.arange(M) % 5).to(torch.uint8)
        o.sb[:, :N] = (125 + torch.arange(N) % 3).to(torch.uint8)
        o.sa[blk, :M] += 7
        o.sb[blk, :N] += 4
        D = torch.empty(M, N, device="cuda")
        o.run([coda.store(D, f32=True)])
        n = min(128, K - blk * 128)
        want = n * R.scale(o.sa[blk, :M].long())[:, None] * R.scale(o.sb[blk, :N].long())[None, :]
        assert torch.equal(D.cpu().double(), want)


@pytest.mark.parametrize("M,N,K", [(2064, 4112, 400), (2304, 4096, 640)])
def test_large_tiles_programs(M, N, K):
    o = OnDevice(M, N, K, True, 31)
    r = torch.rand(M, generator=o.g) + 0.5
    C = torch.randn(M, N, generator=o.g).to(torch.bfloat16)
    part = torch.full((coda.coda_row_partial_blocks(N), M), G.SENTINEL_F32, device="cuda")
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.row_scale(r.cuda()), coda.add_tile(C.cuda()), coda.row_sumsq(part), coda.store(D.t)])
    v, noise = o.product() * r.double()[:, None], o.noise() * r.double()[:, None]
    D.check_guards(); D.written()
    assert_near(D.t, v + C.double(), noise, "residual")
    G.assert_sumsq_close(part.sum(0).cpu().double().numpy(), ((v + C.double()) ** 2).sum(1).numpy(), "row sums")
    out = Q8Out(M, N)
    o.run([coda.row_scale(r.cuda()), coda.store_q8(out.q, out.s)])
    out.check(v, "store_q8")


@pytest.mark.parametrize("M,N,K", [(2064, 4128, 400), (2304, 4096, 640)])
def test_large_tiles_swiglu_in_8_bits(M, N, K):
    o = OnDevice(M, N, K, True, 32, std=0.3, lo=122, hi=128)
    H, Z = Q8Out(M, N // 2), Q8Out(M, N)
    o.run([coda.swiglu_fwd_q8(Z.q, Z.s), coda.store_q8(H.q, H.s)])
    H.check(R.swiglu(o.product()), "H"); Z.check(o.product(), "Z")
    alone = Q8Out(M, N // 2)
    o.run([coda.swiglu_fwd_q8(), coda.store_q8(alone.q, alone.s)])
    assert torch.equal(alone.q, H.q) and torch.equal(alone.s, H.s)
    o = OnDevice(M, N, K, False, 33)
    zq, zs = R.random_codes(o.g, (M, 2 * N), 60.0), R.random_scales(o.g, R.blocks(2 * N), M, 118, 122)
    z = R.decode(zq) * R.per_element(zs, M, 2 * N)
    dZ, part = Q8Out(M, 2 * N), torch.zeros(coda.coda_row_partial_blocks(N), M, device="cuda")
    o.run([coda.swiglu_bwd_q8(zq.cuda(), zs.cuda(), stat_out=part), coda.store_q8(dZ.q, dZ.s)])
    want = R.swiglu_bwd(o.product(), z)
    dZ.check(want, "dZ")
    G.assert_f32_signed_close(part.sum(0).cpu().double().numpy(), (want * z).sum(1).numpy(), "row statistic")


# 1 to 32 rows: 16 and 32 columns to a workgroup, one and two sets of rows; fewer blocks than waves, as many, a few more, rounds of four; short last blocks
FEW = [(1, 16, 16), (1, 4112, 128), (2, 4096, 1040), (7, 528, 3984), (8, 8192, 1024), (15, 2064, 4112), (16, 6160, 1168), (17, 784, 5008), (24, 4624, 256), (32, 2048, 4096),
       (32, 8208, 400)]


@pytest.mark.parametrize("M,N,K", FEW)
@pytest.mark.parametrize("ws", [True, False])
def test_few_rows(M, N, K, ws):
    o = OnDevice(M, N, K, True, M + N)
    r = torch.rand(M, generator=o.g) + 0.5
    C, gamma = torch.randn(M, N, generator=o.g).to(torch.bfloat16), torch.rand(N, generator=o.g) + 0.5
    w = o.workspace() if ws else None
    D, side, F = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N, torch.float32)
    o.run([coda.row_scale(r.cuda()), coda.add_tile(C.cuda()), coda.col_scale_side(gamma.cuda(), side.t), coda.store(D.t)], workspace=w)
    v, noise = o.product() * r.double()[:, None], o.noise() * r.double()[:, None]
    for x in (D, side):
        x.check_guards(); x.written()
    assert_near(D.t, v + C.double(), noise, "residual")
    assert_near(side.t, (v + C.double()) * gamma.double(), noise * gamma.double(), "side")
    o.run([coda.store(F.t, f32=True)], workspace=w)
    F.check_guards(); F.written()
    assert ((F.t.cpu().double() - o.product()).abs() <= o.noise()).all()
    in_place = C.cuda()
    o.run([coda.row_scale(r.cuda()), coda.add_tile(in_place), coda.store(in_place)], workspace=w)
    assert torch.equal(in_place, D.t)


@pytest.mark.parametrize("M,N,K", [(1, 6144, 1024), (9, 528, 400), (30, 4224, 528)])
@pytest.mark.parametrize("ws", [True, False])
def test_few_rows_rope_and_swiglu(M, N, K, ws):
    o = OnDevice(M, N, K, True, 41, std=0.3, lo=122, hi=128)
    w, v = o.workspace() if ws else None, o.product()
    T, hd = 64, 48
    cols = N // 2 // hd * hd
    ang, pos = torch.rand(T, hd // 2, generator=o.g) * 6.28, torch.randint(0, T, (M,), generator=o.g).to(torch.int32)
    D = G.Guarded(M, N, torch.bfloat16)
    o.run([coda.rope(ang.cos().cuda(), ang.sin().cuda(), pos.cuda(), hd, cols), coda.store(D.t)], workspace=w)
    want = v.clone()
    c, s = (f.double()[pos.long()].repeat(1, cols // hd) for f in (ang.cos(), ang.sin()))
    x0, x1 = v[:, 0:cols:2], v[:, 1:cols:2]
    want[:, 0:cols:2], want[:, 1:cols:2] = x0 * c - x1 * s, x0 * s + x1 * c
    D.check_guards(); D.written()
    G.assert_bf16_close(G.host_f64(D.t), want.numpy(), "rope")
    Z, H = G.Guarded(M, N, torch.bfloat16), G.Guarded(M, N // 2, torch.bfloat16)
    o.run([coda.swiglu_fwd(Z.t), coda.store(H.t)], workspace=w)
    for x in (Z, H):
        x.check_guards(); x.written()
    G.assert_bf16_close(G.host_f64(Z.t), v.numpy(), "pre-activation")
    G.assert_bf16_close(G.host_f64(H.t), R.swiglu(v).numpy(), "swiglu")
    only = torch.empty(M, N // 2, dtype=torch.bfloat16, device="cuda")
    o.run([coda.swiglu_fwd(), coda.store(only)], workspace=w)
    assert torch.equal(only, H.t)


# at least 128 tiles of 256 x 256 and more than 256 tokens
@pytest.mark.parametrize("M,N,K", [(2048, 4096, 320), (2064, 4112, 333), (4112, 2064, 1000), (2048, 4096, 257)])
@pytest.mark.parametrize("b8", [True, False])
def test_gradient_in_large_tiles(M, N, K, b8):
    g = torch.Generator().manual_seed(M + K)
    N = N if b8 else N + 8
    a, sa = R.random_codes(g, (K, M)), R.random_scales(g, R.blocks(M), K)
    A = (R.decode(a) * R.per_element(sa, K, M)).cuda()
    b, sb = (R.random_codes(g, (K, N)), R.random_scales(g, R.blocks(N), K)) if b8 else (torch.randn(K, N, generator=g).to(torch.bfloat16), None)
    B = (R.decode(b) * R.per_element(sb, K, N) if b8 else b.double()).cuda()
    G0 = torch.randn(M, N, generator=g).cuda()
    out = G.Guarded(M, N, torch.float32)
    out.t.copy_(G0)
    coda.coda_grad_scaled(a.cuda(), sa.cuda(), b.cuda(), sb.cuda() if b8 else None, out.t)
    out.check_guards()
    want, size = A.t().contiguous() @ B + G0.double(), A.abs().t().contiguous() @ B.abs() + G0.double().abs()
    err = (out.t.double() - want).abs()
    assert (err <= (K + 1) * 2.0 ** -24 * size).all()
    assert err.norm() <= 1e-6 * want.norm()


# ---------------------------------------------------------------- operands of more than 2^31 bytes
ROWS, COLS = 140016, 16384


def codes(rows, cols, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (rows, cols), dtype=torch.uint8, device="cuda", generator=g).bitwise_and_(0xFE)          # no NaN


def scales(nb, rows, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(118, 132, (nb, (rows + 15) // 16 * 16), dtype=torch.uint8, device="cuda", generator=g)


def value(q, s):
    q, s = q.cpu(), s.cpu()
    return R.decode(q) * R.per_element(s, *q.shape)


def test_offsets_past_32_bits_of_products():
    tall, st = codes(ROWS, COLS, 1), scales(COLS // 128, ROWS, 2)
    flat, sf = codes(48, COLS, 3), scales(COLS // 128, 48, 4)
    ends = torch.cat([torch.arange(8), torch.arange(ROWS - 8, ROWS)]).cuda()
    t64, f64 = value(tall[ends], st[:, ends]), value(flat, sf)
    want, noise = f64 @ t64.t(), 1e-3 * (f64.square() @ t64.square().t()).sqrt()
    for M in (3, 48):                                        # the tall one is B: few rows in one kernel, partials, tiles
        for ws in (True, False):
            need = coda.coda_gemm_scaled_workspace_bytes(M, ROWS, COLS)
            D = torch.empty(M, ROWS, dtype=torch.bfloat16, device="cuda")
            coda.coda_gemm_scaled(flat[:M], sf, tall, st, [coda.store(D)], transB=True, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if ws and need else None)
            assert_near(D[:, ends], want[:M], noise[:M], "tall B, %d rows" % M)
    wide = torch.empty(ROWS, COLS, dtype=torch.bfloat16, device="cuda")
    coda.coda_gemm_scaled(tall, st, flat, sf, [coda.store(wide[:, :48])], transB=True)
    assert_near(wide[ends, :48], want.t(), noise.t(), "tall A")
    q, s = torch.empty(ROWS, COLS, dtype=torch.uint8, device="cuda"), scales(1, ROWS)
    coda.coda_gemm_scaled(tall, st, flat, sf, [coda.store_q8(q[:, :48], s)], transB=True)
    got, per = value(q[ends, :48], s[:, ends]), R.per_element(s[:, ends].cpu(), 16, 48)
    bound = torch.maximum(want.t().abs() * 2.0 ** -4, per * 2.0 ** -10) + noise.t()
    assert ((got - want.t()).abs() <= bound).all()


def test_offsets_past_32_bits_of_conversions():
    X = torch.empty(ROWS, COLS, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    q, s, s2 = torch.empty(ROWS, COLS, dtype=torch.uint8, device="cuda"), scales(COLS // 128, ROWS), scales((ROWS + 127) // 128, COLS)
    last = slice(ROWS - 112, ROWS)                           # 140016 = 1093 * 128 + 112
    part, ps, ps2 = torch.empty(112, COLS, dtype=torch.uint8, device="cuda"), scales(COLS // 128, 112), scales(1, COLS)
    for square in (False, True):
        coda.coda_quantize(X, q, s, scales_t=s2 if square else None, square=square)
        coda.coda_quantize(X[last], part, ps, scales_t=ps2 if square else None, square=square)
        assert torch.equal(q[last], part) and torch.equal(s[:, last], ps)
        if square:
            assert torch.equal(s2[-1:], ps2)
    coda.coda_quantize(X, q, s)
    coda.coda_dequantize(q, s, X)
    assert torch.equal(X[last].cpu().double(), value(q[last], s[:, last]).to(torch.bfloat16).double())


@pytest.mark.parametrize("N", [16, 528])
def test_offsets_past_32_bits_of_gradients(N):
    """Tokens of zeros in front; behind them ones, halves and twos, whose sums are exact."""
    A, sa = torch.zeros(ROWS, COLS, dtype=torch.uint8, device="cuda"), torch.full((COLS // 128, ROWS), 127, dtype=torch.uint8, device="cuda")
    B, sb = torch.zeros(ROWS, N, dtype=torch.uint8, device="cuda"), torch.full(((N + 127) // 128, ROWS), 127, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    few = torch.tensor([0x30, 0x38, 0x40, 0xB8], dtype=torch.uint8, device="cuda")
    A[-100:] = few[torch.randint(0, 4, (100, COLS), device="cuda", generator=g)]
    B[-100:] = few[torch.randint(0, 4, (100, N), device="cuda", generator=g)]
    sa[:, -50:] = 129
    want = value(A[-100:], sa[:, -100:]).t() @ value(B[-100:], sb[:, -100:])
    need = coda.coda_grad_scaled_workspace_bytes(COLS, N, ROWS)
    out = torch.zeros(COLS, N, device="cuda")
    coda.coda_grad_scaled(A, sa, B, sb, out, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    assert torch.equal(out.cpu().double(), want)


# ---------------------------------------------------------------- calls beside each other
def prepared(M, N, K, seed):
    o = Operands(M, N, K, True, seed)
    dev = [t.cuda() for t in (o.a, o.sa, o.b, o.sb)]
    D = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    return dev, D, coda.coda_gemm_scaled_workspace_bytes(M, N, K)


def multiply(dev, D, workspace, stream=None):
    coda.coda_gemm_scaled(*dev, [coda.store(D)], transB=True, workspace=workspace, stream=stream)


def test_two_graphs_take_turns_with_one_workspace():
    calls = [prepared(96, 1024, 4096, 1), prepared(64, 2048, 2048, 2)]
    assert all(need for _, _, need in calls)
    w = torch.empty(max(need for _, _, need in calls), dtype=torch.uint8, device="cuda")
    once = []
    for dev, D, _ in calls:
        multiply(dev, D, w)
        once.append(D.clone())
    graphs = []
    for dev, D, _ in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            multiply(dev, D, w)
        graphs.append(g)
    for k in range(4):
        for _, D, _ in calls:
            D.zero_()
        for g in graphs if k % 2 else reversed(graphs):
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(D, want) for (_, D, _), want in zip(calls, once))


def test_two_streams_at_once():
    calls = [prepared(96, 1024, 4096, 1), prepared(64, 2048, 2048, 2), prepared(8, 4096, 2048, 3)]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") if need else None for _, _, need in calls]
    once = []
    for (dev, D, _), w in zip(calls, spaces):
        multiply(dev, D, w)
        once.append(D.clone())
        D.zero_()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for (dev, D, _), w, s in zip(calls, spaces, streams):
            multiply(dev, D, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(D, want) for (_, D, _), want in zip(calls, once))


def test_one_operand_twice():
    """A product of a matrix with itself, and its gradient form: the same codes and scales on both sides."""
    o = Operands(256, 256, 384, True, 5)
    a, sa = o.a.cuda(), o.sa.cuda()
    A = R.decode(o.a) * R.per_element(o.sa, 256, 384)
    D = torch.empty(256, 256, dtype=torch.bfloat16, device="cuda")
    coda.coda_gemm_scaled(a, sa, a, sa, [coda.store(D)], transB=True)
    assert_near(D, A @ A.t(), 1e-3 * (A.square() @ A.square().t()).sqrt(), "A A^T")
    out = torch.zeros(384, 384, device="cuda")
    coda.coda_grad_scaled(a, sa, a, sa, out)
    want = A.t() @ A
    assert ((out.cpu().double() - want).abs() <= 257 * 2.0 ** -24 * (A.abs().t() @ A.abs())).all() and torch.equal(out, out.t())
