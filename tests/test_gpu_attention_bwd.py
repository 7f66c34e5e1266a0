"""coda_attention_bwd against the formulas in 64 bits, and coda_attention with it against differences."""
import math

import pytest
import torch

from tests import attn_ref as R
from tests.test_gpu_attention import FILL, behind_empty, coda, device, offsets, qkv  # noqa: F401

pytestmark = pytest.mark.gpu


def tables(rows, D):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    return angle.cos().float(), angle.sin().float()


class Pass:
    """Inputs of one backward pass, the saved ones from coda_attention, and its outputs between guard columns"""

    def __init__(self, coda, lens, past, heads, kv_heads, D, causal, seed, behind=0, rope=False, scale=None, pad=8, size=1.0):
        self.coda, self.heads, self.kv_heads, self.D, self.causal, self.scale = coda, heads, kv_heads, D, causal, scale or D ** -0.5
        self.q_at = offsets(lens)
        self.k_at = self.q_at if past is None else offsets([max(0, n + past) for n in lens])
        T, Tk = self.q_at[-1] + behind, self.k_at[-1] + behind
        self.Q, self.K, self.V = qkv(T, heads, kv_heads, D, seed, size, pad)
        if past is not None:
            _, self.K, self.V = qkv(Tk, heads, kv_heads, D, seed + 1, size, pad)
        self.seq_q, self.seq_k = device(self.q_at), None if past is None else device(self.k_at)
        self.out, self.lse = torch.zeros((T, heads * D), dtype=torch.bfloat16, device="cuda"), torch.zeros((heads, T), device="cuda")
        coda.coda_attention(self.Q, self.K, self.V, self.seq_q, self.out, heads, kv_heads, self.scale, lse=self.lse, seq_k=self.seq_k, causal=causal)
        g = torch.Generator().manual_seed(seed + 2)
        self.dout = torch.randn((T, heads * D), generator=g).to(torch.bfloat16).cuda()
        self.rope = None
        if rope:
            cos, sin = tables(37, D)
            self.rope = (cos, sin, torch.randint(-3, 45, (T,), generator=g, dtype=torch.int32), torch.randint(-3, 45, (Tk,), generator=g, dtype=torch.int32))
        self.full = [torch.empty((n, w * D + pad), dtype=torch.bfloat16, device="cuda") for n, w in ((T, heads), (Tk, kv_heads), (Tk, kv_heads))]
        need = coda.coda_attention_bwd_workspace_bytes(T, Tk, len(lens), heads, kv_heads, D)
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def grads(self):
        return [x[:, : w * self.D] for x, w in zip(self.full, (self.heads, self.kv_heads, self.kv_heads))]

    def run(self, stream=None):
        for x in self.full:
            x.fill_(FILL)
        self.ws.fill_(0xFF)
        rope = None if self.rope is None else tuple(x.cuda() for x in self.rope)
        torch.cuda.synchronize()
        self.call(rope, stream)
        torch.cuda.synchronize()
        for x, y in zip(self.full, self.grads()):
            assert (x[:, y.shape[1]:] == FILL).all(), "wrote beyond its columns"
        return [x.clone() for x in self.grads()]

    def call(self, rope=None, stream=None):
        self.coda.coda_attention_bwd(self.Q, self.K, self.V, self.out, self.dout, self.lse, self.seq_q, *self.grads(), self.heads, self.kv_heads, self.scale, self.ws,
                                     seq_k=self.seq_k, causal=self.causal, rope=rope, stream=stream)

    def expected(self):
        D, H, G = self.D, self.heads, self.kv_heads
        want = [torch.full(x.shape, FILL, dtype=torch.float64) for x in self.grads()]
        bound = [torch.zeros(x.shape, dtype=torch.float64) for x in self.grads()]
        for a, b, ka, kb in zip(self.q_at, self.q_at[1:], self.k_at, self.k_at[1:]):
            see = R.visible(b - a, kb - ka, self.causal)
            for g in range(G):
                kt = slice(g * D, (g + 1) * D)
                dk, dv, b_dk, b_dv = (torch.zeros((kb - ka, D), dtype=torch.float64) for _ in range(4))
                for h in range(g * H // G, (g + 1) * H // G):
                    at = slice(h * D, (h + 1) * D)
                    r = R.gradients(R.head(self.Q[a:b], h, D), R.head(self.K[ka:kb], g, D), R.head(self.V[ka:kb], g, D), R.head(self.out[a:b], h, D),
                                    R.head(self.dout[a:b], h, D), self.lse[h, a:b].double().cpu(), self.scale, see)
                    dq, b_dq = r[0], r[3]
                    if self.rope:
                        b_dq = R.turn_bound(b_dq + 4 * R.F32 * dq.abs(), *self.rope[:2], self.rope[2][a:b])
                        dq = R.turn_back(dq, *self.rope[:2], self.rope[2][a:b])
                    want[0][a:b, at], bound[0][a:b, at] = dq, R.rounded(dq, b_dq)
                    dk, dv, b_dk, b_dv = dk + r[1], dv + r[2], b_dk + r[4], b_dv + r[5]
                if self.rope:
                    b_dk = R.turn_bound(b_dk + 4 * R.F32 * dk.abs(), *self.rope[:2], self.rope[3][ka:kb])
                    dk = R.turn_back(dk, *self.rope[:2], self.rope[3][ka:kb])
                want[1][ka:kb, kt], bound[1][ka:kb, kt] = dk, R.rounded(dk, b_dk)
                want[2][ka:kb, kt], bound[2][ka:kb, kt] = dv, R.rounded(dv, b_dv)
        return want, bound

    def check(self):
        got = self.run()
        for x, w, b, name in zip(got, *self.expected(), ("dQ", "dK", "dV")):
            R.check(x, w, b, name)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1], [31], [33], [64], [65], [127, 1, 0, 2], [128], [129], [0, 200], [257, 64, 63]])
def test_causal(coda, lens, D):
    Pass(coda, lens, None, 4, 2, D, True, seed=len(lens) * 100 + D).check()


@pytest.mark.parametrize("D", [8, 24, 40, 72, 80, 96, 120])
@pytest.mark.parametrize("rope", [False, True])
def test_other_head_dimensions(coda, D, rope):
    Pass(coda, [70, 1, 131], None, 3, 1, D, True, seed=D, rope=rope).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (7, 1), (8, 8), (16, 8), (24, 3)])
def test_gradients_of_shared_heads(coda, heads, kv_heads):
    Pass(coda, [40, 97], None, heads, kv_heads, 64, True, seed=heads, rope=heads % 2 == 0).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("past", [1, 37, 200, -1, -40])
def test_other_numbers_of_keys_than_rows(coda, past, causal, D):
    """Rows that see no key have a gradient of zero, and so have the keys of a sequence without rows"""
    Pass(coda, [50, 1, 0, 129], past, 4, 2, D, causal, seed=past + 50, rope=True).check()


@pytest.mark.parametrize("lens", [[1], [64], [130, 5]])
def test_full(coda, lens):
    Pass(coda, lens, None, 2, 1, 128, False, seed=3).check()


@pytest.mark.parametrize("D", [64, 128])
def test_rope_and_rows_of_no_sequence(coda, D):
    Pass(coda, [33, 70], None, 4, 2, D, True, seed=4, behind=9, rope=True).check()


@pytest.mark.parametrize("D", [40, 64, 96, 128])
@pytest.mark.parametrize("streams", [1, 2, 4])
@pytest.mark.parametrize("lens,past,causal", [([65], None, True), ([129, 31, 1], None, True), ([257, 0, 64], None, False), ([300, 140], -37, True)])
def test_rows_shared_by_waves(coda, lens, past, causal, streams, D):
    """However many waves share 32 rows, and 32 or 64 keys a workgroup (empty sequences stand for their half tile there too)"""
    p = Pass(coda, lens + [0] * behind_empty(D, 4, streams), past, 4, 2, D, causal, seed=streams, rope=streams == 2)
    p.check()


@pytest.mark.parametrize("streams", [1, 2, 4])
def test_what_is_masked_has_no_effect_on_shared_rows(coda, streams):
    p = Pass(coda, [200, 90] + [0] * behind_empty(64, 2, streams), None, 2, 1, 64, True, seed=31)
    clean = p.run()
    p.K[150], p.V[160:200] = math.nan, math.inf
    coda.coda_attention(p.Q, p.K, p.V, p.seq_q, p.out, 2, 1, p.scale, lse=p.lse)           # what is saved is that of these keys and values
    got = p.run()
    for x, y in zip(got, clean):
        assert torch.equal(x[200:], y[200:])
    assert torch.equal(got[0][:150], clean[0][:150]) and not torch.isfinite(got[0][150:200]).all(1).any()


@pytest.mark.parametrize("scale,size", [(1e-6, 1.0), (3.0, 1.0)])
def test_flat_and_steep_weights(coda, scale, size):
    Pass(coda, [150], None, 2, 1, 64, True, seed=5, scale=scale, size=size).check()


def test_many_sequences(coda):
    Pass(coda, [(i * 7) % 5 for i in range(200)], None, 2, 1, 64, True, seed=7).check()


def test_the_same_twice(coda):
    p = Pass(coda, [300, 41], None, 8, 2, 128, True, seed=8, rope=True)
    a, b = p.run(), p.run()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("D", [64, 128, 96])
@pytest.mark.parametrize("fill", [math.nan, math.inf])
def test_what_is_masked_has_no_effect(coda, fill, D):
    """Row 71's output gradient is not finite: keys behind it and other sequences do not notice, neither do other rows.  Keys and values from row 100 on are
    not finite either: the rows ahead of them do not notice."""
    p = Pass(coda, [150, 40], None, 2, 1, D, True, seed=9)
    clean = p.run()
    p.dout[71] = fill
    dq, dk, dv = p.run()
    rows = torch.arange(190, device="cuda")
    assert torch.equal(dq[rows != 71], clean[0][rows != 71]) and torch.equal(dk[72:], clean[1][72:]) and torch.equal(dv[72:], clean[2][72:])
    assert not torch.isfinite(dq[71]).any() and not torch.isfinite(dv[:72]).any() and not torch.isfinite(dk[:72]).any()
    p.dout[71] = 1.0
    clean = p.run()
    p.K[100:150], p.V[100:150] = fill, fill
    p.coda.coda_attention(p.Q, p.K, p.V, p.seq_q, p.out, 2, 1, p.scale, lse=p.lse)
    dq, dk, dv = p.run()
    assert torch.equal(dq[:100], clean[0][:100]) and torch.equal(dq[150:], clean[0][150:]) and not torch.isfinite(dq[100:150]).any()
    assert torch.equal(dk[150:], clean[1][150:]) and torch.equal(dv[150:], clean[2][150:])


@pytest.mark.parametrize("causal", [True, False])
def test_rows_of_the_next_sequence_are_not_read_into_this_one(coda, causal):
    p = Pass(coda, [45, 20], None, 2, 1, 128, causal, seed=10)
    clean = p.run()
    for x in (p.Q, p.K, p.V, p.out, p.dout):
        x[45:] = math.nan
    p.lse[:, 45:] = math.nan
    for x, y in zip(p.run(), clean):
        assert torch.equal(x[:45], y[:45]) and torch.isnan(x[45:]).all()


def test_offsets_past_the_rows_write_nothing_outside(coda):
    p = Pass(coda, [30, 10], None, 2, 1, 64, True, seed=11)
    want = p.run()
    p.seq_q = device([-4, 30, 95])
    for x, y in zip(p.run(), want):
        assert torch.equal(x, y)


def test_differences(coda):
    """The sum of out * dout, with outputs in 64 bits, changes along a direction as the gradients say"""
    heads, kv_heads, D, T = 2, 1, 64, 40
    p = Pass(coda, [T], None, heads, kv_heads, D, True, seed=12)
    grads = [x.double().cpu() for x in p.run()]
    see = R.visible(T, T, True)

    def total(Q, K, V):
        return sum((R.attend(Q[:, h * D:(h + 1) * D], K, V, p.scale, see)[0] * R.head(p.dout, h, D)).sum() for h in range(heads))

    at = [x.double().cpu() for x in (p.Q, p.K, p.V)]
    g = torch.Generator().manual_seed(1)
    for i in range(3):
        d = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
        step = 1e-4
        moved = [[x + s * step * d if j == i else x for j, x in enumerate(at)] for s in (1, -1)]
        slope = (total(*moved[0]) - total(*moved[1])) / (2 * step)
        # each element of a gradient is off by a few roundings of 2^-8 of itself and of its terms; in the sum over the direction they are independent
        off = 6 * R.B16 * float((grads[i] * d).norm()) + 0.02 * float(grads[i].norm()) / T ** 0.5 * 2
        assert abs(float(slope) - float((grads[i] * d).sum())) <= off, ("QKV"[i], float(slope), float((grads[i] * d).sum()), off)


def test_matrices_past_2_gib(coda):
    pitch, T, D = 1 << 18, 8400, 64
    small = Pass(coda, [150], None, 2, 1, D, True, seed=14)
    want = small.run()
    p = Pass(coda, [T - 150, 150], None, 2, 1, D, True, seed=15)
    big = torch.empty((T, pitch), dtype=torch.bfloat16, device="cuda")
    views = [big[:, i * 128: i * 128 + w] for i, w in enumerate((128, 64, 64, 128, 128, 128, 64, 64))]
    for v, x, y in zip(views, (p.Q, p.K, p.V, p.out, p.dout), (small.Q, small.K, small.V, small.out, small.dout)):
        v[: T - 150], v[T - 150:] = x[: T - 150], y
    p.lse[:, T - 150:] = small.lse
    coda.coda_attention_bwd(*views[:5], p.lse, p.seq_q, *views[5:], 2, 1, p.scale, p.ws)
    torch.cuda.synchronize()
    for v, w in zip(views[5:], want):
        assert torch.equal(v[T - 150:], w)
