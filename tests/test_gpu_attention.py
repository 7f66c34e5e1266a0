"""coda_attention against attention in 64 bits."""
import math

import pytest
import torch

from tests import attn_ref as R

pytestmark = pytest.mark.gpu

FILL = -7.25


@pytest.fixture(scope="module")
def coda():
    from paper_2605_19269_amd import coda as c
    return c


def offsets(lens, behind=0):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def device(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).cuda()


def qkv(T, heads, kv_heads, D, seed, size=1.0, pad=0):
    """Column blocks of one matrix with `pad` further columns"""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((T, (heads + 2 * kv_heads) * D + pad), generator=g) * size).to(torch.bfloat16).cuda()
    return x[:, : heads * D], x[:, heads * D: (heads + kv_heads) * D], x[:, (heads + kv_heads) * D: (heads + 2 * kv_heads) * D]


def expected(Q, K, V, q_at, k_at, heads, kv_heads, D, scale, causal):
    Tq = Q.shape[0]
    out, b_out = torch.full((Tq, heads * D), FILL, dtype=torch.float64), torch.zeros((Tq, heads * D), dtype=torch.float64)
    lse, b_lse = torch.full((heads, Tq), FILL, dtype=torch.float64), torch.zeros((heads, Tq), dtype=torch.float64)
    for a, b, ka, kb in zip(q_at, q_at[1:], k_at, k_at[1:]):
        see = R.visible(b - a, kb - ka, causal)
        for h in range(heads):
            kv = h // (heads // kv_heads)
            r = R.attend(R.head(Q[a:b], h, D), R.head(K[ka:kb], kv, D), R.head(V[ka:kb], kv, D), scale, see)
            out[a:b, h * D: (h + 1) * D], lse[h, a:b], b_out[a:b, h * D: (h + 1) * D], b_lse[h, a:b] = r
    return out, lse, b_out, b_lse


def run(coda, Q, K, V, q_at, k_at, heads, kv_heads, scale, causal, pad=0, stats=True):
    full = torch.full((Q.shape[0], Q.shape[1] + pad), FILL, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((heads, Q.shape[0]), FILL, device="cuda") if stats else None
    coda.coda_attention(Q, K, V, device(q_at), full[:, : Q.shape[1]], heads, kv_heads, scale, lse=lse, seq_k=None if k_at is q_at else device(k_at), causal=causal)
    torch.cuda.synchronize()
    assert (full[:, Q.shape[1]:] == FILL).all(), "wrote beyond its columns"
    return full[:, : Q.shape[1]], lse


def both(coda, lens, past, heads, kv_heads, D, causal, seed, behind=0, scale=None, size=1.0, pad=0):
    q_at = offsets(lens)
    k_at = q_at if past is None else offsets([max(0, n + past) for n in lens])
    scale = scale or D ** -0.5
    Q, K, V = qkv(q_at[-1] + behind, heads, kv_heads, D, seed, size, pad)
    if past is not None:
        _, K, V = qkv(k_at[-1] + behind, heads, kv_heads, D, seed + 1, size, pad)
    out, lse = run(coda, Q, K, V, q_at, k_at, heads, kv_heads, scale, causal, pad)
    o, m, b_o, b_m = expected(Q, K, V, q_at, k_at, heads, kv_heads, D, scale, causal)
    R.check(out, o, b_o, "out")
    R.check(lse, m, b_m, "lse")


# lengths around the 32, 64 and 128 of the tiles, one, none, several sequences
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1], [31], [64], [65], [127, 1, 0, 2], [128], [129], [0, 300], [257, 64, 63], [509]])
def test_causal(coda, lens, D):
    both(coda, lens, None, 4, 2, D, True, seed=len(lens) * 100 + D)


@pytest.mark.parametrize("D", [8, 24, 40, 72, 80, 96, 120])
def test_other_head_dimensions(coda, D):
    both(coda, [70, 1, 131], None, 3, 1, D, True, seed=D)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (7, 1), (8, 8), (16, 8), (24, 3)])
def test_grouped_heads(coda, heads, kv_heads):
    both(coda, [40, 97], None, heads, kv_heads, 64, True, seed=heads)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("past", [1, 37, 64, 200, -1, -40])
def test_other_numbers_of_keys_than_rows(coda, past, causal, D):
    """Keys ahead of the rows; fewer keys than rows: with a causal mask the first rows see none, and a sequence may have none at all."""
    both(coda, [50, 1, 129], past, 4, 2, D, causal, seed=past + 50)


@pytest.mark.parametrize("lens", [[1], [64], [130, 5]])
def test_full(coda, lens):
    both(coda, lens, None, 2, 1, 128, False, seed=3)


def test_rows_of_no_sequence_and_columns_beside_the_output_stay(coda):
    both(coda, [33, 70], None, 4, 2, 64, True, seed=4, behind=9, pad=24)


def behind_empty(D, heads, streams):
    """How many empty sequences a call takes along for its rows to be shared by `streams` waves: sequences count half a tile each.  With 600 and two key heads
    the gradients of keys are formed 64 keys at a time."""
    room = 288 if D > 64 else 576
    return {4: 0, 2: 2 * room // heads + 20, 1: max(4 * room // heads + 20, 600)}[streams]


@pytest.mark.parametrize("D", [40, 64, 96, 128])
@pytest.mark.parametrize("streams", [1, 2, 4])
@pytest.mark.parametrize("lens,past,causal", [([65], None, True), ([129, 31, 1], None, True), ([257, 0, 64], None, False), ([300], 70, True), ([300, 140], -37, True),
                                              ([40], 500, False)])
def test_rows_shared_by_waves(coda, lens, past, causal, streams, D):
    """However many waves share 32 rows, and whatever tile of keys is a stream's last"""
    extra = behind_empty(D, 4, streams)
    if past is not None and past > 0:                                                    # no rows, but keys
        q_at, k_at = offsets(lens + [0] * extra), offsets([n + past for n in lens] + [0] * extra)
        Q = qkv(q_at[-1], 4, 2, D, streams)[0]
        _, K, V = qkv(k_at[-1], 4, 2, D, streams + 10)
        out, lse = run(coda, Q, K, V, q_at, k_at, 4, 2, D ** -0.5, causal)
        o, m, b_o, b_m = expected(Q, K, V, q_at, k_at, 4, 2, D, D ** -0.5, causal)
        R.check(out, o, b_o, "out")
        R.check(lse, m, b_m, "lse")
    else:
        both(coda, lens + [0] * extra, past, 4, 2, D, causal, seed=streams)


@pytest.mark.parametrize("streams", [1, 2, 4])
def test_what_is_masked_has_no_effect_on_shared_rows(coda, streams):
    D, lens = 64, [300, 90]
    at = offsets(lens + [0] * behind_empty(D, 2, streams))
    Q, K, V = qkv(at[-1], 2, 1, D, 21)
    clean = run(coda, Q, K, V, at, at, 2, 1, D ** -0.5, True)
    V[140, 3], V[141, 3], V[150, 5], V[260, 7], K[280] = math.inf, -math.inf, math.nan, -math.inf, math.nan
    out, lse = run(coda, Q, K, V, at, at, 2, 1, D ** -0.5, True)
    keep = [c for c in range(64) if c not in (3, 5, 7)]
    for h in range(2):
        x, y = out[:, h * D: (h + 1) * D], clean[0][:, h * D: (h + 1) * D]
        assert torch.equal(x[:140], y[:140]) and torch.equal(x[300:], y[300:]) and torch.equal(x[:280, keep], y[:280, keep])
        assert x[140, 3] == math.inf and torch.isnan(x[141:300, 3]).all() and torch.isnan(x[150:300, 5]).all() and (x[260:280, 7] == -math.inf).all()
        assert torch.equal(x[:150, 5], y[:150, 5]) and torch.equal(x[:260, 7], y[:260, 7]) and torch.isnan(x[280:300]).all()
    assert torch.equal(lse[:, :280], clean[1][:, :280]) and torch.isnan(lse[:, 280:300]).all() and torch.equal(lse[:, 300:], clean[1][:, 300:])


@pytest.mark.parametrize("scale,size", [(1e-6, 1.0), (3.0, 1.0), (0.125, 30.0)])
def test_flat_and_steep_weights(coda, scale, size):
    """Scores next to each other, and so far apart that one key has all the weight: hundreds between them"""
    both(coda, [150], None, 2, 1, 64, True, seed=5, scale=scale, size=size)


def test_rising_scores_renew_the_maximum_in_every_tile(coda):
    T, D = 400, 64
    Q, K, V = qkv(T, 1, 1, D, 6)
    Q.fill_(1.0)
    K.copy_((torch.arange(T, device="cuda")[:, None] * 0.05).expand(T, D).to(torch.bfloat16))
    at = [0, T]
    out, lse = run(coda, Q, K, V, at, at, 1, 1, 0.125, True)
    o, m, b_o, b_m = expected(Q, K, V, at, at, 1, 1, D, 0.125, True)
    R.check(out, o, b_o, "out")
    R.check(lse, m, b_m, "lse")


def test_many_sequences(coda):
    """More than the 64 that are looked at at once, empty ones among them"""
    lens = [(i * 7) % 5 for i in range(300)]
    both(coda, lens, None, 2, 1, 64, True, seed=7)


def test_more_than_64_times_64_sequences(coda):
    lens = [1 + (i % 3 == 0) for i in range(4200)]
    q_at = offsets(lens)
    Q, K, V = qkv(q_at[-1], 1, 1, 8, 8)
    out, lse = run(coda, Q, K, V, q_at, q_at, 1, 1, 1.0, True)
    first = torch.tensor(q_at[:-1])
    assert torch.equal(out[first.cuda()], V[first.cuda()])                                # the first row of a sequence sees itself alone
    o, m, b_o, b_m = expected(Q[:60], K[:60], V[:60], [a for a in q_at if a <= 60], [a for a in q_at if a <= 60], 1, 1, 8, 1.0, True)
    n = max(a for a in q_at if a <= 60)
    R.check(out[:n], o[:n], b_o[:n], "out")


@pytest.mark.parametrize("D", [64, 128, 96])
@pytest.mark.parametrize("what", ["nan", "inf", "mixed"])
def test_what_is_masked_has_no_effect(coda, what, D):
    """Keys and values from a row on, and the sequence behind, are not finite: rows ahead of them do not notice, and those that see one are
    what the sums make of it."""
    lens, bad = [150, 40], 71
    q_at = offsets(lens)
    Q, K, V = qkv(q_at[-1] + 5, 2, 1, D, 9)
    clean = run(coda, Q, K, V, q_at, q_at, 2, 1, D ** -0.5, True)
    fill = {"nan": math.nan, "inf": math.inf, "mixed": math.inf}[what]
    V[bad, 3] = fill
    if what == "mixed":
        V[bad + 1, 3], V[bad + 1, 5], V[bad + 20, 1] = -math.inf, -math.inf, math.nan
    else:
        V[bad:] = fill
        K[bad + 30:] = math.nan
    out, lse = run(coda, Q, K, V, q_at, q_at, 2, 1, D ** -0.5, True)
    assert torch.equal(out[:bad], clean[0][:bad]) and torch.equal(lse[:, :bad], clean[1][:, :bad])
    for h in range(2):
        mine, before = out[:, h * D: (h + 1) * D], clean[0][:, h * D: (h + 1) * D]
        if what == "mixed":
            assert (mine[bad, 3] == math.inf) and torch.isnan(mine[bad + 1:150, 3]).all()
            assert torch.equal(mine[bad:bad + 1, :3], before[bad:bad + 1, :3]) and (mine[bad + 1: 150, 5] == -math.inf).all()
            assert torch.isnan(mine[bad + 20: 150, 1]).all() and torch.equal(mine[:150, 7], before[:150, 7])
            assert torch.equal(mine[150:190], before[150:190])
        else:
            first = mine[bad: bad + 30]
            assert (torch.isnan(first) if what == "nan" else first == math.inf).all()
            assert torch.isnan(mine[bad + 30: 190]).all()


@pytest.mark.parametrize("causal", [True, False])
def test_rows_of_the_next_sequence_are_not_read_into_this_one(coda, causal):
    q_at = offsets([45, 20])
    Q, K, V = qkv(q_at[-1], 2, 1, 128, 10)
    clean, _ = run(coda, Q, K, V, q_at, q_at, 2, 1, 0.1, causal)
    K[45:], V[45:] = math.nan, math.inf
    out, _ = run(coda, Q, K, V, q_at, q_at, 2, 1, 0.1, causal)
    assert torch.equal(out[:45], clean[:45]) and torch.isnan(out[45:]).all()


def test_a_row_that_is_not_finite_keeps_to_itself(coda):
    at = [0, 100]
    Q, K, V = qkv(100, 1, 1, 64, 11)
    clean, m0 = run(coda, Q, K, V, at, at, 1, 1, 0.125, True)
    Q[50] = math.nan
    out, m1 = run(coda, Q, K, V, at, at, 1, 1, 0.125, True)
    keep = torch.arange(100, device="cuda") != 50
    assert torch.equal(out[keep], clean[keep]) and torch.equal(m0[:, keep], m1[:, keep]) and torch.isnan(out[50]).all() and torch.isnan(m1[:, 50]).all()


def test_offsets_past_the_rows_and_falling_ones_write_nothing_outside(coda):
    Q, K, V = qkv(40, 2, 1, 64, 12)
    guard = torch.full((60, 128), FILL, dtype=torch.bfloat16, device="cuda")
    coda.coda_attention(Q, K, V, device([-5, 30, 10, 90]), guard[10:50], 2, 1, 0.125)
    torch.cuda.synchronize()
    assert (guard[:10] == FILL).all() and (guard[50:] == FILL).all()
    o, _, b_o, _ = expected(Q[:30], K[:30], V[:30], [0, 30], [0, 30], 2, 1, 64, 0.125, True)
    R.check(guard[10:20], o[:10], b_o[:10], "rows of the first sequence alone")


def test_without_lse(coda):
    at = [0, 77]
    Q, K, V = qkv(77, 4, 4, 64, 13)
    a, _ = run(coda, Q, K, V, at, at, 4, 4, 0.125, True)
    b, none = run(coda, Q, K, V, at, at, 4, 4, 0.125, True, stats=False)
    assert none is None and torch.equal(a, b)


def test_matrices_past_2_gib(coda):
    """Offsets beyond 32 bits: the rows behind 2^31 elements of a matrix with a wide pitch"""
    pitch, T, D = 1 << 18, 8400, 64                                                     # 8400 * 2^18 * 2 bytes = 4.4 GB
    big = torch.empty((T, pitch), dtype=torch.bfloat16, device="cuda")
    small = qkv(150, 2, 1, D, 14)
    q_at = [0, T - 150, T]
    Q, K, V = big[:, :128], big[:, 128:192], big[:, 192:256]
    for x in (Q, K, V):
        x[: T - 150].fill_(0.25)
    for x, y in zip((Q, K, V), small):
        x[T - 150:] = y
    out, lse = run(coda, Q, K, V, q_at, q_at, 2, 1, 0.125, True)
    o, m, b_o, b_m = expected(*small, [0, 150], [0, 150], 2, 1, D, 0.125, True)
    R.check(out[T - 150:], o, b_o, "out")
    R.check(lse[:, T - 150:], m, b_m, "lse")
    assert (out[: T - 150] == 0.25).all()
