"""Infinities in what rows do see: a key with an infinite element whose score is -inf has a weight of zero, and everything else is as if the key were not there; an infinite
element of an output's gradient reaches its own column of dV.  Wherever the key or the row lies, in a tile that a mask touches or in one that all rows see."""
import math

import pytest
import torch

from tests import attn_ref as R
from tests.test_gpu_attention import behind_empty, coda, device, offsets  # noqa: F401
from tests.test_gpu_attention_bwd import Pass
from tests.test_gpu_attention_cached import Cache

pytestmark = pytest.mark.gpu


def hidden(key):
    """R.visible of a first sequence whose rows' weight of `key` is zero; the sequences behind it have no rows"""
    see = R.visible
    return lambda rows, keys, causal: see(rows, keys, causal) & (torch.arange(keys) != key)


@pytest.mark.parametrize("D", [64, 128, 40, 96])
@pytest.mark.parametrize("streams", [1, 2, 4])
@pytest.mark.parametrize("rows,past,causal,key", [(300, None, True, 290), (300, None, True, 130), (300, None, True, 3), (77, 200, True, 210), (77, 200, True, 70),
                                                  (150, -30, True, 90), (130, None, False, 129), (130, None, False, 9)])
def test_gradients_with_a_key_of_weight_zero(coda, monkeypatch, rows, past, causal, key, streams, D):
    """The key's column of dQ is NaN (zero times an infinity) for the rows that see it, no other column and no other row notices, dK and dV of the key are zero"""
    col = D - 3
    p = Pass(coda, [rows] + [0] * behind_empty(D, 4, streams), past, 4, 2, D, causal, seed=key + D)
    for h in range(4):
        p.Q[:, h * D + col] = p.Q[:, h * D + col].abs() + 0.25
    p.K[key, [col, D + col]] = -math.inf
    coda.coda_attention(p.Q, p.K, p.V, p.seq_q, p.out, 4, 2, p.scale, lse=p.lse, seq_k=p.seq_k, causal=causal)
    got = p.run()
    sees = R.visible(rows, p.k_at[1], causal)[:, key]
    assert sees.any() and torch.isfinite(p.out).all()
    p.K[key, [col, D + col]] = 0.0
    with monkeypatch.context() as m:
        m.setattr(R, "visible", hidden(key))
        want, bound = p.expected()
    for h in range(4):
        want[0][sees, h * D + col] = math.nan
    for x, w, b, name in zip(got, want, bound, ("dQ", "dK", "dV")):
        R.check(x, w, b, name)


@pytest.mark.parametrize("D", [64, 128, 40, 96])
@pytest.mark.parametrize("streams", [1, 4])            # 64 keys a workgroup, and 32
@pytest.mark.parametrize("fill", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("rows,past,causal,row", [(300, None, True, 71), (300, None, True, 299), (77, 200, True, 5), (150, -30, True, 40), (130, None, False, 129), (130, None, False, 9)])
def test_gradients_with_an_infinite_element_of_the_outputs_gradient(coda, rows, past, causal, row, fill, streams, D):
    """It reaches its own column of dV for the keys that its row sees, all of their dK, and all of its row of dQ; nothing else notices"""
    col = D - 5
    p = Pass(coda, [rows] + [0] * behind_empty(D, 4, streams), past, 4, 2, D, causal, seed=row + D)
    p.dout[row, D + col] = fill                                                          # of the second head, which the first head of keys is for
    got = p.run()
    seen = R.visible(rows, p.k_at[1], causal)[row]
    assert seen.any()
    p.dout[row, D + col] = 0.0
    want, bound = p.expected()
    seen = torch.cat((seen, torch.zeros(p.K.shape[0] - p.k_at[1], dtype=torch.bool)))
    want[2][seen, col] = fill                                                            # weights are positive
    for x, w, b, name, left_out in zip(got, want, bound, ("dQ", "dK", "dV"), ((row, slice(D, 2 * D)), (seen, slice(0, D)), None)):
        x = x.double().cpu()
        if left_out is not None:
            assert not torch.isfinite(x[left_out]).any(), name
            x[left_out] = w[left_out]
        R.check(x, w, b, name)


@pytest.mark.parametrize("D", [64, 128, 96])
@pytest.mark.parametrize("lens,rows,tree", [([40, 3, 2], [1, 1, 2], None), ([6000, 5], [1, 3], None), ([300], [40], None), ([6000, 70], [33, 70], None), ([20, 3, 9], [4, 5, 1], "rows"),
                                            ([300, 40], [40, 40], "rows"), ([50], [60], "nobody"), ([6000, 4], [20, 70], "nobody")])
def test_rows_that_see_keys_of_no_weight_alone(coda, lens, rows, tree, D):
    """Every score is -inf: NaN, with a log-sum-exp of -inf, as coda_attention has it; rows that see no key are zeros"""
    c = Cache(coda, lens, rows, 4, 2, D, 16, seed=D + len(lens), tree={None: None, "rows": lambda n: [1 << i for i in range(n)], "nobody": lambda n: [0] * n}[tree])
    for h in range(4):
        c.Q[:, h * D] = c.Q[:, h * D].abs() + 0.25
    for g in range(2):
        c.K[:, g * D] = -math.inf
    coda.coda_cache_store(c.K, c.V, c.slots, c.k, c.v)
    out, lse = c.run()
    assert (lse == -math.inf).all()
    k_at = offsets(lens)
    for s, (a, b) in enumerate(zip(c.q_at, c.q_at[1:])):
        n = lens[s]
        see = R.visible(b - a, n, True) if tree is None else R.tree_visible(b - a, n, c.bits[a:b])
        some = see.any(1)
        assert torch.isnan(out[a:b][some]).all() and (out[a:b][~some] == 0).all(), s
        if tree is None:
            plain, m = torch.empty_like(out[a:b]), torch.empty((4, b - a), device="cuda")
            coda.coda_attention(c.Q[a:b], c.K[k_at[s]: k_at[s + 1]], c.V[k_at[s]: k_at[s + 1]], device([0, b - a]), plain, 4, 2, c.scale, lse=m, seq_k=device([0, n]))
            assert torch.equal(plain.isnan(), out[a:b].isnan()) and torch.equal(plain.nan_to_num(), out[a:b].nan_to_num()) and torch.equal(m, lse[:, a:b])


@pytest.mark.parametrize("D", [64, 128, 40, 96])
@pytest.mark.parametrize("streams", [1, 2, 4])
@pytest.mark.parametrize("rows,past,causal,key", [(300, None, True, 290), (300, None, True, 130), (300, None, True, 3), (77, 200, True, 210), (150, -30, True, 90), (130, None, False, 9)])
def test_gradients_with_an_infinite_value(coda, rows, past, causal, key, streams, D):
    """Rows that see it have no finite dQ and delta, and the keys that they see no finite dK; weights are finite, and so is all of dV"""
    p = Pass(coda, [rows] + [0] * behind_empty(D, 4, streams), past, 4, 2, D, causal, seed=key + D)
    clean = p.run()
    p.V[key, D + 2] = math.inf                                                           # of the second head of keys
    coda.coda_attention(p.Q, p.K, p.V, p.seq_q, p.out, 4, 2, p.scale, lse=p.lse, seq_k=p.seq_k, causal=causal)
    see = R.visible(rows, p.k_at[1], causal)
    sees = see[:, key].cuda()
    hit = torch.cat((see[see[:, key]].any(0), torch.zeros(p.K.shape[0] - p.k_at[1], dtype=torch.bool))).cuda()
    dq, dk, dv = p.run()
    assert torch.equal(dv, clean[2])
    assert torch.equal(dq[:, : 2 * D], clean[0][:, : 2 * D]) and torch.equal(dk[:, :D], clean[1][:, :D])
    assert torch.equal(dq[~sees], clean[0][~sees]) and not torch.isfinite(dq[sees, 2 * D:]).any()
    assert torch.equal(dk[~hit], clean[1][~hit]) and not torch.isfinite(dk[hit, D:]).any()
