"""Calls of which one side is empty: no rows of Q, no keys, no sequences with either."""
import math

import pytest
import torch

from tests.test_gpu_attention import FILL, coda, device, qkv  # noqa: F401
from tests.test_gpu_attention_bwd import tables

pytestmark = pytest.mark.gpu


def call(coda, T, Tk, q_at, k_at, D, causal, rope):
    heads, kv_heads = 4, 2
    Q, K, V = qkv(T, heads, kv_heads, D, 1)[0], *qkv(Tk, heads, kv_heads, D, 2)[1:]
    seq_q, seq_k = device(q_at), device(k_at)
    out, lse = torch.full((T, heads * D), FILL, dtype=torch.bfloat16, device="cuda"), torch.full((heads, T), FILL, device="cuda")
    coda.coda_attention(Q, K, V, seq_q, out, heads, kv_heads, 0.1, lse=lse, seq_k=seq_k, causal=causal)
    grads = [torch.full((n, w * D), FILL, dtype=torch.bfloat16, device="cuda") for n, w in ((T, heads), (Tk, kv_heads), (Tk, kv_heads))]
    ws = torch.empty(coda.coda_attention_bwd_workspace_bytes(T, Tk, len(q_at) - 1, heads, kv_heads, D), dtype=torch.uint8, device="cuda")
    turn = None if not rope else tuple(x.cuda() for x in tables(9, D)) + (device([3] * T), device([5] * Tk))
    coda.coda_attention_bwd(Q, K, V, out, torch.ones_like(out), lse, seq_q, *grads, heads, kv_heads, 0.1, ws, seq_k=seq_k, causal=causal, rope=turn)
    torch.cuda.synchronize()
    return out, lse, grads


@pytest.mark.parametrize("D", [64, 128, 72])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rope", [False, True])
def test_no_keys(coda, D, causal, rope):
    out, lse, (dq, dk, dv) = call(coda, 70, 0, [0, 33, 70], [0, 0, 0], D, causal, rope)
    assert (out == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.numel() == dv.numel() == 0


@pytest.mark.parametrize("D", [64, 128, 72])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("n", [1, 700])
def test_no_rows(coda, D, causal, rope, n):
    """32 and 64 keys a workgroup"""
    _, _, (dq, dk, dv) = call(coda, 0, 70, [0] * (n + 1), [0, 33] + [70] * (n - 1) if n > 1 else [0, 70], D, causal, rope)
    assert dq.numel() == 0 and (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_rows_and_keys_of_no_sequence(coda, D):
    out, lse, grads = call(coda, 5, 7, [2, 2, 2], [7, 7, 7], D, True, False)
    assert all((x == FILL).all() for x in (out, lse, *grads))
