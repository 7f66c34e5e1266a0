"""Refusals of the attention entry points (status codes before anything is launched), workspace sizes, the binding's checks, and the 64-bit
reference of the GPU tests against automatic differentiation."""
import ctypes
import math

import pytest
import torch

from tests import attn_ref as R

P = 0x10000      # an address that is aligned and never touched: no call here gets as far as a launch


@pytest.fixture(scope="module")
def coda():
    from paper_2605_19269_amd import coda as c
    return c


def mat(coda, rows, cols, ptr=P, ld=None, trans=0, dtype=0):
    return coda.coda_mat(ptr, rows, cols, cols if ld is None else ld, trans, dtype)


def ref(x):
    return None if x is None else ctypes.byref(x)


FWD = dict(T=64, Tk=None, heads=4, kv=2, D=64, Q={}, K={}, V={}, seq_q=P, seq_k=None, n=3, scale=0.125, causal=1, out=P, ldo=256, lse=P)


def forward(coda, **over):
    a = {**FWD, **over}
    Tk = a["T"] if a["Tk"] is None else a["Tk"]
    m = {}
    for name, rows, h in (("Q", a["T"], a["heads"]), ("K", Tk, a["kv"]), ("V", Tk, a["kv"])):
        m[name] = None if a[name] is None else mat(coda, **{**dict(rows=rows, cols=h * a["D"]), **a[name]})
    return coda._lib.coda_attention(None, ref(m["Q"]), ref(m["K"]), ref(m["V"]), a["seq_q"], a["seq_k"], a["n"], a["heads"], a["kv"], a["scale"], a["causal"],
                                    a["out"], a["ldo"], a["lse"])


# what a call of either kind refuses of its operands
OPERANDS = [
    ("NULL", dict(Q=None)), ("NULL", dict(K=None)), ("NULL", dict(V=None)), ("NULL", dict(Q=dict(ptr=0))), ("NULL", dict(K=dict(ptr=0))),
    ("NULL", dict(V=dict(ptr=0))), ("NULL", dict(seq_q=0)),
    ("DTYPE", dict(Q=dict(dtype=2))), ("DTYPE", dict(K=dict(dtype=1))), ("DTYPE", dict(V=dict(dtype=2))),
    ("SHAPE", dict(Q=dict(trans=1))), ("SHAPE", dict(K=dict(trans=1))), ("SHAPE", dict(heads=0)), ("SHAPE", dict(kv=0)), ("SHAPE", dict(heads=3)), ("SHAPE", dict(heads=-4)),
    ("SHAPE", dict(Q=dict(cols=260))), ("SHAPE", dict(D=136)), ("SHAPE", dict(D=60)), ("SHAPE", dict(D=4)), ("SHAPE", dict(K=dict(cols=120, ld=128))),
    ("SHAPE", dict(V=dict(rows=63))), ("SHAPE", dict(Tk=65)), ("SHAPE", dict(Q=dict(ld=248))), ("SHAPE", dict(K=dict(ld=(1 << 22) + 8))), ("SHAPE", dict(Q=dict(rows=-1))),
    ("SHAPE", dict(n=-1)), ("SHAPE", dict(scale=0.0)), ("SHAPE", dict(scale=-1.0)), ("SHAPE", dict(scale=math.inf)), ("SHAPE", dict(scale=math.nan)),
    ("SHAPE", dict(scale=2.0 ** 127)), ("SHAPE", dict(T=(1 << 31) - 511, heads=1, kv=1, D=8)), ("SHAPE", dict(T=8, Tk=(1 << 31) - 511, seq_k=P)),
    ("SHAPE", dict(T=(1 << 30) - 255, Tk=8, seq_k=P)),
    ("SHAPE", dict(T=1 << 31, seq_k=P, Tk=8)), ("SHAPE", dict(T=1 << 30, heads=8, kv=1, seq_k=P, Tk=8)),
    ("ALIGN", dict(Q=dict(ptr=P + 8))), ("ALIGN", dict(V=dict(ptr=P + 2))), ("ALIGN", dict(K=dict(ld=132))), ("ALIGN", dict(seq_q=P + 2)), ("ALIGN", dict(seq_k=P + 1)),
]


@pytest.mark.parametrize("want,over", OPERANDS + [
    ("NULL", dict(out=0)), ("SHAPE", dict(ldo=248)), ("SHAPE", dict(ldo=(1 << 22) + 8)), ("ALIGN", dict(ldo=260)), ("ALIGN", dict(out=P + 4)), ("ALIGN", dict(lse=P + 2)),
    ("SHAPE", dict(T=(1 << 28) - 1, heads=32, kv=32, D=8))])
def test_forward_refuses(coda, want, over):
    if over.get("T") == (1 << 28) - 1:
        over = dict(over, ldo=256, n=1 << 20)       # 2^21 + 2^20 tiles of 32 heads: past 2^32 work items
    assert forward(coda, **over) == getattr(coda, "CODA_ERR_" + want)


def test_nothing_to_do(coda):
    assert forward(coda, n=0, out=0, seq_q=0) == coda.CODA_OK
    assert forward(coda, T=0, Q=dict(ptr=0), K=dict(ptr=0), V=dict(ptr=0), out=0, seq_q=0) == coda.CODA_OK
    assert backward(coda, n=0, dQ=0, seq_q=0, ws=0) == coda.CODA_OK
    assert cached(coda, n=0, seq_q=0, lens=0, ws=0, out=0) == coda.CODA_OK
    assert cached(coda, T=0, Q=dict(ptr=0), seq_q=0, lens=0, ws=0, out=0) == coda.CODA_OK
    assert store(coda, T=0, K=dict(ptr=0), V=dict(ptr=0), slots=0) == coda.CODA_OK
    assert store(coda, cache=dict(pages=0, k=0, v=0)) == coda.CODA_OK


BWD = dict(FWD, O={}, dO={}, rope=None, dQ=P, dK=P, dV=P, lq=256, lk=128, lv=128, ws=P, nbytes=1 << 30)


def backward(coda, **over):
    a = {**BWD, **over}
    Tk = a["T"] if a["Tk"] is None else a["Tk"]
    m = {}
    for name, rows, h in (("Q", a["T"], a["heads"]), ("K", Tk, a["kv"]), ("V", Tk, a["kv"]), ("O", a["T"], a["heads"]), ("dO", a["T"], a["heads"])):
        m[name] = None if a[name] is None else mat(coda, **{**dict(rows=rows, cols=h * a["D"]), **a[name]})
    rope = None if a["rope"] is None else coda.coda_rope(*[a["rope"].get(n, P) for n in ("cos", "sin", "pos_q", "pos_k")], a["rope"].get("rows", 64))
    return coda._lib.coda_attention_bwd(None, *[ref(m[n]) for n in ("Q", "K", "V", "O", "dO")], a["lse"], a["seq_q"], a["seq_k"], a["n"], a["heads"], a["kv"], a["scale"],
                                        a["causal"], ref(rope), a["dQ"], a["lq"], a["dK"], a["lk"], a["dV"], a["lv"], a["ws"], a["nbytes"])


@pytest.mark.parametrize("want,over", OPERANDS + [
    ("NULL", dict(O=None)), ("NULL", dict(dO=None)), ("NULL", dict(O=dict(ptr=0))), ("NULL", dict(lse=0)), ("NULL", dict(dQ=0)), ("NULL", dict(dK=0)), ("NULL", dict(dV=0)),
    ("NULL", dict(ws=0)), ("NULL", dict(rope=dict(cos=0))), ("NULL", dict(rope=dict(sin=0))), ("NULL", dict(rope=dict(pos_q=0))), ("NULL", dict(rope=dict(pos_k=0))),
    ("DTYPE", dict(dO=dict(dtype=2))), ("DTYPE", dict(O=dict(dtype=1))), ("SHAPE", dict(dO=dict(rows=63))), ("SHAPE", dict(O=dict(cols=248))), ("SHAPE", dict(lq=248)),
    ("SHAPE", dict(lk=120)), ("SHAPE", dict(rope=dict(rows=0))), ("SHAPE", dict(rope=dict(rows=1 << 31))), ("ALIGN", dict(lv=132)), ("ALIGN", dict(dK=P + 8)),
    ("ALIGN", dict(lse=P + 1)), ("ALIGN", dict(rope=dict(cos=P + 4))), ("ALIGN", dict(rope=dict(pos_q=P + 2))), ("ALIGN", dict(ws=P + 8)),
    ("WORKSPACE", dict(nbytes=64 * 4 * 8 - 1))])
def test_backward_refuses(coda, want, over):
    assert backward(coda, **over) == getattr(coda, "CODA_ERR_" + want)


CACHE = dict(k=P, v=P, pages=10, page=16, kv_heads=2, head_dim=64)
CACHED = dict(T=64, heads=4, Q={}, cache={}, table=P, ld=5, cols=5, lens=P, seq_q=P, n=3, scale=0.125, tree=None, out=P, ldo=256, lse=P, ws=P, nbytes=1 << 30)


def cached(coda, **over):
    a = {**CACHED, **over}
    cache = None if a["cache"] is None else {**CACHE, **a["cache"]}
    Q = None if a["Q"] is None else mat(coda, **{**dict(rows=a["T"], cols=a["heads"] * (cache or CACHE)["head_dim"]), **a["Q"]})
    c = None if cache is None else coda.coda_cache(*[cache[n] for n in ("k", "v", "pages", "page", "kv_heads", "head_dim")])
    return coda._lib.coda_attention_cached(None, ref(Q), ref(c), a["table"], a["ld"], a["cols"], a["lens"], a["seq_q"], a["n"], a["heads"], a["scale"], a["tree"], a["out"],
                                           a["ldo"], a["lse"], a["ws"], a["nbytes"])


CACHES = [("NULL", dict(cache=None)), ("NULL", dict(cache=dict(k=0))), ("NULL", dict(cache=dict(v=0))), ("SHAPE", dict(cache=dict(pages=-1))),
          ("SHAPE", dict(cache=dict(page=0))), ("SHAPE", dict(cache=dict(page=-16))), ("SHAPE", dict(cache=dict(page=24))), ("SHAPE", dict(cache=dict(pages=1 << 27))), ("SHAPE", dict(cache=dict(pages=2, page=1 << 24))),
          ("SHAPE", dict(cache=dict(head_dim=136))), ("SHAPE", dict(cache=dict(head_dim=20))), ("SHAPE", dict(cache=dict(kv_heads=0))), ("ALIGN", dict(cache=dict(k=P + 8)))]


@pytest.mark.parametrize("want,over", CACHES + [
    ("NULL", dict(Q=None)), ("NULL", dict(Q=dict(ptr=0))), ("NULL", dict(table=0)), ("NULL", dict(lens=0)), ("NULL", dict(seq_q=0)), ("NULL", dict(out=0)), ("NULL", dict(ws=0)),
    ("DTYPE", dict(Q=dict(dtype=2))), ("SHAPE", dict(Q=dict(trans=1))), ("SHAPE", dict(heads=3)), ("SHAPE", dict(heads=0)), ("SHAPE", dict(n=-1)), ("SHAPE", dict(scale=0.0)),
    ("SHAPE", dict(ld=4)), ("SHAPE", dict(cols=-1)), ("SHAPE", dict(cols=(1 << 26) + 1, ld=1 << 27)), ("SHAPE", dict(T=1 << 30)), ("SHAPE", dict(T=(1 << 30) - 255)), ("SHAPE", dict(scale=2.0 ** 127)), ("SHAPE", dict(T=1 << 31)), ("SHAPE", dict(ldo=128)),
    ("ALIGN", dict(table=P + 2)), ("ALIGN", dict(lens=P + 1)), ("ALIGN", dict(tree=P + 4)), ("ALIGN", dict(out=P + 8)), ("ALIGN", dict(lse=P + 2)), ("ALIGN", dict(ws=P + 4)),
    ("WORKSPACE", dict(nbytes=1000))])
def test_cached_refuses(coda, want, over):
    assert cached(coda, **over) == getattr(coda, "CODA_ERR_" + want)


STORE = dict(T=64, K={}, V={}, slots=P, cache={})


def store(coda, **over):
    a = {**STORE, **over}
    cache = None if a["cache"] is None else {**CACHE, **a["cache"]}
    K, V = (None if x is None else mat(coda, **{**dict(rows=a["T"], cols=128), **x}) for x in (a["K"], a["V"]))
    c = None if cache is None else coda.coda_cache(*[cache[n] for n in ("k", "v", "pages", "page", "kv_heads", "head_dim")])
    return coda._lib.coda_cache_store(None, ref(K), ref(V), a["slots"], ref(c))


@pytest.mark.parametrize("want,over", CACHES + [
    ("NULL", dict(K=None)), ("NULL", dict(V=None)), ("NULL", dict(K=dict(ptr=0))), ("NULL", dict(slots=0)), ("DTYPE", dict(V=dict(dtype=1))), ("SHAPE", dict(K=dict(cols=64))),
    ("SHAPE", dict(V=dict(rows=63))), ("SHAPE", dict(K=dict(trans=1))), ("ALIGN", dict(K=dict(ptr=P + 8))), ("ALIGN", dict(slots=P + 2))])
def test_store_refuses(coda, want, over):
    assert store(coda, **over) == getattr(coda, "CODA_ERR_" + want)


def test_workspace_sizes(coda):
    assert coda.coda_attention_bwd_workspace_bytes(1000, 1000, 2, 32, 8, 64) >= 1000 * 32 * 8
    small, large = coda.coda_attention_cached_workspace_bytes(1, 1, 32, 8, 128), coda.coda_attention_cached_workspace_bytes(64, 64, 32, 8, 128)
    assert 0 < small < large < 64 << 20
    for bad in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 3, 2, 64), (1, 1, 4, 2, 65), (1 << 31, 1, 4, 2, 64)):
        assert coda.coda_attention_cached_workspace_bytes(*bad) == 0
        assert coda.coda_attention_bwd_workspace_bytes(bad[0], 1, *bad[1:]) == 0


def test_the_binding_asks_for_the_right_tensors(coda):
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    good = dict(Q=bf(8, 128), K=bf(8, 64), V=bf(8, 64), seq_q=ints(2), out=bf(8, 128), heads=2, kv_heads=1, scale=0.1, stream=0)
    for name, value in dict(seq_q=torch.zeros(2, dtype=torch.int64), out=bf(7, 128), lse=torch.zeros(8, 2), seq_k=ints(3)).items():
        with pytest.raises(AssertionError):
            coda.coda_attention(**{**good, name: value})
    with pytest.raises(AssertionError):
        coda.coda_attention(**{**good, "Q": bf(128, 8).t()})
    cache = dict(cache_k=bf(4, 1, 16, 64), cache_v=bf(4, 1, 16, 64))
    good = dict(Q=bf(8, 128), **cache, table=ints(1, 4), lens=ints(1), seq_q=ints(2), out=bf(8, 128), heads=2, scale=0.1, workspace=bf(1), stream=0)
    for name, value in dict(cache_v=bf(4, 1, 16, 32), cache_k=bf(4, 1, 16, 128)[..., :64], table=ints(2, 4), lens=ints(2), tree=ints(8), lse=torch.zeros(8, 2)).items():
        with pytest.raises(AssertionError):
            coda.coda_attention_cached(**{**good, name: value})
    with pytest.raises(AssertionError):     # a table whose rows lie on each other
        coda.coda_attention_cached(**{**good, "table": ints(1, 4).expand(2, 4), "lens": ints(2), "seq_q": ints(3)})
    with pytest.raises(AssertionError):
        coda.coda_cache_store(bf(8, 64), bf(8, 64), torch.zeros(8, dtype=torch.int64), **cache, stream=0)
    with pytest.raises(AssertionError):
        coda.coda_attention_bwd(bf(8, 128), bf(8, 64), bf(8, 64), bf(8, 128), bf(8, 128), torch.zeros(2, 8), ints(2), bf(8, 128), bf(8, 64), bf(8, 64), 2, 1, 0.1, bf(1),
                                rope=(torch.zeros(4, 31), torch.zeros(4, 31), ints(8)), stream=0)


def test_addresses_of_vectors_matrices_and_caches(coda):
    b = coda._binding
    v, m = torch.zeros(6, dtype=torch.int32), torch.zeros(4, 8)
    assert b.vec(None, torch.int32, 6, None, "v") is None and b.vec(v, torch.int32, 6, None, "v") == v.data_ptr()
    assert b.vec(v[2:], torch.int32, 4, None, "v") == v.data_ptr() + 8 and b.vec(m, torch.float32, 4, 8, "m") == m.data_ptr()
    for size in ((0, 8), (4, 0), (0, 0)):                                                   # nothing in it: any strides
        b.vec(torch.zeros(size), torch.float32, *size, "m")
        b.vec(torch.zeros(size[::-1]).t(), torch.float32, *size, "m")
    b.vec(torch.zeros(1, 8)[:, ::8], torch.float32, 1, 1, "m")
    for bad in (v[::2], v.long()[:3], v[:2], v[:3].view(3, 1), torch.zeros(3), torch.tensor(3, dtype=torch.int32)):
        with pytest.raises(AssertionError, match="v: a dense tensor of 3 of torch.int32"):
            b.vec(bad, torch.int32, 3, None, "v")
    for bad in (m.t(), m[:, :4], m[::2], m.double(), v):
        with pytest.raises(AssertionError, match="m: a dense tensor of 8 x 4 of torch.float32"):
            b.vec(bad, torch.float32, 8, 4, "m")
    for t, pitch in ((m, 8), (torch.zeros(4, 24)[:, 8:16], 24), (torch.zeros(8, 8)[::2], 16)):
        assert b.rows(t, m, torch.float32, "out") == (t.data_ptr(), pitch)
    for bad in (m.bfloat16(), m.t(), m[:3], torch.zeros(8, 4).t(), v, None):
        with pytest.raises((AssertionError, AttributeError)):
            b.rows(bad, m, torch.float32, "out")
    k, w = (torch.zeros(3, 2, 16, 8, dtype=torch.bfloat16) for _ in range(2))
    rows, slots = torch.zeros(0, 16, dtype=torch.bfloat16), torch.zeros(0, dtype=torch.int32)
    coda.coda_cache_store(rows, rows, slots, k, w, stream=0)
    with pytest.raises(coda.CodaError):                                                     # heads and columns of the cache, not of K
        coda.coda_cache_store(rows[:, :8], rows[:, :8], slots, k, w, stream=0)
    for bad in ((k, w.float()), (k[:2], w), (k[:, :1], w[:, :1]), (k.transpose(0, 1), w.transpose(0, 1)), (k[0], w[0])):
        with pytest.raises(AssertionError, match="dense caches"):
            coda.coda_cache_store(rows, rows, slots, *bad, stream=0)


def test_calls_take_every_form_of_argument(coda):
    """Whole numbers for the scale, streams as objects, numbers past 32 bits: as ctypes takes them"""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    for stream in (0, ctypes.c_void_p(None), type("S", (), {"cuda_stream": 0})()):
        coda.coda_attention(bf(0, 128), bf(0, 64), bf(0, 64), ints(2), bf(0, 128), 2, 1, 1, stream=stream)
        coda.coda_attention_bwd(bf(0, 128), bf(0, 64), bf(0, 64), bf(0, 128), bf(0, 128), torch.zeros(2, 0), ints(2), bf(0, 128), bf(0, 64), bf(0, 64), 2, 1, 1, bf(8),
                                rope=(torch.zeros(4, 32), torch.zeros(4, 32), ints(0)), stream=stream)
        coda.coda_cache_store(bf(0, 64), bf(0, 64), ints(0), bf(4, 1, 16, 64), bf(4, 1, 16, 64), stream=stream)
        coda.coda_attention_cached(bf(0, 128), bf(4, 1, 16, 64), bf(4, 1, 16, 64), ints(1, 4), ints(1), ints(2), bf(0, 128), 2, 1, bf(8), stream=stream)
    good = (bf(8, 128), bf(8, 64), bf(8, 64), ints(2), bf(8, 128))
    with pytest.raises(coda.CodaError):
        coda.coda_attention(*good, 0, 1, 0.1, stream=0)
    with pytest.raises(coda.CodaError):
        coda.coda_attention_bwd(*good[:3], bf(8, 128), bf(8, 128), torch.zeros(0, 8), ints(2), bf(8, 128), bf(8, 64), bf(8, 64), 0, 1, 0.1, bf(8),
                                rope=(torch.zeros(4, 64), torch.zeros(4, 64), ints(8)), stream=0)
    for bad in (dict(heads=2 ** 40), dict(heads=-2 ** 70), dict(kv_heads=2 ** 32 + 1), dict(scale=1e300)):
        with pytest.raises((coda.CodaError, OverflowError)):
            coda.coda_attention(*good, **{**dict(heads=2, kv_heads=1, scale=0.1, stream=0), **bad})
    for bad in (dict(heads=2.0), dict(heads="2"), dict(scale="x"), dict(stream="s")):
        with pytest.raises((ctypes.ArgumentError, TypeError, ValueError, AttributeError)):
            coda.coda_attention(*good, **{**dict(heads=2, kv_heads=1, scale=0.1, stream=0), **bad})


@pytest.mark.parametrize("rows,keys,causal", [(5, 5, True), (4, 9, True), (6, 4, False), (1, 1, True)])
def test_the_reference_against_automatic_differentiation(rows, keys, causal):
    g = torch.Generator().manual_seed(rows)
    q, k, v, do = (torch.randn((n, 16), generator=g, dtype=torch.float64) for n in (rows, keys, keys, rows))
    for x in (q, k, v):
        x.requires_grad_()
    see = R.visible(rows, keys, causal)
    o, lse, b_o, b_lse = R.attend(q, k, v, 0.3, see)
    s = (q @ k.t() * 0.3).masked_fill(~see, -math.inf)
    assert torch.allclose(o, torch.softmax(s, 1) @ v, rtol=1e-12, atol=1e-12)
    o.backward(do)
    with torch.no_grad():
        for got, want in zip(R.gradients(q, k, v, o, do, lse, 0.3, see)[:3], (q.grad, k.grad, v.grad)):
            assert torch.allclose(got, want, rtol=1e-10, atol=1e-12)
        assert (b_o > 0).all() and (b_o < 0.1).all() and (b_lse < 1e-3).all()


def test_the_reference_of_trees_and_of_rows_that_see_nothing():
    see = R.tree_visible(3, 5, [1, 3, 5])
    assert see.tolist() == [[True, True, True, False, False], [True, True, True, True, False], [True, True, True, False, True]]
    assert not R.visible(4, 2, True)[:2].any() and R.visible(4, 2, True)[3].all()
    x = torch.randn((4, 8), dtype=torch.float64)
    o, lse, _, _ = R.attend(x, x[:2], x[:2], 0.3, R.visible(4, 2, True))
    assert (o[:2] == 0).all() and (lse[:2] == -math.inf).all() and torch.equal(o[2], x[0])


def test_turning_back_undoes_the_rotation():
    g = torch.Generator().manual_seed(1)
    x, angle = torch.randn((6, 16), generator=g, dtype=torch.float64), torch.rand((4, 8), generator=g)
    pos = torch.tensor([0, 1, 2, 3, 9, -2], dtype=torch.int32)
    at = pos.clamp(0, 3).long()
    c, s = angle.cos().double()[at], angle.sin().double()[at]
    y = torch.stack((x[:, 0::2] * c - x[:, 1::2] * s, x[:, 0::2] * s + x[:, 1::2] * c), 2).reshape(x.shape)
    assert torch.allclose(R.turn_back(y, angle.cos(), angle.sin(), pos), x, atol=1e-6)


def test_registers_and_local_memory_of_the_kernels():
    """Two waves a SIMD at least (one where LDS has no room for more), two workgroups of four waves a CU, no spilled registers but the few of one kernel (outside
    its loop, and where it masks a tile)"""
    import os
    import re
    from paper_2605_19269_amd import build as B
    if not os.path.exists(B.RESOURCES):
        B.build(force=True)
    seen = {}
    for line in open(B.RESOURCES):
        name, vgpr, agpr, scratch, spill, lds = line.split()
        m = re.search(r"attention_(kernel|dq_kernel|dkv_kernel|cached_kernel|join_kernel)I|(cache_store)_kernel", name)
        if not m:
            continue
        kind = m.group(1) or m.group(2)
        seen[kind] = seen.get(kind, 0) + 1
        few, alone = kind == "dkv_kernel" and re.search("ILi128ELb[01]ELi2E", name), re.search("dkv_kernelILi128ELb[01]ELi1E|cached_kernelILi[0-9]+ELb[01]ELb0E", name)
        assert int(vgpr) + int(agpr) <= (512 if alone else 256) and int(spill) <= (4 if few else 0) and int(scratch) <= (20 if few else 0), line
        wide = "ILi128E" in name and "ELi4ELi32E" in name                                 # four streams of 128 columns: one workgroup a CU
        assert int(lds) <= (80 if kind in ("kernel", "dq_kernel") and not wide else 160) * 1024, line
    assert seen == {"kernel": 12, "dq_kernel": 10, "dkv_kernel": 8, "cached_kernel": 8, "join_kernel": 8, "cache_store": 1}
