"""The attention calls as a program uses them together: a layer from its QKV projection to the gradients of its weights, a prompt that goes
into the cache and the tokens after it, drafts kept and turned down, other streams, captured graphs."""
import math

import pytest
import torch

from tests import attn_ref as R
from tests.test_gpu_attention import FILL, coda, device, expected, offsets, qkv  # noqa: F401
from tests.test_gpu_attention_bwd import Pass, tables
from tests.test_gpu_attention_cached import Cache, some_tree

pytestmark = pytest.mark.gpu


def product(coda, a, b, got, what, ta=False, tb=False, add=None, rounded=True):
    """got against a b (+ add) in 64 bits: K products summed in fp32, one rounding"""
    a, b = (x.double().cpu() for x in (a, b))
    a, b = a.t() if ta else a, b.t() if tb else b
    want, bound = a @ b, (a.shape[1] + 2) * R.F32 * (a.abs() @ b.abs())
    if add is not None:
        want = want + add.double().cpu()
        bound = bound + 2 * R.F32 * (want.abs() + add.double().cpu().abs())
    R.check(got, want, R.rounded(want, bound) if rounded else bound + R.F32 * want.abs(), what)


@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 32), (2, 2, 64), (4, 1, 128)])
def test_a_layer_and_its_gradients(coda, heads, kv_heads, D):
    lens, d = [37, 130, 1, 64], 192
    T, at, width, cols = sum(lens), offsets(lens), (heads + 2 * kv_heads) * D, heads * D
    g = torch.Generator().manual_seed(D)
    rand = lambda *s, size=1.0: (torch.randn(s, generator=g) * size).to(torch.bfloat16).cuda()
    new = lambda *s, dtype=torch.bfloat16: torch.full(s, math.nan, dtype=dtype, device="cuda")
    X, Wqkv, Wo, dY = rand(T, d), rand(d, width, size=d ** -0.5), rand(cols, d, size=cols ** -0.5), rand(T, d)
    cos, sin = (x.cuda() for x in tables(160, D))
    pos = device([i for n in lens for i in range(n)])
    seq = device(at)
    blocks = lambda x: (x[:, :cols], x[:, cols: cols + kv_heads * D], x[:, cols + kv_heads * D:])
    QKV, O, Y, lse = new(T, width), new(T, cols), new(T, d), new(heads, T, dtype=torch.float32)
    part = new(coda.coda_row_partial_blocks(d), T, dtype=torch.float32)
    coda.coda_gemm(X, Wqkv, [coda.rope(cos, sin, pos, D, cols + kv_heads * D), coda.store(QKV)])
    coda.coda_attention(*blocks(QKV), seq, O, heads, kv_heads, D ** -0.5, lse=lse)
    coda.coda_gemm(O, Wo, [coda.add_tile(X), coda.row_sumsq(part), coda.store(Y)])
    # and back
    dO, dQKV, dX, dW = new(T, cols), new(T, width), new(T, d), torch.zeros((d, width), device="cuda")
    ws = torch.empty(coda.coda_attention_bwd_workspace_bytes(T, T, len(lens), heads, kv_heads, D), dtype=torch.uint8, device="cuda")
    coda.coda_gemm(dY, Wo, [coda.store(dO)], transB=True)
    coda.coda_attention_bwd(*blocks(QKV), O, dO, lse, seq, *blocks(dQKV), heads, kv_heads, D ** -0.5, ws, rope=(cos, sin, pos))
    coda.coda_gemm(dQKV, Wqkv, [coda.store(dX)], transB=True)
    coda.coda_gemm(X, dQKV, [coda.accum_f32(dW)], transA=True)
    torch.cuda.synchronize()

    o, m, b_o, b_m = expected(*blocks(QKV), at, at, heads, kv_heads, D, D ** -0.5, True)
    R.check(O, o, b_o, "O")
    R.check(lse, m, b_m, "lse")
    product(coda, O, Wo, Y, "Y", add=X)
    p = Pass.__new__(Pass)
    p.heads, p.kv_heads, p.D, p.causal, p.scale, p.q_at, p.k_at = heads, kv_heads, D, True, D ** -0.5, at, at
    (p.Q, p.K, p.V), p.out, p.dout, p.lse, p.rope = blocks(QKV), O, dO, lse, tuple(x.cpu() for x in (cos, sin, pos, pos))
    p.full = list(blocks(dQKV))
    for got, want, bound, name in zip(blocks(dQKV), *p.expected(), ("dQ", "dK", "dV")):
        R.check(got, want, bound, name)
    product(coda, dQKV, Wqkv, dX, "dX", tb=True)
    product(coda, X, dQKV, dW, "dW", ta=True, rounded=False)


@pytest.mark.parametrize("D,page", [(64, 16), (128, 8)])
def test_a_prompt_then_tokens_and_drafts(coda, D, page):
    """Prompts into the cache by chunks, then single tokens, then drafts of which some stay: every step sees what attention over the whole
    sequence sees"""
    heads, kv_heads, lens, room = 8, 2, [37, 1, 100], 192
    n, pages = len(lens), len(lens) * room // page
    g = torch.Generator().manual_seed(page)
    order = torch.randperm(pages, generator=g).view(n, room // page).to(torch.int32)
    table = order.cuda()
    ck, cv = (torch.full((pages, kv_heads, page, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slot = lambda s, j: int(order[s, j // page]) * page + j % page
    past = [qkv(0, heads, kv_heads, D, 0) for _ in range(n)]                                # what each sequence holds so far
    scale = D ** -0.5

    def step(rows, seed, tree=None):
        """New rows of each sequence: stored, attended to the cache; -> their Q, K, V and the outputs"""
        at, T = offsets(rows), sum(rows)
        Q, K, V = qkv(T, heads, kv_heads, D, seed)
        held = [p[1].shape[0] for p in past]
        coda.coda_cache_store(K, V, device([slot(s, held[s] + i) for s in range(n) for i in range(rows[s])]), ck, cv)
        out = torch.full((T, heads * D), FILL, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(coda.coda_attention_cached_workspace_bytes(T, n, heads, kv_heads, D), dtype=torch.uint8, device="cuda")
        bits = None if tree is None else device([b for r in rows for b in tree(r)], torch.int64)
        coda.coda_attention_cached(Q, ck, cv, table, device([a + b for a, b in zip(held, rows)]), device(at), out, heads, scale, ws, tree=bits)
        return at, Q, K, V, out

    def keep(at, Q, K, V, kept):
        for s in range(n):
            rows = [at[s] + i for i in kept[s]]
            past[s] = tuple(torch.cat((old, x[rows])) for old, x in zip(past[s], (Q, K, V)))

    def check(at, Q, out, tree, K, V):
        for s, (a, b) in enumerate(zip(at, at[1:])):
            k, v = (torch.cat((past[s][i], x[a:b])) for i, x in ((1, K), (2, V)))
            see = R.visible(b - a, k.shape[0], True) if tree is None else R.tree_visible(b - a, k.shape[0], tree(b - a))
            for h in range(heads):
                kv = h * kv_heads // heads
                o, _, b_o, _ = R.attend(R.head(Q[a:b], h, D), R.head(k, kv, D), R.head(v, kv, D), scale, see)
                R.check(R.head(out[a:b], h, D), o, b_o + 64 * R.F32 * o.abs(), "sequence %d head %d" % (s, h))

    for seed, rows in enumerate(([20, 1, 64], [17, 0, 36])):                                # a prompt in two chunks
        at, Q, K, V, out = step(rows, 50 + seed)
        check(at, Q, out, None, K, V)
        keep(at, Q, K, V, [range(r) for r in rows])
    assert [p[1].shape[0] for p in past] == lens
    # the same rows by the prompt's own call
    whole = [torch.cat([p[i] for p in past]) for i in range(3)]
    out2, seq = torch.empty((sum(lens), heads * D), dtype=torch.bfloat16, device="cuda"), device(offsets(lens))
    coda.coda_attention(*whole, seq, out2, heads, kv_heads, scale)
    o, _, b_o, _ = expected(*whole, offsets(lens), offsets(lens), heads, kv_heads, D, scale, True)
    R.check(out2, o, b_o, "prompt")
    for seed in range(3):                                                                    # tokens one by one
        at, Q, K, V, out = step([1] * n, 70 + seed)
        check(at, Q, out, None, K, V)
        keep(at, Q, K, V, [[0]] * n)
    for seed, kept in enumerate(([[0, 1, 4], [], [0, 2]], [[0], [0, 1], [0, 3, 4]])):        # trees; a path of each stays
        rows = [6, 3, 9]
        at, Q, K, V, out = step(rows, 90 + seed, some_tree)
        check(at, Q, out, some_tree, K, V)
        held = [p[1].shape[0] for p in past]
        slots = [-1] * at[-1]
        for s in range(n):
            for i, r in enumerate(kept[s]):
                slots[at[s] + r] = slot(s, held[s] + i)
        coda.coda_cache_store(K, V, device(slots), ck, cv)
        keep(at, Q, K, V, kept)
    at, Q, K, V, out = step([1] * n, 99)
    check(at, Q, out, None, K, V)


def test_keys_of_no_row_have_gradients_of_zero(coda):
    """No rows at all, and sequences without rows beside others"""
    heads, kv_heads, D, Tk = 4, 2, 64, 150
    Q, _, _ = qkv(0, heads, kv_heads, D, 1)
    _, K, V = qkv(Tk, heads, kv_heads, D, 2)
    dK, dV = (torch.full((Tk, kv_heads * D), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.empty((heads, 0), device="cuda")
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    coda.coda_attention_bwd(Q, K, V, Q, Q, lse, device([0, 0, 0]), Q, dK, dV, heads, kv_heads, D ** -0.5, ws, seq_k=device([0, 70, 140]))
    torch.cuda.synchronize()
    for x in (dK, dV):
        assert (x[:140] == 0).all() and (x[140:] == FILL).all()
    p = Pass(coda, [0, 40, 0], None, heads, kv_heads, D, True, seed=3)
    p.K, p.V = K, V
    p.k_at = [0, 33, 100, 150]
    p.seq_k = device(p.k_at)
    coda.coda_attention(p.Q, p.K, p.V, p.seq_q, p.out, heads, kv_heads, p.scale, lse=p.lse, seq_k=p.seq_k)
    p.full = p.full[:1] + [torch.empty((Tk, kv_heads * D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    p.check()
    dK, dV = p.grads()[1:]
    assert (dK[:33] == 0).all() and (dV[100:] == 0).all()


class Calls:
    """All calls over inputs that a stream makes just before them"""

    def __init__(self, coda):
        self.coda, self.heads, self.kv_heads, self.D = coda, 8, 2, 64
        self.T, self.room, self.page = 260, 600, 16
        self.src = torch.randn((self.T, 12 * 64), generator=torch.Generator().manual_seed(7)).cuda()
        self.dout = torch.randn((self.T, 512), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
        self.seq = device([0, 100, 100, 259])
        self.rows_at, self.lens = device([0, 5, 6, 40]), device([300, 1, 511])
        self.order = torch.randperm(3 * 38).to(torch.int32).view(3, 38).cuda()
        self.slots = torch.randperm(3 * 38 * 16)[: self.T].to(torch.int32).cuda()
        self.filled = torch.randn((2, 3 * 38, 2, 16, 64), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
        cos, sin = tables(300, 64)
        self.rope = (cos.cuda(), sin.cuda(), torch.arange(self.T, dtype=torch.int32, device="cuda"))
        self.x = torch.empty((self.T, 12 * 64), dtype=torch.bfloat16, device="cuda")
        self.cache = torch.empty_like(self.filled)
        self.ws = torch.empty(max(coda.coda_attention_bwd_workspace_bytes(self.T, self.T, 3, 8, 2, 64), coda.coda_attention_cached_workspace_bytes(self.T, 3, 8, 2, 64)),
                              dtype=torch.uint8, device="cuda")

    def outputs(self):
        return dict(out=torch.full((self.T, 512), FILL, dtype=torch.bfloat16, device="cuda"), lse=torch.full((8, self.T), FILL, device="cuda"),
                    grads=torch.full((self.T, 12 * 64), FILL, dtype=torch.bfloat16, device="cuda"),
                    cached=torch.full((self.T, 512), FILL, dtype=torch.bfloat16, device="cuda"), lse2=torch.full((8, self.T), FILL, device="cuda"))

    def blocks(self, x):
        return x[:, :512], x[:, 512:640], x[:, 640:]

    def run(self, o, stream=None):
        c, a = self.coda, (8, 2, 0.125)
        self.x.copy_(self.src)
        self.cache.copy_(self.filled)
        c.coda_attention(*self.blocks(self.x), self.seq, o["out"], *a, lse=o["lse"], stream=stream)
        c.coda_attention_bwd(*self.blocks(self.x), o["out"], self.dout, o["lse"], self.seq, *self.blocks(o["grads"]), *a, self.ws, rope=self.rope, stream=stream)
        c.coda_cache_store(self.x[:, 512:640], self.x[:, 640:], self.slots, self.cache[0], self.cache[1], stream=stream)
        c.coda_attention_cached(self.x[:, :512], self.cache[0], self.cache[1], self.order, self.lens, self.rows_at, o["cached"], 8, 0.125, self.ws, lse=o["lse2"], stream=stream)

    def eager(self):
        o = self.outputs()
        self.run(o)
        torch.cuda.synchronize()
        return o


def same(got, want, what):
    for k in want:
        assert torch.equal(got[k].view(torch.uint8), want[k].view(torch.uint8)), "%s: %s differs" % (what, k)


def test_on_another_stream(coda):
    """By argument and as the current one; the inputs are made on it, behind work that keeps it busy"""
    c = Calls(coda)
    want = c.eager()
    busy = torch.randn((4096, 4096), device="cuda")
    for given in (False, True):
        o, side = c.outputs(), torch.cuda.Stream()
        c.x.fill_(math.nan)
        c.cache.fill_(math.nan)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(3):
                busy @ busy
            c.run(o, side if given else None)
        side.synchronize()
        same(o, want, "given" if given else "current")


def test_captured_calls_follow_lengths_that_change_on_the_device(coda):
    c = Calls(coda)
    cap, side = c.outputs(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.run(cap)                                                   # kernels loaded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.run(cap)
    torch.cuda.synchronize()
    for seq, rows, lens in (([0, 100, 100, 259], [0, 5, 6, 40], [300, 1, 511]), ([0, 0, 0, 260], [0, 130, 130, 260], [130, 0, 608]), ([0, 1, 2, 3], [0, 1, 2, 3], [9, 9, 9]),
                            ([0, 0, 0, 0], [0, 0, 0, 0], [5, 5, 5]), ([7, 64, 128, 200], [3, 4, 5, 6], [608, 608, 608])):
        c.seq.copy_(device(seq))
        c.rows_at.copy_(device(rows))
        c.lens.copy_(device(lens))
        want = c.eager()                                             # eager work between the replays
        for _ in range(2):
            for x in cap.values():
                x.fill_(FILL)
            c.ws.fill_(0xA5)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            same(cap, want, "%s %s" % (seq, lens))


def test_two_graphs_share_a_workspace_one_after_the_other(coda):
    c, d = Calls(coda), Calls(coda)
    d.src.mul_(0.5)
    d.seq.copy_(device([0, 30, 200, 260]))
    d.rows_at.copy_(device([0, 1, 2, 3]))
    d.ws = c.ws
    want = c.eager(), d.eager()
    graphs, outs = [], []
    for x in (c, d):
        o, g, side = x.outputs(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            x.run(o)
        graphs.append(g)
        outs.append(o)
    for _ in range(3):
        for o in outs:
            for x in o.values():
                x.fill_(FILL)
        for i in (0, 1, 1, 0):
            graphs[i].replay()                                       # no wait between: one stream
        torch.cuda.synchronize()
        for i in (0, 1):
            same(outs[i], want[i], "graph %d" % i)
