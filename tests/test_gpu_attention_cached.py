"""coda_attention_cached and coda_cache_store against attention in 64 bits."""
import math

import pytest
import torch

from tests import attn_ref as R
from tests.test_gpu_attention import FILL, coda, device, offsets  # noqa: F401

pytestmark = pytest.mark.gpu


class Cache:
    """Sequences in shuffled pages; places that no sequence has are NaN, table entries behind a sequence's pages point outside the cache"""

    def __init__(self, coda, lens, rows, heads, kv_heads, D, page, seed, tree=None, spare=2, behind=0, size=1.0):
        self.coda, self.lens, self.rows, self.heads, self.kv_heads, self.D, self.page = coda, lens, rows, heads, kv_heads, D, page
        g = torch.Generator().manual_seed(seed)
        counts = [-(-n // page) for n in lens]
        self.pages = sum(counts) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        width = max(counts + [1])
        table, at = torch.full((len(lens), width + 3), 2 ** 31 - 1, dtype=torch.int32), 0
        self.k, self.v = (torch.full((self.pages, kv_heads, page, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        total = sum(lens)
        self.K, self.V = ((torch.randn((total, kv_heads * D), generator=g) * size).to(torch.bfloat16).cuda() for _ in range(2))
        slots = []
        for s, n in enumerate(lens):
            mine = order[at: at + counts[s]]
            at += counts[s]
            table[s, : counts[s]] = torch.tensor(mine, dtype=torch.int32)
            slots += [mine[j // page] * page + j % page for j in range(n)]
        self.slots = device(slots)
        coda.coda_cache_store(self.K, self.V, self.slots, self.k, self.v)
        self.table = table.cuda()[:, :width]                                             # a pitch of its own
        self.q_at = offsets(rows)
        T = self.q_at[-1] + behind
        self.Q = (torch.randn((T, heads * D), generator=g) * size).to(torch.bfloat16).cuda()
        self.tree = None
        if tree is not None:
            bits = [b for n in rows for b in tree(n)] + [0] * behind
            self.bits, self.tree = bits, device([b - 2 ** 64 if b >= 2 ** 63 else b for b in bits], torch.int64)
        self.seq_q, self.seq_lens = device(self.q_at), device(lens)
        self.ws = torch.empty(coda.coda_attention_cached_workspace_bytes(T, len(lens), heads, kv_heads, D), dtype=torch.uint8, device="cuda")
        self.scale = D ** -0.5

    def run(self, stats=True, stream=None):
        T = self.Q.shape[0]
        full = torch.full((T, self.Q.shape[1] + 8), FILL, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.heads, T), FILL, device="cuda") if stats else None
        self.ws.fill_(0xFF)
        torch.cuda.synchronize()
        self.call(full[:, :-8], lse, stream)
        torch.cuda.synchronize()
        assert (full[:, -8:] == FILL).all()
        return full[:, :-8].clone(), lse

    def call(self, out, lse, stream=None):
        self.coda.coda_attention_cached(self.Q, self.k, self.v, self.table, self.seq_lens, self.seq_q, out, self.heads, self.scale, self.ws, tree=self.tree, lse=lse,
                                        stream=stream)

    def expected(self):
        H, G, D, T = self.heads, self.kv_heads, self.D, self.Q.shape[0]
        out, b_out = torch.full((T, H * D), FILL, dtype=torch.float64), torch.zeros((T, H * D), dtype=torch.float64)
        lse, b_lse = torch.full((H, T), FILL, dtype=torch.float64), torch.zeros((H, T), dtype=torch.float64)
        k_at = offsets(self.lens)
        for s, (a, b) in enumerate(zip(self.q_at, self.q_at[1:])):
            K, V = self.K[k_at[s]: k_at[s + 1]], self.V[k_at[s]: k_at[s + 1]]
            see = R.visible(b - a, K.shape[0], True) if self.tree is None else R.tree_visible(b - a, K.shape[0], self.bits[a:b])
            for h in range(H):
                r = R.attend(R.head(self.Q[a:b], h, D), R.head(K, h * G // H, D), R.head(V, h * G // H, D), self.scale, see)
                out[a:b, h * D: (h + 1) * D], lse[h, a:b], b_out[a:b, h * D: (h + 1) * D], b_lse[h, a:b] = r
        return out, lse, b_out, b_lse

    def check(self):
        out, lse = self.run()
        o, m, b_o, b_m = self.expected()
        # joining parts: each part's sums are scaled by one exponential more
        R.check(out, o, b_o + 64 * R.F32 * o.abs(), "out")
        R.check(lse, m, b_m, "lse")


def some_tree(n):
    bits = []
    for i in range(n):
        parent = (i * 7 + 3) % i if i else -1
        bits.append((bits[parent] if parent >= 0 else 0) | 1 << i)
    return bits


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [1, 16, 64, 256])
@pytest.mark.parametrize("lens", [[1], [2, 31, 33], [700], [64, 65, 127, 128, 129, 255, 256, 257]])
def test_single_tokens(coda, lens, page, D):
    Cache(coda, lens, [1] * len(lens), 8, 2, D, page, seed=len(lens) + page).check()


@pytest.mark.parametrize("D", [8, 40, 72, 96, 120])
@pytest.mark.parametrize("rows", [[1, 1], [20, 3]])
def test_other_head_dimensions(coda, D, rows):
    Cache(coda, [150, 77], rows, 6, 2, D, 16, seed=D).check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (7, 1), (33, 1), (40, 1), (24, 3)])
def test_grouped_heads(coda, heads, kv_heads):
    """Groups that do not divide a tile of rows, and one of more heads than a tile has rows"""
    Cache(coda, [90, 41], [1, 1], heads, kv_heads, 64, 8, seed=heads).check()
    Cache(coda, [90, 41], [5, 2], heads, kv_heads, 64, 8, seed=heads).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [[2], [7, 1, 0, 40], [64, 33], [150]])
def test_chains(coda, rows, D):
    Cache(coda, [n + 37 * i for i, n in enumerate(rows)], rows, 4, 2, D, 16, seed=sum(rows)).check()
    Cache(coda, [n + 300 for n in rows], rows, 4, 1, D, 32, seed=sum(rows)).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [[1], [2, 3], [32, 5], [61], [64, 64, 0, 17]])
def test_trees(coda, rows, D):
    Cache(coda, [n + 101 + i for i, n in enumerate(rows)], rows, 4, 2, D, 16, seed=sum(rows), tree=some_tree).check()
    Cache(coda, list(rows), rows, 4, 1, D, 16, seed=sum(rows), tree=some_tree).check()


def test_trees_of_more_rows_than_bits(coda):
    """Rows from 64 on see what their bits say; keys from 64 on are seen by none"""
    Cache(coda, [120], [80], 2, 1, 64, 16, seed=3, tree=lambda n: [(i * 0x9E3779B97F4A7C15 + 1) % 2 ** 64 for i in range(n)]).check()


def test_rows_that_see_nothing(coda):
    """No bit set and no key ahead; no keys at all; fewer keys than rows"""
    Cache(coda, [5, 0, 20], [5, 3, 1], 4, 2, 64, 16, seed=4, tree=lambda n: [0] * n).check()
    Cache(coda, [3, 0, 20], [5, 3, 40], 4, 2, 64, 16, seed=5).check()
    Cache(coda, [0, 0], [1, 1], 4, 2, 128, 16, seed=5).check()


def test_rows_of_no_sequence_stay(coda):
    Cache(coda, [100, 50], [1, 2], 4, 2, 64, 16, seed=6, behind=5).check()


@pytest.mark.parametrize("lens", [[6000, 3, 1, 900], [4097], [1, 2, 3, 9000]])
def test_ranges_that_begin_and_end_within_sequences(coda, lens):
    Cache(coda, lens, [1] * len(lens), 8, 2, 64, 32, seed=7).check()
    Cache(coda, lens, [1] * len(lens), 2, 2, 128, 32, seed=7).check()


def test_more_sequences_than_threads(coda):
    lens = [1 + (i * 37) % 90 for i in range(600)]
    Cache(coda, lens, [(i % 3 > 0) * 1 for i in range(600)], 2, 1, 64, 16, seed=8).check()


def test_more_sequences_than_threads_in_tiles_of_128_rows(coda):
    lens = [40 + (i * 37) % 90 for i in range(300)]
    Cache(coda, lens, [(i % 3) * 10 for i in range(300)], 8, 1, 64, 16, seed=9).check()


def test_places_of_no_key_are_not_read(coda):
    """The cache of every test here is NaN where no sequence has a key; a page that ends inside a tile, and a sequence that ends inside a page"""
    c = Cache(coda, [67, 130], [1, 2], 4, 2, 128, 8, seed=10)
    assert torch.isnan(c.k).any() and torch.isfinite(c.run()[0]).all()


@pytest.mark.parametrize("rows", [4, 30])
def test_what_is_masked_has_no_effect(coda, rows):
    """A draft's key and value that are not finite reach only the rows that see it"""
    c = Cache(coda, [200], [rows], 4, 1, 128, 16, seed=11, tree=some_tree)
    clean, m0 = c.run()
    bad = 200 - rows + 2
    slot = int(c.slots[bad])
    c.v[slot // 16, :, slot % 16], c.k[slot // 16, :, slot % 16] = math.inf, math.nan
    out, m1 = c.run()
    sees = torch.tensor([b >> 2 & 1 for b in c.bits], dtype=torch.bool, device="cuda")
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(m1[:, ~sees], m0[:, ~sees]) and torch.isnan(out[sees]).all()
    assert 0 < int(sees.sum()) < rows
    c.k[slot // 16, :, slot % 16] = 0.0
    out, _ = c.run()
    assert torch.equal(out[~sees], clean[~sees]) and (out[sees] == math.inf).all()


def test_pages_and_lengths_out_of_range_stay_inside_the_cache(coda):
    """A page that does not exist is the nearest that does, a length beyond the table the table's"""
    c = Cache(coda, [40, 64], [1, 1], 4, 2, 64, 16, seed=12, spare=0)
    c.k.copy_(torch.nan_to_num(c.k))
    c.v.copy_(torch.nan_to_num(c.v))
    c.table[0, 0], c.table[1, 0] = -9, 2 ** 31 - 1
    a = c.run()
    c.table[0, 0], c.table[1, 0] = 0, c.pages - 1
    b = c.run()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.seq_lens[1], c.seq_lens[0] = 2 ** 31 - 1, -3
    out, lse = c.run()
    assert torch.equal(out[1], b[0][1]) and (out[0] == 0).all() and (lse[:, 0] == -math.inf).all()


def test_offsets_out_of_range_write_nothing_outside(coda):
    c = Cache(coda, [40, 64], [3, 4], 4, 2, 64, 16, seed=13)
    want = c.run()
    c.seq_q = device([-6, 3, 1000])
    out, lse = c.run()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_the_same_twice_and_without_lse(coda):
    c = Cache(coda, [3000, 1, 500], [3, 1, 9], 8, 2, 128, 16, seed=14)
    a, b = c.run(), c.run(stats=False)
    assert torch.equal(a[0], b[0]) and b[1] is None


def test_sequences_may_share_pages(coda):
    """A common beginning kept once"""
    c = Cache(coda, [128, 128], [1, 1], 4, 2, 64, 16, seed=15)
    c.table[1] = c.table[0]
    c.Q[1] = c.Q[0]
    out, _ = c.run()
    assert torch.equal(out[0], out[1])


def test_a_cache_past_4_gib(coda):
    """Slots whose elements lie beyond 2^32 bytes"""
    pages, page, G, D = 20000, 128, 8, 128                                               # 5.2 GB each
    k, v = (torch.full((pages, G, page, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = 200
    g = torch.Generator().manual_seed(16)
    K, V, Q = (torch.randn((r, w * D), generator=g).to(torch.bfloat16).cuda() for r, w in ((n, G), (n, G), (1, 2 * G)))
    mine = [pages - 1, pages - 7]
    slots = device([mine[j // page] * page + j % page for j in range(n)])
    coda.coda_cache_store(K, V, slots, k, v)
    ws = torch.empty(coda.coda_attention_cached_workspace_bytes(1, 1, 2 * G, G, D), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(Q)
    coda.coda_attention_cached(Q, k, v, device([mine]), device([n]), device([0, 1]), out, 2 * G, 0.1, ws)
    torch.cuda.synchronize()
    for h in range(2 * G):
        o, _, b_o, _ = R.attend(R.head(Q, h, D), R.head(K, h // 2, D), R.head(V, h // 2, D), 0.1, R.visible(1, n, True))
        R.check(out[:, h * D: (h + 1) * D], o, b_o + 64 * R.F32 * o.abs(), "head %d" % h)


# ---------------------------------------------------------------- storing
@pytest.mark.parametrize("D", [8, 64, 80, 128])
@pytest.mark.parametrize("T,page", [(1, 1), (5, 16), (300, 64)])
def test_store(coda, T, page, D):
    G, pages = 3, -(-T // page) + 2
    g = torch.Generator().manual_seed(T + D)
    qkv = torch.randn((T, 4 * G * D), generator=g).to(torch.bfloat16).cuda()
    K, V = qkv[:, G * D: 2 * G * D], qkv[:, 2 * G * D: 3 * G * D]
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    left_out = torch.rand(T, generator=g) < 0.3
    slots[left_out] = torch.tensor([-1, -7, pages * page, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(left_out.sum())) % 4]
    k, v = (torch.full((pages + 2, G, page, D), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    coda.coda_cache_store(K, V, slots.cuda(), k[1:-1], v[1:-1])
    torch.cuda.synchronize()
    for cache, rows in ((k, K), (v, V)):
        want = torch.full((pages + 2, G, page, D), FILL, dtype=torch.bfloat16)
        for t in range(T):
            s = int(slots[t])
            if 0 <= s < pages * page:
                want[1 + s // page, :, s % page] = rows[t].cpu().view(G, D)
        assert torch.equal(cache.cpu(), want)
