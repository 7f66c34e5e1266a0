"""Attention between the QKV projection and the output projection, for timing and for comparing outputs.

Each case is one pass through one operator, called the way a training or serving program calls it (outputs and scratch buffers kept
between passes), or, where `own` is false, computed in elementary torch operations in 32 bits:

  prompt   attention over whole prompts or packed training sequences, grouped heads -> output, log-sum-exp
  grad     its backward pass from the saved output and log-sum-exp -> gradients of Q, K and V, turned back through RoPE where the case says so
  cached   attention of single tokens, chains or trees of drafted tokens over a paged cache -> output, log-sum-exp
  store    rows of K and V into the pages of a cache

Q, K and V are column blocks of one matrix [tokens x (heads + 2 kv_heads) * dim], as one QKV projection leaves them, and the gradients
are column blocks of another.  `lens` are the new tokens of each sequence, `past` keys lie ahead of them (prompt, grad: in K and V;
cached: `lens` are the keys in the cache, of which the last `drafts` belong to the rows).
"""
import math

import torch

own = False


def _text(numbers):
    return " ".join(str(int(n)) for n in numbers)


def _numbers(text):
    return [int(n) for n in text.split()]


_1B = {"heads": 32, "kv_heads": 8, "dim": 64}       # 1B-style: hidden size 2048
_8B = {"heads": 32, "kv_heads": 8, "dim": 128}      # 8B-style: hidden size 4096


def listed():
    return [
        # one short prompt of an odd length
        dict(_1B, name="prompt-509", path="prompt", lens="509", past=0, causal=True),
        # a training batch of documents of very different lengths, packed
        dict(_8B, name="prompt-packed-8192", path="prompt", lens="4096 1777 1023 1 812 483", past=0, causal=True),
        # one long prompt
        dict(_8B, name="prompt-16384", path="prompt", lens="16384", past=0, causal=True),
        # the backward pass of two short sequences of odd lengths
        dict(_1B, name="grad-1000", path="grad", lens="619 381", past=0, causal=True, rope=True),
        # the 1B-style training step
        dict(_1B, name="grad-4x2048", path="grad", lens="2048 2048 2048 2048", past=0, causal=True, rope=True),
        # the 8B-style training step on packed documents
        dict(_8B, name="grad-packed-8192", path="grad", lens="4096 1777 1023 1 812 483", past=0, causal=True, rope=True),
        # one sequence decoding: all latency
        dict(_8B, name="cached-1x4097", path="cached", lens="4097", drafts=1, tree=False, page=16),
        # a serving batch of sequences of all lengths, a token each
        dict(_8B, name="cached-64", path="cached", lens=_text(1 + (i * 4099 + 977) % 8192 for i in range(64)), drafts=1, tree=False, page=64),
        # eight sequences that check trees of 32 drafted tokens
        dict(_8B, name="cached-tree-8x32", path="cached", lens="2081 4000 611 8191 5234 96 3333 7040", drafts=32, tree=True, page=16),
        # one long sequence with a tree of an odd size
        dict(_1B, name="cached-tree-61", path="cached", lens="16411", drafts=61, tree=True, page=128),
        # the new token of every sequence of a serving batch
        dict(_8B, name="store-64", path="store", lens=_text([1] * 64), page=64),
        # a long prompt into its pages
        dict(_8B, name="store-16384", path="store", lens="16384", page=64),
    ]


_LARGEST = {"prompt": 0.5 * 16384 * 16384 * 32 * 128, "grad": 1.1e7 * 32 * 128, "cached": 64 * 4096 * 8 * 128, "store": 16384 * 8 * 128}


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    path = rng.choice(["prompt", "prompt", "grad", "grad", "grad", "cached", "cached", "cached", "store"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    case = {"path": path, "kv_heads": kv_heads, "heads": kv_heads * rng.choice([1, 2, 3, 4, 4, 7, 8]), "dim": rng.choice([64, 64, 128, 128, 128, 40, 80, 96])}
    case["heads"] = min(case["heads"], 32 // kv_heads * kv_heads)
    if path in ("prompt", "grad"):
        # the gradients of a lone key's row are zero: a batch of such rows alone is none that is trained on
        total = _log_int(rng, 1 if path == "prompt" else 64, 8192)
        count = min(total, _log_int(rng, 1, 12))
        cuts = sorted(rng.sample(range(1, total), count - 1)) if count > 1 else []
        lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        case.update(lens=_text(lens), past=rng.choice([0, 0, 0, _log_int(rng, 1, 2048)]), causal=rng.random() < 0.85)
        if path == "grad":
            case["rope"] = rng.random() < 0.6
            if case["past"] and not case["causal"]:
                case["past"] = 0
        while _pairs(case) * case["heads"] * case["dim"] > _LARGEST[path]:
            lens = [(n + 1) // 2 for n in lens]
            case.update(lens=_text(lens), past=case["past"] // 2)
        return case
    case["page"] = rng.choice([1, 8, 16, 32, 64, 128, 256])
    if path == "store":
        case["lens"] = _text(_log_int(rng, 1, 512) for _ in range(_log_int(rng, 1, 32)))
        return case
    case["tree"] = rng.random() < 0.5
    case["drafts"] = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
    longest = _log_int(rng, 64, 32768)
    lens = [max(case["drafts"], rng.randint(1, longest)) for _ in range(_log_int(rng, 1, 64))]
    while sum(lens) * case["kv_heads"] * case["dim"] > _LARGEST["cached"] or sum(lens) * case["drafts"] > 2 ** 21:
        lens = [max(case["drafts"], n // 2) for n in lens[: max(1, len(lens) * 3 // 4)]]
    case["lens"] = _text(lens)
    return case


def _pairs(case):
    """Visible (row, key) pairs of one head."""
    n = _numbers(case["lens"])
    if case["path"] == "cached":
        d = case["drafts"]
        if case["tree"]:
            return sum((k - d) * d for k in n) + len(n) * sum(bin(m).count("1") for m in _tree(d))
        return sum((k - d) * d + d * (d + 1) // 2 for k in n)
    return sum(q * case["past"] + (q * (q + 1) // 2 if case["causal"] else q * q) for q in n)


def _tree(drafts):
    """Bits of the drafts that each draft sees: itself and those it follows.  Every second draft follows the one before it, the others an earlier one."""
    masks = []
    for i in range(drafts):
        parent = i - 1 if i % 2 else (i * 7 + 3) % i if i else -1
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
    return masks


# ---------------------------------------------------------------- inputs and buffers
def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _device(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).cuda()


def _qkv(case, rows, g):
    """Projections with some channels of K that are larger than the rest, and rows of different size."""
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    x = torch.randn((rows, (H + 2 * G) * D), device="cuda", dtype=torch.bfloat16, generator=g)
    channel = torch.ones((H + 2 * G) * D, device="cuda")
    channel[H * D: (H + G) * D].masked_fill_(torch.rand(G * D, device="cuda", generator=g) < 0.03, 4.0)
    row = torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))
    return x.mul_(channel.to(x.dtype)).mul_(row.to(x.dtype))


def _blocks(x, case):
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    return x[:, : H * D], x[:, H * D: (H + G) * D], x[:, (H + G) * D:]


def _u8(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    path, H, G, D = case["path"], case["heads"], case["kv_heads"], case["dim"]
    lens = _numbers(case["lens"])
    s = {"case": dict(case), "lens": lens, "scale": D ** -0.5}
    if path in ("prompt", "grad"):
        T, past = sum(lens), case["past"]
        s["q_at"], s["k_at"] = _offsets(lens), _offsets([n + past for n in lens])
        s["seq_q"] = _device(s["q_at"])
        s["seq_k"] = _device(s["k_at"]) if past else None
        s["Q"], K, V = _blocks(_qkv(case, T, g), case)
        if past:
            _, K, V = _blocks(_qkv(case, s["k_at"][-1], g), case)
        s["K"], s["V"] = K, V
        s["out"] = torch.zeros((T, H * D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((H, T), dtype=torch.float32, device="cuda")
        if path == "grad":
            saved = _plain_prompt(s)
            s["out"], s["lse"] = saved["out"], saved["lse"]
            s["dout"] = torch.randn((T, H * D), device="cuda", dtype=torch.bfloat16, generator=g).mul_(1e-2)
            s["dQ"], dK, dV = _blocks(torch.zeros((T, (H + 2 * G) * D), dtype=torch.bfloat16, device="cuda"), case)
            if past:
                _, dK, dV = _blocks(torch.zeros((s["k_at"][-1], (H + 2 * G) * D), dtype=torch.bfloat16, device="cuda"), case)
            s["dK"], s["dV"] = dK, dV
            if case["rope"]:
                rows = max(lens) + past
                angle = torch.arange(rows, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
                s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
                s["pos_k"] = _device([p for n in lens for p in range(n + past)])
                s["pos_q"] = _device([p for n in lens for p in range(past, n + past)]) if past else s["pos_k"]
            if own:
                from paper_2605_19269_amd import coda
                s["ws"] = _u8(coda.coda_attention_bwd_workspace_bytes(T, s["k_at"][-1], len(lens), H, G, D))
        return s
    page = case["page"]
    counts = [(n + page - 1) // page for n in lens]
    total = sum(counts) + 3
    order = torch.randperm(total, device="cuda", generator=g).cpu().tolist()
    s["pages"] = [order[a: a + n] for a, n in zip(_offsets(counts), counts)]
    if path == "store":
        T = sum(lens)
        _, s["K"], s["V"] = _blocks(_qkv(case, T, g), case)
        s["slots"] = _device([p[i // page] * page + i % page for n, p in zip(lens, s["pages"]) for i in range(n)])
        s["cache_k"], s["cache_v"] = (torch.zeros((total, G, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    _, K, V = _blocks(_qkv(case, total * page, g), case)
    s["cache_k"], s["cache_v"] = (x.reshape(total, page, G, D).permute(0, 2, 1, 3).contiguous() for x in (K, V))
    T = len(lens) * case["drafts"]
    s["Q"] = _blocks(_qkv(case, T, g), case)[0]
    s["q_at"] = _offsets([case["drafts"]] * len(lens))
    s["seq_q"], s["seq_lens"] = _device(s["q_at"]), _device(lens)
    s["table"] = _device([p + [0] * (max(counts) - len(p)) for p in s["pages"]])
    if case["tree"]:
        bits = [m - 2 ** 64 if m >= 2 ** 63 else m for m in _tree(case["drafts"])]
        s["tree"] = _device(bits * len(lens), torch.int64)
    s["out"] = torch.zeros((T, H * D), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((H, T), dtype=torch.float32, device="cuda")
    if own:
        from paper_2605_19269_amd import coda
        s["ws"] = _u8(coda.coda_attention_cached_workspace_bytes(T, len(lens), H, G, D))
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["path"]](s)


def _own_prompt(s):
    from paper_2605_19269_amd import coda
    c = s["case"]
    coda.coda_attention(s["Q"], s["K"], s["V"], s["seq_q"], s["out"], c["heads"], c["kv_heads"], s["scale"], lse=s["lse"], seq_k=s["seq_k"], causal=c["causal"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_grad(s):
    from paper_2605_19269_amd import coda
    c = s["case"]
    rope = (s["cos"], s["sin"], s["pos_q"], s["pos_k"]) if c["rope"] else None
    coda.coda_attention_bwd(s["Q"], s["K"], s["V"], s["out"], s["dout"], s["lse"], s["seq_q"], s["dQ"], s["dK"], s["dV"], c["heads"], c["kv_heads"], s["scale"],
                            s["ws"], seq_k=s["seq_k"], causal=c["causal"], rope=rope)
    return {"dQ": s["dQ"], "dK": s["dK"], "dV": s["dV"]}


def _own_cached(s):
    from paper_2605_19269_amd import coda
    coda.coda_attention_cached(s["Q"], s["cache_k"], s["cache_v"], s["table"], s["seq_lens"], s["seq_q"], s["out"], s["case"]["heads"], s["scale"], s["ws"],
                               tree=s.get("tree"), lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_store(s):
    from paper_2605_19269_amd import coda
    coda.coda_cache_store(s["K"], s["V"], s["slots"], s["cache_k"], s["cache_v"])
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}


_OWN = {"prompt": _own_prompt, "grad": _own_grad, "cached": _own_cached, "store": _own_store}

_CHUNK = 1 << 28        # elements of a matrix of scores that the plain form holds at once


def _by_head(x, heads):
    """[rows x heads * dim] -> fp32 [heads x rows x dim]"""
    return x.float().reshape(x.shape[0], heads, -1).transpose(0, 1).contiguous()


def _chain_mask(rows, keys):
    """Row i sees the keys up to i + keys - rows."""
    i, j = torch.arange(rows, device="cuda"), torch.arange(keys, device="cuda")
    return j[None, :] <= i[:, None] + (keys - rows)


def _weights(q, kt, scale, mask):
    """Scores of [h x r x d] and [h x d x k] -> (exponentials over their row's maximum, their sums, log-sum-exp)."""
    x = torch.matmul(q, kt).mul_(scale)
    if mask is not None:
        x.masked_fill_(~mask, -math.inf)
    m = x.amax(2, keepdim=True)
    p = torch.exp(x.sub_(m.clamp_min(-3e38)))
    total = p.sum(2, keepdim=True)
    return p, total, (m + torch.log(total)).squeeze(2)


def _attend(q, k, v, scale, mask):
    """fp32 q [H x r x d], k and v [G x n x d] -> (outputs [H x r x d], log-sum-exp [H x r])"""
    group, scores = q.shape[0] // k.shape[0], q.shape[1] * k.shape[1]
    if q.shape[0] * scores <= _CHUNK:                                       # all heads at once: rows of a group side by side
        p, total, lse = _weights(q.reshape(k.shape[0], group * q.shape[1], -1), k.transpose(1, 2).contiguous(), scale, None if mask is None else mask.repeat(group, 1))
        o = torch.matmul(p, v) / total.clamp_min(1e-38)
        return o.reshape(q.shape), lse.reshape(q.shape[:2])
    outs, lses, step = [], [], max(1, _CHUNK // scores)
    for g in range(k.shape[0]):
        kt = k[g].t().contiguous()[None]
        for h in range(g * group, (g + 1) * group, step):
            rows = q[h: min(h + step, (g + 1) * group)]
            p, total, lse = _weights(rows.reshape(1, -1, q.shape[2]), kt, scale, None if mask is None else mask.repeat(rows.shape[0], 1))
            outs.append((torch.matmul(p, v[g][None]) / total.clamp_min(1e-38)).reshape(rows.shape))
            lses.append(lse.reshape(rows.shape[:2]))
    return torch.cat(outs), torch.cat(lses)


def _plain_prompt(s):
    c = s["case"]
    H, G = c["heads"], c["kv_heads"]
    outs, lses = [], []
    for a, b, ka, kb in zip(s["q_at"], s["q_at"][1:], s["k_at"], s["k_at"][1:]):
        o, lse = _attend(_by_head(s["Q"][a:b], H), _by_head(s["K"][ka:kb], G), _by_head(s["V"][ka:kb], G), s["scale"],
                         _chain_mask(b - a, kb - ka) if c["causal"] else None)
        outs.append(o.transpose(0, 1).reshape(b - a, -1).to(torch.bfloat16))
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses, 1)}


def _turn_back(x, cos, sin, pos):
    """Adjacent pairs of fp32 [H x rows x dim] turned by minus the angle of their row."""
    c, n = cos[pos.long()], sin[pos.long()]
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c + b * n, b * c - a * n), -1).reshape(x.shape)


def _plain_grad(s):
    c = s["case"]
    H, G, group = c["heads"], c["kv_heads"], c["heads"] // c["kv_heads"]
    grads = [], [], []
    for a, b, ka, kb in zip(s["q_at"], s["q_at"][1:], s["k_at"], s["k_at"][1:]):
        q, o, do = (_by_head(s[n][a:b], H) for n in ("Q", "out", "dout"))
        k, v = (_by_head(s[n][ka:kb], G) for n in ("K", "V"))
        lse, delta = s["lse"][:, a:b], (o * do).sum(2)
        mask = _chain_mask(b - a, kb - ka) if c["causal"] else None
        step = max(1, min(G, _CHUNK // (group * (b - a) * (kb - ka))))      # groups at once
        parts = [], [], []
        for g in range(0, G, step):
            n = min(step, G - g)
            rows = lambda x: x[g * group: (g + n) * group].reshape((n, group * (b - a)) + x.shape[2:])
            p = torch.matmul(rows(q), k[g:g + n].transpose(1, 2).contiguous()).mul_(s["scale"]).sub_(rows(lse)[:, :, None]).exp_()
            if mask is not None:
                p.masked_fill_(~mask.repeat(group, 1), 0.0)
            parts[2].append(torch.matmul(p.transpose(1, 2).contiguous(), rows(do)))
            ds = torch.matmul(rows(do), v[g:g + n].transpose(1, 2).contiguous()).sub_(rows(delta)[:, :, None]).mul_(p).mul_(s["scale"])
            parts[0].append(torch.matmul(ds, k[g:g + n]).reshape(n * group, b - a, -1))
            parts[1].append(torch.matmul(ds.transpose(1, 2).contiguous(), rows(q)))
        dq, dk, dv = (torch.cat(x) for x in parts)
        if c["rope"]:
            dq = _turn_back(dq, s["cos"], s["sin"], s["pos_q"][a:b])
            dk = _turn_back(dk, s["cos"], s["sin"], s["pos_k"][ka:kb])
        for x, all_of in zip((dq, dk, dv), grads):
            all_of.append(x.transpose(0, 1).reshape(x.shape[1], -1).to(torch.bfloat16))
    return {n: torch.cat(x) for n, x in zip(("dQ", "dK", "dV"), grads)}


def _paged(cache, pages, keys):
    """fp32 [G x keys x dim] of one sequence"""
    x = cache[pages]                                                        # [pages x G x page x dim]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :keys].float()


def _plain_cached(s):
    c = s["case"]
    outs, lses = [], []
    for i, (a, b, n) in enumerate(zip(s["q_at"], s["q_at"][1:], s["lens"])):
        pages = s["table"][i, : len(s["pages"][i])].long()
        mask = _chain_mask(b - a, n)
        if c["tree"]:
            bits = s["tree"][a:b, None] >> torch.arange(b - a, device="cuda")[None, :] & 1
            mask = torch.cat((torch.ones((b - a, n - (b - a)), dtype=torch.bool, device="cuda"), bits.bool()), 1)
        o, lse = _attend(_by_head(s["Q"][a:b], c["heads"]), _paged(s["cache_k"], pages, n), _paged(s["cache_v"], pages, n), s["scale"], mask)
        outs.append(o.transpose(0, 1).reshape(b - a, -1).to(torch.bfloat16))
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses, 1)}


def _plain_store(s):
    page, at = s["case"]["page"], s["slots"].long()
    shape = (at.numel(), s["case"]["kv_heads"], -1)
    s["cache_k"][at // page, :, at % page] = s["K"].reshape(shape)
    s["cache_v"][at // page, :, at % page] = s["V"].reshape(shape)
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}


_PLAIN = {"prompt": _plain_prompt, "grad": _plain_grad, "cached": _plain_cached, "store": _plain_store}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Every input read once, every output written once; operations of the matrix products over the visible pairs only (two products
    forward, five backward)."""
    H, G, D, lens = case["heads"], case["kv_heads"], case["dim"], _numbers(case["lens"])
    if case["path"] == "store":
        return {"bytes": sum(lens) * (8.0 * G * D + 4), "flops": 0.0}
    if case["path"] == "cached":
        rows = len(lens) * case["drafts"]
        nbytes = 4.0 * sum(lens) * G * D + rows * H * (4.0 * D + 4) + 4 * sum((n + case["page"] - 1) // case["page"] for n in lens) + (8 * rows if case["tree"] else 0)
        return {"bytes": nbytes, "flops": 4.0 * D * H * _pairs(case)}
    rows, keys = sum(lens), sum(lens) + len(lens) * case["past"]
    if case["path"] == "prompt":
        return {"bytes": rows * H * (4.0 * D + 4) + 4.0 * keys * G * D, "flops": 4.0 * D * H * _pairs(case)}
    tables = 4.0 * D * (max(lens) + case["past"]) + 4 * (rows + keys if case["past"] else rows) if case["rope"] else 0
    return {"bytes": rows * H * (8.0 * D + 4) + 8.0 * keys * G * D + tables, "flops": 10.0 * D * H * _pairs(case)}


# ---------------------------------------------------------------- the operators' definition in 64 bits
def _visible(case, i, rows, keys, first, count):
    """Truth values [count x keys] of rows first .. of sequence i, or None where all is visible."""
    if case["path"] == "cached" and case["tree"]:
        see = torch.ones((rows, keys), dtype=torch.bool)
        for r, bits in enumerate(_tree(rows)):
            see[r, keys - rows:] = torch.tensor([bits >> j & 1 for j in range(rows)], dtype=torch.bool)
        return see[first: first + count].cuda()
    if case["path"] != "cached" and not case["causal"]:
        return None
    return torch.ones((rows, keys), dtype=torch.bool, device="cuda").tril(keys - rows)[first: first + count]


def _head(x, h, D):
    return x[:, h * D: (h + 1) * D].double()


def _wide_attention(case, i, Q, K, V, scale):
    """One sequence, head by head and a few thousand rows at a time."""
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    rows, keys = Q.shape[0], K.shape[0]
    out = torch.empty((rows, H * D), dtype=torch.float64, device="cuda")
    lse = torch.empty((H, rows), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // keys)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        see = _visible(case, i, rows, keys, a, b - a)
        for h in range(H):
            g = h * G // H
            x = torch.mm(_head(Q[a:b], h, D), _head(K, g, D).t()) * scale
            if see is not None:
                x = torch.where(see, x, torch.full_like(x, -math.inf))
            lse[h, a:b] = torch.logsumexp(x, 1)
            out[a:b, h * D: (h + 1) * D] = torch.mm(torch.softmax(x, 1), _head(V, g, D))
    return out, lse


def _wide_gradients(case, s, i):
    H, G, D, scale = case["heads"], case["kv_heads"], case["dim"], s["scale"]
    a, b, ka, kb = s["q_at"][i], s["q_at"][i + 1], s["k_at"][i], s["k_at"][i + 1]
    dQ = torch.zeros((b - a, H * D), dtype=torch.float64, device="cuda")
    dK, dV = (torch.zeros((kb - ka, G * D), dtype=torch.float64, device="cuda") for _ in range(2))
    see = _visible(case, i, b - a, kb - ka, 0, b - a)
    for h in range(H):
        g = h * G // H
        at, kt = slice(h * D, (h + 1) * D), slice(g * D, (g + 1) * D)
        q, do, k, v = _head(s["Q"][a:b], h, D), _head(s["dout"][a:b], h, D), _head(s["K"][ka:kb], g, D), _head(s["V"][ka:kb], g, D)
        P = torch.exp(torch.mm(q, k.t()) * scale - s["lse"][h, a:b, None].double())
        if see is not None:
            P = torch.where(see, P, torch.zeros_like(P))
        dV[:, kt] += torch.mm(P.t(), do)
        dS = P * (torch.mm(do, v.t()) - (do * _head(s["out"][a:b], h, D)).sum(1)[:, None])
        dQ[:, at] = scale * torch.mm(dS, k)
        dK[:, kt] += scale * torch.mm(dS.t(), q)
    if case["rope"]:
        for x, pos, heads in ((dQ, s["pos_q"][a:b], H), (dK, s["pos_k"][ka:kb], G)):
            turn = torch.complex(s["cos"].double(), -s["sin"].double())[pos.long()]
            for h in range(heads):
                pair = torch.view_as_complex(x[:, h * D: (h + 1) * D].reshape(x.shape[0], D // 2, 2).contiguous())
                x[:, h * D: (h + 1) * D] = torch.view_as_real(pair * turn).reshape(x.shape[0], D)
    return dQ, dK, dV


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "store":
        k, v = s["cache_k"].double(), s["cache_v"].double()
        for cache, rows in ((k, s["K"]), (v, s["V"])):
            flat = cache.transpose(1, 2).reshape(-1, case["kv_heads"] * case["dim"]).clone()
            flat.index_copy_(0, s["slots"].long(), rows.double())
            cache.copy_(flat.reshape(cache.shape[0], case["page"], case["kv_heads"], case["dim"]).transpose(1, 2))
        return {"cache_k": k, "cache_v": v}
    if case["path"] == "grad":
        parts = [_wide_gradients(case, s, i) for i in range(len(s["lens"]))]
        return {n: torch.cat(x) for n, x in zip(("dQ", "dK", "dV"), zip(*parts))}
    parts = []
    for i, (a, b) in enumerate(zip(s["q_at"], s["q_at"][1:])):
        if case["path"] == "prompt":
            K, V = s["K"][s["k_at"][i]: s["k_at"][i + 1]], s["V"][s["k_at"][i]: s["k_at"][i + 1]]
        else:
            at = torch.tensor([s["pages"][i][j // case["page"]] * case["page"] + j % case["page"] for j in range(s["lens"][i])], device="cuda")
            K, V = (c.transpose(1, 2).reshape(-1, case["kv_heads"] * case["dim"])[at] for c in (s["cache_k"], s["cache_v"]))
        parts.append(_wide_attention(case, i, s["Q"][a:b], K, V, s["scale"]))
    return {"out": torch.cat([o for o, _ in parts]), "lse": torch.cat([m for _, m in parts], 1)}
