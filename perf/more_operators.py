"""What the operators of a verify step's rows are measured on, through the calls
a user makes of them: appending keys and values to a paged cache
(``append_kv``), attention over it (``attend``), and penalties, biases and
grammar masks on the logits (``adjust_logits``), each for the rows of several
sequences at once (``RowBatch``).

The row counts are the verify step's own: one greedy token, a token each of 32
sequences, token trees of up to 64 rows, a serving batch of drafts (about 850
rows), a prefill chunk of 2048; heads, vocabularies and contexts are those of
workloads/configs.py and batches.py, or generic.  With ``own`` false a pass is
the operator's plain form in elementary torch operations, 32 bits (the angles
of a rotation in 64: positions go up to a million).

The sizes of a case's sequences follow from the case alone; values, trees,
pages and tokens from the seed.
"""

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
NONE = -math.inf


# ------------------------------------------------------------------- the cases

def _attend(seqs, rows, ctx, heads, kv_heads, dim, page=16, dtype="f16", cap=0.0, window=0, slopes=False, docs=0,
            prefix=False, tree=False, pad=0):
    return {"op": "attend", "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "cap": cap,
            "window": window, "slopes": slopes, "docs": docs, "prefix": prefix, "tree": tree, "pad": pad}


def _append(seqs, rows, ctx, heads, kv_heads, dim, page=16, dtype="f16", cache="f16", rot=None, interleaved=False,
            query=True, tree=False, theta=5.0e5, pad=0):
    return {"op": "append", "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "cache": cache,
            "rot": dim if rot is None else rot, "interleaved": interleaved, "query": query, "tree": tree,
            "theta": theta, "pad": pad}


def _adjust(seqs, rows, history, vocab, dtype="f32", repetition=True, counts=True, prompt=0.5, bias=0, allowed=0.0,
            tree=False, write=True, pad=0):
    return {"op": "adjust", "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "ctx_lo": history[0],
            "ctx_hi": history[1], "vocab": vocab, "dtype": dtype, "repetition": repetition, "counts": counts,
            "prompt": prompt, "bias": bias, "allowed": allowed, "tree": tree, "write": write, "pad": pad}


def listed():
    return [
        # a greedy token of one sequence: latency, its keys read by the whole card
        {"name": "attend 1 token", **_attend(1, (1, 1), (2047, 2047), 32, 8, 128)},
        # a token each of a serving batch, capped scores, empty rows behind it
        {"name": "attend 32 tokens cap", **_attend(32, (1, 1), (1024, 8192), 32, 8, 128, 64, "bf16", cap=50.0, pad=3)},
        # token trees of the 32B shape's heads over long contexts
        {"name": "attend 8 trees", **_attend(8, (33, 64), (8192, 8192), 64, 8, 128, tree=True)},
        # a serving batch of chain drafts, a sliding window
        {"name": "attend drafts window", **_attend(32, (9, 44), (1024, 8192), 32, 8, 128, window=4096)},
        # a prefill chunk at the end of a long prompt: bound by the matrix cores
        {"name": "attend prompt 2048", **_attend(1, (2048, 2048), (14336, 14336), 32, 8, 128)},
        # packed prompts of odd lengths: wide heads, documents, a prefix that all rows see, a bias by distance, a cap
        {"name": "attend packed 256", **_attend(3, (701, 2999), (0, 500), 10, 5, 256, 128, "bf16", cap=30.0, slopes=True,
                                                docs=4, prefix=True)},
        # a greedy token's keys, values and query: latency
        {"name": "append 1 token", **_append(1, (1, 1), (2047, 2047), 32, 8, 128, dtype="f32")},
        # a serving batch of drafts from 32-bit projections (the verify step's numerics)
        {"name": "append drafts", **_append(32, (9, 44), (1024, 8192), 32, 8, 128, dtype="f32")},
        # long prompts in 16 bits far into their sequences, neighbouring pairs rotated in a part of an odd head
        {"name": "append prompts far", **_append(3, (4001, 6999), (100000, 1000000), 12, 4, 80, 64, "bf16", "bf16", 48, True,
                                                 theta=1.0e4)},
        # a greedy token: latency
        {"name": "adjust 1 row", **_adjust(1, (1, 1), (512, 512), 128256, bias=16)},
        # a token tree under a grammar, 16-bit logits of the 32B shape
        {"name": "adjust tree grammar", **_adjust(1, (33, 33), (4096, 4096), 152064, "f16", allowed=0.02, tree=True)},
        # a serving batch of drafts, everything at once
        {"name": "adjust drafts", **_adjust(32, (9, 44), (1024, 8192), 128256, bias=64, allowed=0.7)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _range(rng, lo, hi):
    a = _log_int(rng, lo, hi)
    return (a, a) if rng.random() < 0.5 else (max(lo, a // rng.choice((2, 3, 8))), a)


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        for key in w:
            largest[c["op"], key] = max(largest.get((c["op"], key), 0), w[key])
    op = rng.choice(("attend", "attend", "append", "adjust"))
    while True:
        c = {"attend": _draw_attend, "append": _draw_append, "adjust": _draw_adjust}[op](rng)
        w = work(c)
        if _plain_values(c) <= 1.2e9 and all(w[key] <= largest[op, key] for key in w):
            return c


def _draw_rows(rng, kind):
    """Sequences and their rows."""
    if kind == "token":
        return _log_int(rng, 1, 128), (1, 1)
    if kind == "tree":
        return _log_int(rng, 1, 16), _range(rng, 2, 64)
    if kind == "draft":
        return _log_int(rng, 1, 48), _range(rng, 2, 65)
    return _log_int(rng, 1, 6), _range(rng, 66, 4096)


def _draw_heads(rng):
    kv = rng.choice((1, 2, 4, 5, 8, 8))
    return kv * rng.choice((1, 2, 3, 4, 4, 7, 8)), kv, rng.choice((64, 64, 72, 96, 128, 128, 128, 256))


def _draw_attend(rng):
    kind = rng.choice(("token", "tree", "draft", "prompt"))
    seqs, rows = _draw_rows(rng, kind)
    heads, kv, dim = _draw_heads(rng)
    ctx = _range(rng, 1, 16384 if kind != "prompt" else 4096)
    if rng.random() < 0.3:
        ctx = (0, ctx[1])
    return _attend(seqs, rows, ctx, heads, kv, dim, rng.choice((16, 16, 32, 64, 128, 256)), rng.choice(("f16", "bf16")),
                   rng.choice((0.0, 0.0, 30.0, 50.0)), rng.choice((0, 0, _log_int(rng, 1, 4096))), rng.random() < 0.25,
                   rng.choice((0, 0, 5)), rng.random() < 0.25, kind == "tree", rng.choice((0, 0, 0, 7)))


def _draw_append(rng):
    kind = rng.choice(("token", "tree", "draft", "prompt", "prompt"))
    seqs, rows = _draw_rows(rng, kind)
    heads, kv, dim = _draw_heads(rng)
    ctx = _range(rng, 1, 16384 if rng.random() < 0.7 else 1000000)
    cache = rng.choice(("f16", "bf16"))
    return _append(seqs, rows, ctx, heads, kv, dim, rng.choice((16, 16, 32, 64, 128, 256)),
                   rng.choice(("f32", cache)), cache, rng.choice((dim, dim, dim // 2, dim // 4 * 2, 0)),
                   rng.random() < 0.4, rng.random() < 0.7, kind == "tree", rng.choice((1.0e4, 5.0e5, 1.0e6)),
                   rng.choice((0, 0, 0, 7)))


def _draw_adjust(rng):
    seqs, rows = _draw_rows(rng, rng.choice(("token", "tree", "tree", "draft")))
    tree = rows[1] <= 64 and rows[1] > 1 and rng.random() < 0.5
    return _adjust(seqs, rows, _range(rng, 1, 32768), rng.choice((4096, 32000, 32003, 50257, 128256, 152064)),
                   rng.choice(("f32", "f32", "f16", "bf16")), rng.random() < 0.7, rng.random() < 0.7,
                   rng.choice((0.0, 0.5, 1.0)), rng.choice((0, 0, 5, 300)), rng.choice((0.0, 0.0, 0.001, 0.05, 0.9)),
                   tree, rng.random() < 0.7, rng.choice((0, 0, 0, 5)))


def _sizes(case):
    """[(rows, context)] of the sequences, first document starts and prefixes: from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    out = []
    for _ in range(case["seqs"]):
        n, ctx = rng.randint(case["rows_lo"], case["rows_hi"]), rng.randint(case["ctx_lo"], case["ctx_hi"])
        cuts = sorted(rng.randrange(0, ctx + n) for _ in range(case.get("docs", 0)))
        prefix = rng.randint(0, ctx + n) if case.get("prefix") else 0
        out.append((n, ctx, cuts, prefix))
    return out


def _plain_values(case):
    """Values of the plain form's largest array."""
    s = _sizes(case)
    n, L = max(x[0] for x in s), max(x[0] + x[1] for x in s)
    if case["op"] == "attend":
        return case["seqs"] * max(n * case["heads"], 2 * case["kv_heads"] * case["dim"]) * L
    T = sum(x[0] for x in s) + case["pad"]
    if case["op"] == "append":
        return max(T * (case["heads"] + 2 * case["kv_heads"]) * case["dim"], case["seqs"] * L)
    return max(T * case["vocab"], case["seqs"] * L)


# ------------------------------------------------------------------- the inputs

def _starts(sizes):
    at = [0]
    for s in sizes:
        at.append(at[-1] + s[0])
    return at


def _parents(rng, n):
    """A token tree: each row's parent row, row 0 (the pending token) without one."""
    return [-1] + [rng.randrange(max(0, j - 8), j) for j in range(1, n)]


def _tree_masks(parents):
    """Bit j of row i: row j lies on its path (i itself included)."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return [m - (1 << 64) if m >> 63 else m for m in out]


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _data(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 23)
    rng = random.Random(seed * 7919 + 23)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32)
    sizes = _sizes(case)
    S, T = case["seqs"], sum(s[0] for s in sizes) + case["pad"]
    d = {"starts": _ints(_starts(sizes)), "lengths": _ints([s[0] + s[1] for s in sizes]), "tree": None}
    if case["tree"]:
        masks = [m for s in sizes for m in _tree_masks(_parents(rng, s[0]))]
        d["tree"] = _ints(masks + [0] * case["pad"], torch.int64)
    if case["op"] == "adjust":
        return {**d, **_logits(case, sizes, T, g, rnd)}
    H, D, page = case["kv_heads"], case["dim"], case["page"]
    whole = case["op"] == "attend"  # the append needs no page before its rows
    first = [0 if whole else s[1] // page for s in sizes]
    last = [-(-(s[0] + s[1]) // page) for s in sizes]
    need = sum(b - a for a, b in zip(first, last))
    n_pages = need + need // 8 + 1
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    pages = torch.full((S, max(last)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s in range(S):
        pages[s, first[s]: last[s]] = ids[at: at + last[s] - first[s]]
        at += last[s] - first[s]
    d["pages"] = pages
    cache = DTYPES[case["dtype"] if whole else case["cache"]]
    for name in ("k_cache", "v_cache"):
        d[name] = torch.empty(n_pages, H, page, D, dtype=cache, device="cuda").normal_(generator=g)
    if whole:
        d["q"] = rnd(T, case["heads"], D).to(cache)
        d["slopes"] = None
        if case["slopes"]:
            d["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["heads"] + 1, device="cuda") / case["heads"])
        d["first"] = d["prefix"] = None
        if case["docs"]:  # the first key of the document that a row belongs to
            d["first"] = _ints([max([c for c in s[2] if c <= s[1] + i], default=0) for s in sizes for i in range(s[0])]
                               + [0] * case["pad"])
        if case["prefix"]:
            d["prefix"] = _ints([s[3] for s in sizes])
        return d
    # what a fused projection gives: query, key and value heads side by side in a row
    both = rnd(T, case["heads"] + 2 * H, D).to(DTYPES[case["dtype"]])
    d["q"], d["k"], d["v"] = (x for x in both.split((case["heads"], H, H), dim=1))
    if not case["query"]:
        d["q"] = None
    d["freqs"] = None
    if case["rot"]:
        d["freqs"] = case["theta"] ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
    return d


def _logits(case, sizes, T, g, rnd):
    S, V, N = case["seqs"], case["vocab"], case["ctx_hi"] + 1
    uni = lambda *s: torch.rand(*s, generator=g, device="cuda")
    some = lambda *s: (uni(*s) ** 3 * V).to(torch.int32).clamp_(max=V - 1)  # low ids far more often
    l = 2.0 * rnd(T, V)
    history, tokens = some(S, N), some(T)
    # a model likes to repeat itself: 64 tokens of the history lead
    lead = history[:, :64].long()
    for s, at in enumerate(_starts(sizes)[:-1]):
        l[at: at + sizes[s][0], lead[s]] += 4.0
    d = {"logits": l.to(DTYPES[case["dtype"]]), "history": history, "tokens": tokens,
         "history_lengths": _ints([s[1] for s in sizes]), "prompt_lengths": _ints([int(case["prompt"] * s[1]) for s in sizes]),
         "repetition": None, "frequency": None, "presence": None, "bias_ids": None, "bias": None, "allowed": None}
    if case["repetition"]:
        d["repetition"] = 1.0 + 0.3 * uni(S)
    if case["counts"]:
        d["frequency"], d["presence"] = 0.5 * uni(S), uni(S) - 0.2
    if case["bias"]:  # ids of a sequence are distinct; one place is empty
        ids = torch.randint(0, V // case["bias"], (S, case["bias"]), generator=g, device="cuda")
        ids = (ids + torch.arange(case["bias"], device="cuda") * (V // case["bias"])).to(torch.int32)
        ids[:, case["bias"] // 2] = -1
        d["bias_ids"], d["bias"] = ids, 3.0 * rnd(S, case["bias"])
    if case["allowed"]:
        bits = (uni(T, -(-V // 32), 32) < case["allowed"]).to(torch.int64) << torch.arange(32, device="cuda")
        d["allowed"] = bits.sum(dim=2).to(torch.int32)
    return d


def prepare(case, seed):
    st = {"case": case, **_data(case, seed)}
    sizes = _sizes(case)
    st["n"], st["max_rows"] = sum(s[0] for s in sizes), max(s[0] for s in sizes)
    if own:
        import paper_2606_01019_amd as hvd
        # the step's rows, checked once: every layer's calls take the same
        st["batch"] = hvd.RowBatch(st["starts"], None if case["op"] == "adjust" else st["lengths"], st.get("pages"),
                                   tree=st["tree"])
    return st


# -------------------------------------------------------------------- one pass

def run(st):
    c = st["case"]
    if own:
        import paper_2606_01019_amd as hvd
        if c["op"] == "attend":
            return {"out": hvd.attend(st["q"], st["k_cache"], st["v_cache"], st["batch"], cap=c["cap"], window=c["window"],
                                      slopes=st["slopes"], first=st["first"], prefix=st["prefix"])}
        if c["op"] == "append":
            q = hvd.append_kv(st["k_cache"], st["v_cache"], st["k"], st["v"], st["batch"], q=st["q"], freqs=st["freqs"],
                              interleaved=c["interleaved"])
            return {"k_cache": st["k_cache"], "v_cache": st["v_cache"], "q": q}
        out, best = hvd.adjust_logits(st["logits"], st["batch"], tokens=st["tokens"], history=st["history"],
                                      history_lengths=st["history_lengths"], prompt_lengths=st["prompt_lengths"],
                                      repetition=st["repetition"], frequency=st["frequency"], presence=st["presence"],
                                      bias_ids=st["bias_ids"], bias=st["bias"], allowed=st["allowed"], write=c["write"])
        return {"logits": out, "best": best}
    return {"attend": _plain_attend, "append": _plain_append, "adjust": _plain_adjust}[c["op"]](st)


def _of_rows(st, T):
    """Each row's sequence and its place there; rows behind the last sequence count to none."""
    row = torch.arange(T, device="cuda")
    seq = torch.searchsorted(st["starts"][1:].long(), row, right=True)
    live = seq < len(st["starts"]) - 1
    seq = seq.clamp(max=len(st["starts"]) - 2)
    return seq, row - st["starts"].long()[seq], live


def _bits(mask, n):
    return (mask[..., None] >> torch.arange(n, device="cuda")) & 1


def _plain_attend(st):
    c, q = st["case"], st["q"]
    T, Hq, D = q.shape
    H, S, n = c["kv_heads"], c["seqs"], st["max_rows"]
    G = Hq // H
    pages = st["pages"].long().clamp(min=0)
    L = pages.shape[1] * c["page"]
    lens, starts = st["lengths"].long(), st["starts"].long()
    key = torch.arange(L, device="cuda")
    held = key < lens[:, None]  # [S, L]
    k = st["k_cache"][pages].permute(0, 2, 4, 1, 3).reshape(S, H, D, L).float()
    v = st["v_cache"][pages].permute(0, 2, 1, 3, 4).reshape(S, H, L, D).float()
    k, v = k * held[:, None, None], v * held[:, None, :, None]
    i = torch.arange(n, device="cuda")
    rows = (starts[:-1, None] + i).clamp(max=T - 1)  # [S, n]
    qs = q[rows].float().view(S, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * n, D)
    s = torch.matmul(qs, k).view(S, H, G, n, L) * D ** -0.5
    if c["cap"]:
        s = c["cap"] * torch.tanh(s / c["cap"])
    ctx = (lens - (starts[1:] - starts[:-1]))[:, None, None]  # [S, 1, 1]
    at = key[None, None, :].expand(S, n, L)  # positions of the keys as a row sees them
    mine = ctx[:, :, 0] + i
    past = at <= mine[:, :, None]
    if c["prefix"]:
        past = past | (at < st["prefix"].long()[:, None, None])
    if st["tree"] is not None:
        bit = _bits(st["tree"][rows], 64)  # [S, n, 64]
        depth = torch.cumsum(bit, dim=2)
        j = (at - ctx).clamp(0, 63)
        new = at >= ctx
        past = torch.where(new, (torch.gather(bit, 2, j) == 1) & (at - ctx < 64), past)
        at = torch.where(new, ctx + torch.gather(depth, 2, j) - 1, at)
        mine = ctx[:, :, 0] + depth[:, :, 63] - 1
    apart = mine[:, :, None] - at  # [S, n, L]
    if c["slopes"]:
        s = s - st["slopes"].view(1, H, G, 1, 1) * apart.abs()[:, None, None].float()
    seen = past & held[:, None]
    if c["window"]:
        seen = seen & (apart < c["window"])
    if c["docs"]:
        seen = seen & (key >= st["first"].long()[rows][:, :, None])
    s = s.masked_fill(~seen[:, None, None], NONE)
    top = s.amax(dim=4, keepdim=True)
    p = torch.exp(s - torch.where(top == NONE, torch.zeros_like(top), top))
    o = torch.matmul(p.view(S, H, G * n, L), v).view(S, H, G, n, D)
    total = p.sum(dim=4)[..., None]
    o = o / torch.where(total == 0.0, torch.ones_like(total), total)
    seq, local, live = _of_rows(st, T)
    o = o.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, D)[seq, local.clamp(max=n - 1)]
    return {"out": (o * live[:, None, None]).to(q.dtype)}


def _plain_append(st):
    c, n = st["case"], st["n"]
    T = st["k"].shape[0]
    seq, local, live = _of_rows(st, T)
    lens, starts = st["lengths"].long(), st["starts"].long()
    ctx = (lens - (starts[1:] - starts[:-1]))[seq]
    slot = ctx + local
    at = slot
    if st["tree"] is not None:
        at = ctx + _bits(st["tree"], 64).sum(dim=1) - 1

    def turn(x):
        x = x.float()
        r = c["rot"]
        if not r:
            return x
        angle = at.double()[:, None] * st["freqs"]
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        if c["interleaved"]:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=3).flatten(2)
        else:
            a, b = x[..., : r // 2], x[..., r // 2: r]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
        return torch.cat((y, x[..., r:]), dim=2)

    # (the rows behind the last sequence have no place in the cache)
    page = st["pages"].long()[seq[:n], (slot // c["page"])[:n]]
    off = (slot % c["page"])[:n]
    st["k_cache"][page, :, off] = turn(st["k"])[:n].to(st["k_cache"].dtype)
    st["v_cache"][page, :, off] = st["v"][:n].to(st["v_cache"].dtype)
    q = None
    if st["q"] is not None:
        q = (turn(st["q"]) * live[:, None, None]).to(st["k_cache"].dtype)
    return {"k_cache": st["k_cache"], "v_cache": st["v_cache"], "q": q}


def _plain_adjust(st):
    c = st["case"]
    x = st["logits"].float()
    T, V = x.shape
    S, n = c["seqs"], st["max_rows"]
    seq, local, live = _of_rows(st, T)
    place = torch.arange(st["history"].shape[1], device="cuda")
    history = st["history"].long()
    held = place < st["history_lengths"].long()[:, None]
    made = held & (place >= st["prompt_lengths"].long()[:, None])
    base = torch.zeros(S, V, dtype=torch.int32, device="cuda")
    said = base.scatter_add(1, history, made.int())[seq]  # tokens a sequence has generated
    seen = base.scatter_add(1, history, held.int())[seq] > 0  # and those of its prompt too
    # this step's own tokens on a row's path
    j = torch.arange(n, device="cuda")
    rows = (st["starts"].long()[seq][:, None] + j).clamp(max=T - 1)
    on = j <= local[:, None] if st["tree"] is None else _bits(st["tree"], 64)[:, :n] == 1
    on = on & (st["starts"].long()[seq][:, None] + j < st["starts"].long()[seq + 1][:, None])
    said = said.scatter_add(1, st["tokens"].long()[rows], on.int())
    seen = seen | (said > 0)
    of_row = lambda t: t[seq][:, None]
    if c["repetition"]:
        r = of_row(st["repetition"])
        x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    if c["counts"]:
        x = x - of_row(st["frequency"]) * said.float()
        x = x - of_row(st["presence"]) * (said > 0).float()
    if c["bias"]:
        ids = st["bias_ids"].long()
        table = torch.zeros(S, V, device="cuda").scatter_add(1, ids.clamp(min=0), torch.where(ids >= 0, st["bias"], 0.0))
        x = x + table[seq]
    x = torch.where(live[:, None], x, st["logits"].float())
    if c["allowed"]:
        col = torch.arange(V, device="cuda")
        ok = (st["allowed"][:, col >> 5] >> (col & 31)) & 1 == 1
        x = x.masked_fill(~ok & live[:, None], NONE)
    top, best = x.max(dim=1).values, torch.arange(V, device="cuda", dtype=torch.int32)
    best = torch.where(x == top[:, None], best, V).amin(dim=1)
    best = best.masked_fill((top == NONE) | ~live, -1).to(torch.int32)
    return {"logits": x.to(st["logits"].dtype) if c["write"] else None, "best": best}


# ------------------------------------------------------------- what a pass takes

def work(case):
    sizes = _sizes(case)
    T = sum(s[0] for s in sizes)
    if case["op"] == "append":
        values = T * case["dim"] * (2 * case["kv_heads"] + (case["heads"] if case["query"] else 0))
        return {"bytes": values * (BYTES[case["dtype"]] + BYTES[case["cache"]]), "flops": 3 * values}
    if case["op"] == "adjust":
        values = T * case["vocab"]
        return {"bytes": int(values * BYTES[case["dtype"]] * (1 + case["write"]) + (values / 8 if case["allowed"] else 0)
                             + 4 * sum(s[1] for s in sizes)), "flops": 4 * values}
    keys = pairs = 0
    for n, ctx, cuts, prefix in sizes:
        lo = ctx + n
        for i in range(n):
            depth = min(i, 8) if case["tree"] else i  # (a tree's paths are short)
            first = max([x for x in cuts if x <= ctx + i], default=0)
            if case["window"]:
                first = max(first, ctx + depth + 1 - case["window"])
            lo = min(lo, first)
            pairs += max(ctx + depth + 1, min(prefix, ctx + n)) - first
        keys += ctx + n - lo
    return {"bytes": 2 * case["dim"] * (2 * case["kv_heads"] * keys + 2 * case["heads"] * T),
            "flops": 4 * case["dim"] * case["heads"] * pairs}


# ------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    return {"attend": _exact_attend, "append": _exact_append, "adjust": _exact_adjust}[case["op"]](case, _data(case, seed))


def _path(parents_mask, i):
    m = parents_mask[i] % (1 << 64)
    return [j for j in range(64) if m >> j & 1]


def _exact_attend(case, d):
    sizes, page, D = _sizes(case), case["page"], case["dim"]
    H = case["kv_heads"]
    G = case["heads"] // H
    q = d["q"].double()
    out = torch.zeros_like(q)
    masks = None if d["tree"] is None else d["tree"].tolist()
    for s, (n, ctx, cuts, prefix) in enumerate(sizes):
        a, L = int(d["starts"][s]), ctx + n
        ids = d["pages"][s, : -(-L // page)].long()
        K, V = ([t[ids, h].reshape(-1, D)[:L].double() for h in range(H)] for t in (d["k_cache"], d["v_cache"]))
        where = torch.arange(L, dtype=torch.float64, device="cuda").repeat(n, 1)
        me = torch.arange(ctx, L, dtype=torch.float64, device="cuda")[:, None]
        see = (where <= me) | (where < prefix)
        if masks is not None:
            see[:, ctx:] = False
            depths = []
            for i in range(n):
                path = _path(masks[a: a + n], i)
                for step, j in enumerate(path):
                    see[i, ctx + j] = True
                    where[i, ctx + j] = ctx + step
                depths.append(float(ctx + len(path) - 1))
            me = torch.tensor(depths, dtype=torch.float64, device="cuda")[:, None]
        if case["window"]:
            see &= me - where < case["window"]
        if case["docs"]:
            for i in range(n):
                see[i, : max([c for c in cuts if c <= ctx + i], default=0)] = False
        for h in range(H * G):
            z = torch.mm(q[a: a + n, h].contiguous(), K[h // G].t().contiguous()) / math.sqrt(D)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["slopes"]:
                z -= 2.0 ** (-8.0 * (h + 1) / case["heads"]) * (me - where).abs()
            z[~see] = NONE
            out[a: a + n, h] = torch.mm(torch.nan_to_num(torch.softmax(z, dim=1)), V[h // G])
    return {"out": out}


def _exact_append(case, d):
    kc, vc = d["k_cache"].double(), d["v_cache"].double()
    q = None if d["q"] is None else torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda")
    masks = None if d["tree"] is None else d["tree"].tolist()
    r = case["rot"]
    for s, (n, ctx, _, _) in enumerate(_sizes(case)):
        a = int(d["starts"][s])
        slot = torch.arange(ctx, ctx + n, device="cuda")
        pos = slot.double()
        if masks is not None:
            pos = torch.tensor([float(ctx + len(_path(masks[a: a + n], i)) - 1) for i in range(n)], device="cuda",
                               dtype=torch.float64)
        pairs = torch.arange(r // 2, device="cuda")
        one, two = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + r // 2)
        for name in ("k", "v", "q"):
            if d[name] is None:
                continue
            z = d[name][a: a + n].double()
            if r and name != "v":
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, None, None] * d["freqs"])
                w = torch.complex(z[..., one], z[..., two]) * turn
                z[..., one], z[..., two] = w.real, w.imag
            if name == "q":
                q[a: a + n] = z
            else:
                dst = kc if name == "k" else vc
                dst[d["pages"][s].long()[slot // case["page"]], :, slot % case["page"]] = z
    return {"k_cache": kc, "v_cache": vc, "q": q}


def _exact_adjust(case, d):
    if not case["write"]:  # the best token alone: a comparison of 32-bit values
        return None
    V = case["vocab"]
    x = d["logits"].double()
    masks = None if d["tree"] is None else d["tree"].tolist()
    count = lambda t: torch.bincount(t.long(), minlength=V)
    for s, (n, size, _, _) in enumerate(_sizes(case)):
        a, prompt = int(d["starts"][s]), int(d["prompt_lengths"][s])
        base, before = count(d["history"][s, min(prompt, size): size]), count(d["history"][s, : min(prompt, size)])
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        if case["bias"]:
            real = d["bias_ids"][s] >= 0
            bias[d["bias_ids"][s][real].long()] = d["bias"][s][real].double()
        for i in range(n):
            path = list(range(i + 1)) if masks is None else _path(masks[a: a + n], i)
            said = base + count(d["tokens"][a: a + n][path])
            l = x[a + i]
            if case["repetition"]:
                r = d["repetition"][s].double()
                hit = (said + before) > 0
                l[hit] = torch.where(l[hit] > 0, l[hit] / r, l[hit] * r)
            if case["counts"]:
                l -= d["frequency"][s].double() * said + d["presence"][s].double() * (said > 0)
            l += bias
            if case["allowed"]:
                word = d["allowed"][a + i].long() & 0xFFFFFFFF
                ok = ((word[:, None] >> torch.arange(32, device="cuda")) & 1).flatten()[:V] == 1
                l[~ok] = NONE
    return {"logits": x, "best": None}
