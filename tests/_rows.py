"""Plain implementations of the operators on a step's rows, row by row from
their definitions in 64 bits (the adjusted logits in the 32-bit steps that the
operator promises), and makers of batches."""

import numpy as np
import torch


class Case:
    """Sequences with (rows, context) each, their pages dealt at random."""

    def __init__(self, sizes, H, D, page=16, dtype=torch.float16, seed=0, tree=False, pad=0, spare=3, device="cuda",
                 layout="head", max_pages=None):
        self.sizes, self.H, self.D, self.page, self.dtype, self.pad = sizes, H, D, page, dtype, pad
        self.g = torch.Generator().manual_seed(seed * 31 + 7)
        rng = np.random.default_rng(seed)
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in sizes])]).astype(np.int32)
        self.lengths = np.array([n + c for n, c in sizes], np.int32)
        self.T = int(self.starts[-1]) + pad
        need = [-(-(n + c) // page) for n, c in sizes]
        P = max(need + [1]) if max_pages is None else max_pages
        self.n_pages = sum(need) + spare
        ids = rng.permutation(self.n_pages).astype(np.int32)
        self.pages = np.full((len(sizes), P), -1, np.int32)
        at = 0
        for s, k in enumerate(need):
            self.pages[s, :k] = ids[at: at + k]
            at += k
        self.tree = None
        if tree:
            masks = []
            for n, _ in sizes:
                own = []
                for i in range(n):
                    p = int(rng.integers(max(0, i - 5), i)) if i else -1
                    own.append((own[p] if p >= 0 else 0) | 1 << i)
                masks += own
            self.tree = np.array([m - (1 << 64) if m >> 63 else m for m in masks] + [0] * pad, np.int64)
        shape = (self.n_pages, H, page, D) if layout == "head" else (self.n_pages, page, H, D)
        self.k_cache, self.v_cache = (self.rnd(*shape).to(dtype).to(device) for _ in range(2))
        if layout != "head":
            self.k_cache, self.v_cache = self.k_cache.transpose(1, 2), self.v_cache.transpose(1, 2)
        self.device = device

    def rnd(self, *shape):
        return torch.randn(*shape, generator=self.g)

    def batch(self, hvd, tree=True):
        t = lambda a: torch.from_numpy(a).to(self.device)
        return hvd.RowBatch(t(self.starts), t(self.lengths), t(self.pages), tree=t(self.tree) if tree and self.tree is not None else None)

    def rows(self):
        """(row, sequence, place in it, rows of it, context) of each row that has a sequence."""
        for s, (n, c) in enumerate(self.sizes):
            for i in range(n):
                yield int(self.starts[s]) + i, s, i, n, c

    def path(self, row):
        m = int(self.tree[row]) % (1 << 64)
        return [j for j in range(64) if m >> j & 1]


def attend_ref(case, q, scale=None, cap=0.0, window=0, slopes=None, first=None, prefix=None):
    """(out, tolerance) in 64 bits.  The tolerance counts, with u half a step of
    the cache's type: the output's rounding, u |out|; the weights' rounding, u A
    with A the weighted mean of |v|; the scores' 32-bit errors d, twice in a
    quotient of sums, 2 d A -- d counts D + 8 roundings of 2^-23 of the largest
    sum |q k| scale (sums in blocks may round towards 0), the exponential and tanh
    (a few 2^-23 of the score, or of the cap), the bias; the sums' own 32-bit
    roundings, n 2^-23 A; and what a weight below fp16's normal range loses, 2^-25
    of a largest weight of 2^7."""
    D, H, page = case.D, case.H, case.page
    Hq = q.shape[1]
    G = Hq // H
    scale = D ** -0.5 if scale is None else scale
    Q = q.double().cpu()
    K, V = case.k_cache.double().cpu(), case.v_cache.double().cpu()
    out = torch.zeros(q.shape, dtype=torch.float64)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    u = torch.finfo(q.dtype).eps / 2
    for row, s, i, n, ctx in case.rows():
        L = n + ctx
        keys, at = [], []
        path = None if case.tree is None else case.path(row)
        pos = ctx + i if path is None else ctx + len(path) - 1
        for j in range(L):
            if path is not None and j >= ctx:
                if j - ctx not in path:
                    continue
                p = ctx + path.index(j - ctx)
            else:
                p = j
                if not (p <= pos or (prefix is not None and j < int(prefix[s]))):
                    continue
            if window and not pos - p < window:
                continue
            if first is not None and j < int(first[row]):
                continue
            page_id = int(case.pages[s, j // page]) if j // page < case.pages.shape[1] else -1
            if not 0 <= page_id < case.n_pages:
                continue
            keys.append((page_id, j % page))
            at.append(p)
        if not keys:
            continue
        pg, tk = (torch.tensor(x) for x in zip(*keys))
        dist = (torch.tensor(at, dtype=torch.float64) - pos).abs()
        for h in range(Hq):
            k, v = K[pg, h // G, tk], V[pg, h // G, tk]
            x = k @ Q[row, h] * scale
            big = float((k.abs() @ Q[row, h].abs()).nan_to_num(0, 0, 0).max()) * abs(scale)
            d = (D + 8) * 2.0 ** -23 * big
            if cap:
                x = cap * torch.tanh(x / cap)
                d += 8 * 2.0 ** -23 * max(cap, big)
            if slopes is not None:
                x = x - float(slopes[h]) * dist
                d += 4 * 2.0 ** -23 * float(slopes[h]) * float(dist.max())
            top = x.max()
            if top == -np.inf:
                continue
            p = torch.exp(x - top)
            d += 8 * 2.0 ** -23 * float(x[x > -np.inf].abs().max().nan_to_num(0, 0, 0))
            p = p / p.sum()
            o = torch.where(p[:, None] > 0, p[:, None] * v, 0.0).sum(0)
            A = (p[:, None] * v.abs()).sum(0)
            out[row, h] = o
            tol[row, h] = 1.02 * (u * o.abs() + (u + 2 * d + len(keys) * 2.0 ** -23) * A + len(keys) * 2.0 ** -32 * v.abs().max(0).values)
    return out, tol


def check_attend(case, got, q, **kw):
    ref, tol = attend_ref(case, q, **kw)
    g = got.double().cpu()
    assert got.shape == q.shape and got.dtype == q.dtype
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(ref), torch.isnan(g))
    assert torch.equal(ref[~fine & ~torch.isnan(ref)], g[~fine & ~torch.isnan(ref)])
    bad = (g - ref).abs()[fine] - tol[fine]
    assert bad.numel() == 0 or float(bad.max()) <= 0, f"off by {float((g - ref).abs()[fine].max()):.3g}, {float(bad.max()):.3g} too much"


def append_ref(case, k, v, q=None, freqs=None, interleaved=False, positions=None):
    """The caches and queries after the call, and their tolerances, 64 bits: half a
    step of the type, and before it 8 roundings of 2^-24 of the pair's size (the
    fraction of a turn, the cosine and sine with up to 2 units, three operations)."""
    u = torch.finfo(case.dtype).eps / 2
    outs = {"k": case.k_cache.double().cpu().clone(), "v": case.v_cache.double().cpu().clone()}
    tols = {n: torch.zeros_like(t) for n, t in outs.items()}
    x = {"k": k, "v": v}
    if q is not None:
        x["q"] = q
        outs["q"] = torch.zeros(q.shape, dtype=torch.float64)
        tols["q"] = torch.zeros(q.shape, dtype=torch.float64)
    f = None if freqs is None else freqs.double().cpu()
    for row, s, i, n, ctx in case.rows():
        pos = ctx + i if case.tree is None else ctx + len(case.path(row)) - 1
        if positions is not None:
            pos = int(positions[row])
        for name, t in x.items():
            y = t[row].double().cpu().clone()
            size = y.abs()
            if f is not None and name != "v" and len(f):
                r = 2 * len(f)
                a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
                c, z = torch.cos(pos * f), torch.sin(pos * f)
                one, two = y[:, a].clone(), y[:, b].clone()
                y[:, a], y[:, b] = one * c - two * z, two * c + one * z
                size[:, a] = size[:, b] = one.abs() + two.abs()
                tol = u * y.abs() + 8 * 2.0 ** -24 * size
            else:
                tol = u * y.abs()
            if name == "q":
                outs[name][row], tols[name][row] = y, tol
                continue
            j = ctx + i
            if not 0 <= j // case.page < case.pages.shape[1]:
                continue
            page = int(case.pages[s, j // case.page])
            if 0 <= page < case.n_pages:
                outs[name][page, :, j % case.page], tols[name][page, :, j % case.page] = y, tol
    # (an fp16 below 2^-14 has a step of 2^-24)
    return outs, {n: t + (2.0 ** -25 if case.dtype == torch.float16 else 0) for n, t in tols.items()}


def adjust_ref(starts, logits, tree=None, tokens=None, history=None, history_lengths=None, prompt_lengths=None,
               repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, allowed=None):
    """(adjusted float32 [rows, vocab], best): every step is a float32 operation."""
    x = logits.float().cpu().numpy().copy()
    T, V = x.shape
    n = lambda t: None if t is None else t.cpu().numpy()
    tree, tokens, history, history_lengths, prompt_lengths = map(n, (tree, tokens, history, history_lengths, prompt_lengths))
    repetition, frequency, presence, bias_ids, bias, allowed = map(n, (repetition, frequency, presence, bias_ids, bias, allowed))
    best = np.full(T, -1, np.int32)
    f = np.float32
    with np.errstate(all="ignore"):
        for s in range(len(starts) - 1):
            a, e = int(starts[s]), int(starts[s + 1])
            base, seen = np.zeros(V, np.int64), np.zeros(V, bool)
            if history is not None:
                m = min(max(int(history_lengths[s]), 0), history.shape[1])
                p = 0 if prompt_lengths is None else int(prompt_lengths[s])
                for i in range(m):
                    t = int(history[s, i])
                    if 0 <= t < V:
                        seen[t] = True
                        if i >= p:
                            base[t] += 1
            for row in range(a, e):
                c = base.copy()
                if tokens is not None:
                    if tree is None:
                        path = range(a, row + 1)
                    else:
                        path = [a + j for j in range(64) if int(tree[row]) % (1 << 64) >> j & 1 and a + j < e]
                    for j in path:
                        if 0 <= tokens[j] < V:
                            c[tokens[j]] += 1
                l = x[row]
                hit = seen | (c > 0)
                if repetition is not None:
                    l[hit] = np.where(l[hit] > 0, l[hit] / f(repetition[s]), l[hit] * f(repetition[s]))
                made = c > 0
                if frequency is not None:
                    l[made] = l[made] - f(frequency[s]) * c[made].astype(f)
                if presence is not None:
                    l[made] = l[made] - f(presence[s])
                if bias is not None:
                    last = {int(v): i for i, v in enumerate(bias_ids[s]) if 0 <= v < V}
                    for v, i in last.items():
                        l[v] = l[v] + f(bias[s, i])
                if allowed is not None:
                    w = allowed[row if allowed.shape[0] > 1 else 0].view(np.uint32)
                    l[(w[np.arange(V) >> 5] >> (np.arange(V) & 31).astype(np.uint32)) & 1 == 0] = -np.inf
                live = l > -np.inf  # (not for NaN)
                if live.any():
                    best[row] = int(np.flatnonzero(live & (l == l[live].max()))[0])
    return x, best
