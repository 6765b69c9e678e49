"""What the operators of an expert layer are measured on, through the calls a
user makes of them: routing (``route``), the chosen experts' products
(``Experts.forward``) and the norms around a block with its gate and residual
scale (``block_norm``).

The row counts are the verify step's own: one greedy token, a chain of 8 drafts
(9 rows), a token tree (33), a serving batch of drafts (848), a prefill chunk
(2048); the widths are those of workloads/configs.py (256, 4096, 5120) and
generic ones.  With ``own`` false a pass is the operator's plain form in
elementary torch operations, 32 bits (routing scores in 64: two experts next to
each other have to come out in the same order everywhere).
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
MAX_EXPERT_FLOPS = 6.0 * 2048 * 8 * 4096 * 1024  # of the largest listed case
MAX_EXPERT_PARAMS = 3 * 64 * 4096 * 1024


# ------------------------------------------------------------------- the cases

def _route(rows, experts, k, score="softmax", groups=1, top_groups=1, renorm=True, bias=False, scale=1.0,
           dtype="f32", masked=0):
    return {"op": "route", "rows": rows, "experts": experts, "k": k, "score": score, "groups": groups,
            "top_groups": top_groups, "renorm": renorm, "bias": bias, "scale": scale, "dtype": dtype, "masked": masked}


def _experts(rows, experts, k, dim, ffn, dtype="bf16", pad=0, skew=0.7):
    return {"op": "experts", "rows": rows, "experts": experts, "k": k, "dim": dim, "ffn": ffn, "dtype": dtype,
            "pad": pad, "skew": skew}


def _norm(rows, dim, x="f32", h="f32", y="f32", post=False, gate="none", scale=1.0):
    return {"op": "norm", "rows": rows, "dim": dim, "x": x, "y": y, "h": h, "post": post, "gate": gate, "scale": scale}


def listed():
    return [
        # a greedy token: latency alone
        {"name": "route 1x64", **_route(1, 64, 8)},
        # a serving batch of drafts; sigmoid scores with a balance bias, experts in groups
        {"name": "route 848x256 groups", **_route(848, 256, 8, "sigmoid", 8, 4, bias=True, scale=2.5)},
        # a long prefill in 16 bits, an odd number of experts of which some are switched off
        {"name": "route 8191x120 bf16", **_route(8191, 120, 6, dtype="bf16", renorm=False, masked=5)},
        # a greedy token through the experts it chose: their weights are all there is to read
        {"name": "experts 1 row", **_experts(1, 64, 8, 4096, 1024)},
        # a chain of 8 drafts, 32-bit activations (the verify step's numerics)
        {"name": "experts 9 rows f32", **_experts(9, 64, 8, 4096, 1024, "f32")},
        # the smallest decoder's width with a padded tail: latency
        {"name": "experts 5 rows small", **_experts(5, 16, 2, 256, 352, "f16", pad=2)},
        # a token tree: nearly every expert is touched by a few rows
        {"name": "experts 33 rows", **_experts(33, 128, 4, 5120, 704, "f16")},
        # a serving batch of drafts, some rows of it padding
        {"name": "experts 848 rows", **_experts(848, 64, 8, 4096, 1024, "bf16", pad=11)},
        # a prefill chunk: bound by the matrix cores
        {"name": "experts 2048 rows", **_experts(2048, 64, 8, 4096, 1024, "f16")},
        # the step between two blocks of a greedy token
        {"name": "norm 1x4096", **_norm(1, 4096)},
        # a serving batch, norms on both sides, a gate per row
        {"name": "norm 848x5120 post", **_norm(848, 5120, y="bf16", h="f16", post=True, gate="row", scale=0.25)},
        # a long prefill with 16-bit streams, an odd width and a gate per element
        {"name": "norm 16383x4099 bf16", **_norm(16383, 4099, x="bf16", y="bf16", h="bf16", gate="full")},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("route", "experts", "experts", "experts", "norm"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * max(1, _log_int(rng, 8, 512) // groups)
        top_groups = rng.randint(1, groups)
        k = min(_log_int(rng, 1, 16), E // groups * top_groups)
        return _route(min(_log_int(rng, 1, 8192), 8192 * 120 // E), E, k, rng.choice(("softmax", "sigmoid")), groups,
                      top_groups, rng.random() < 0.6, rng.random() < 0.5, rng.choice((1.0, 2.5)),
                      rng.choice(("f32", "f32", "bf16", "f16")), rng.choice((0, 0, E // 16)))
    if op == "norm":
        dim = _log_int(rng, 64, 8192)
        if rng.random() < 0.7:  # mostly whole vectors, sometimes any width
            dim = (dim + 63) // 64 * 64
        t = rng.choice(("f32", "f32", "bf16", "f16"))
        o = t if t != "f32" else rng.choice(("f32", "bf16", "f16"))
        return _norm(min(_log_int(rng, 1, 16383), 16383 * 4099 // dim), dim, t, o, rng.choice(("f32", o)),
                     rng.random() < 0.5, rng.choice(("none", "none", "row", "full")), rng.choice((1.0, 0.22)))
    while True:
        rows = _log_int(rng, 1, 2048)
        E = _log_int(rng, 4, 128)
        k = min(E, rng.choice((1, 2, 4, 6, 8)))
        dim = rng.choice((256, 1024, 2048, 4096, 5120))
        ffn = 32 * _log_int(rng, 3, 64)
        if 6.0 * rows * k * dim * ffn <= MAX_EXPERT_FLOPS and 3 * E * dim * ffn <= MAX_EXPERT_PARAMS:
            pad = rng.randrange(1, max(2, rows // 3)) if rows > 1 and rng.random() < 0.3 else 0
            return _experts(rows, E, k, dim, ffn, rng.choice(("bf16", "bf16", "f16", "f32")), pad, rng.choice((0.0, 0.7, 1.5)))


# ------------------------------------------------------------------- the inputs

def _data(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32)
    if case["op"] == "route":
        E = case["experts"]
        l = 1.5 * rnd(case["rows"], E) + 0.7 * rnd(E)
        if case["masked"]:  # experts that are switched off
            l[:, torch.randperm(E, generator=g, device="cuda")[: case["masked"]]] = -math.inf
        return {"logits": l.to(DTYPES[case["dtype"]]), "bias": 0.05 * rnd(E) if case["bias"] else None}
    if case["op"] == "norm":
        n, d = case["rows"], case["dim"]
        out = {"x": (3.0 * rnd(n, d)).to(DTYPES[case["x"]]), "y": (0.7 * rnd(n, d)).to(DTYPES[case["y"]]),
               "gain": 1.0 + 0.1 * rnd(d), "post": 1.0 + 0.1 * rnd(d) if case["post"] else None, "gate": None}
        if case["gate"] != "none":
            shape = (n, 1) if case["gate"] == "row" else (n, d)
            out["gate"] = torch.sigmoid(rnd(*shape)).to(DTYPES[case["y"]])
        return out
    T, E, k, D, F = case["rows"], case["experts"], case["k"], case["dim"], case["ffn"]
    wt = torch.float16 if case["dtype"] == "f32" else DTYPES[case["dtype"]]

    def mat(o, i):
        w = torch.empty(E, o, i, dtype=wt, device="cuda")
        for e in range(E):
            w[e] = rnd(o, i).mul_(i ** -0.5)
        return w

    l = 1.5 * rnd(T, E) + case["skew"] * rnd(E)
    top, ids = torch.topk(l, k, dim=1)
    w = torch.softmax(top, 1)
    ids = ids.to(torch.int32)
    if case["pad"]:  # empty rows behind the batch
        ids[T - case["pad"]:] = -1
        w[T - case["pad"]:] = 0.0
    return {"x": rnd(T, D).to(DTYPES[case["dtype"]]), "ids": ids.contiguous(), "w": w.contiguous(),
            "gate": mat(F, D), "up": mat(F, D), "down": mat(D, F)}


def prepare(case, seed):
    st = {"case": case, **_data(case, seed)}
    if own and case["op"] == "experts":
        import paper_2606_01019_amd as hvd
        # the layer's weights, laid out once
        st["layer"] = hvd.Experts(st.pop("gate"), st.pop("up"), st.pop("down"))
    return st


# -------------------------------------------------------------------- one pass

def run(st):
    c = st["case"]
    if own:
        import paper_2606_01019_amd as hvd
        if c["op"] == "route":
            ids, w = hvd.route(st["logits"], c["k"], score=c["score"], bias=st["bias"], n_groups=c["groups"],
                               top_groups=c["top_groups"], renorm=c["renorm"], scale=c["scale"])
            return {"ids": ids, "weights": w}
        if c["op"] == "norm":
            x, h = hvd.block_norm(st["x"], st["y"], gain=st["gain"], post_gain=st["post"], gate=st["gate"],
                                  scale=c["scale"], eps=1e-5, h_dtype=DTYPES[c["h"]])
            return {"x": x, "h": h}
        return {"out": st["layer"].forward(st["x"], st["ids"], st["w"])}
    return {"route": _plain_route, "experts": _plain_experts, "norm": _plain_norm}[c["op"]](st)


def _best(c, k):
    """The k largest of each row and their places, the lower place on ties."""
    v, i = torch.sort(c, dim=1, descending=True, stable=True)
    return v[:, :k], i[:, :k]


def _plain_route(st):
    c = st["case"]
    E, G = c["experts"], c["groups"]
    l = st["logits"].to(torch.float64)
    if c["score"] == "softmax":
        p = torch.exp(l - l.max(dim=1, keepdim=True).values)
        s = p / p.sum(dim=1, keepdim=True)
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    choice = s if st["bias"] is None else s + st["bias"].to(torch.float64)
    choice = torch.where(l == -math.inf, torch.full_like(choice, -math.inf), choice)
    if G > 1:
        two = _best(choice.view(-1, E // G), 2)[0]
        rest = torch.where(two[:, 1:] == -math.inf, torch.zeros_like(two[:, 1:]), two[:, 1:])
        keep = _best((two[:, 0] + rest.sum(dim=1)).view(-1, G), c["top_groups"])[1]
        kept = torch.zeros(len(l), G, dtype=torch.bool, device=l.device).scatter_(1, keep, True)
        choice = choice.masked_fill(~kept.repeat_interleave(E // G, dim=1), -math.inf)
    v, ids = _best(choice, c["k"])
    none = v == -math.inf
    w = torch.gather(s, 1, ids).masked_fill(none, 0.0)
    if c["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    return {"ids": ids.to(torch.int32).masked_fill(none, -1), "weights": (w * c["scale"]).to(torch.float32)}


def _plain_experts(st):
    c, x, ids, w = st["case"], st["x"], st["ids"], st["w"]
    E, k = c["experts"], c["k"]
    flat = ids.reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat + 1, minlength=E + 1).tolist()  # the empty slots first
    out = torch.zeros(x.shape, dtype=torch.float32, device=x.device)
    at = counts[0]
    for e in range(E):
        n = counts[e + 1]
        if n == 0:
            continue
        slot = order[at: at + n]
        at += n
        row = slot // k
        v = x[row].float()
        a = v @ st["gate"][e].float().t()
        a = a / (1.0 + torch.exp(-a)) * (v @ st["up"][e].float().t())
        out.index_add_(0, row, (a @ st["down"][e].float().t()) * w.reshape(-1)[slot, None])
    return {"out": out.to(x.dtype)}


def _plain_norm(st):
    c = st["case"]
    rms = lambda v: v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + 1e-5)
    v = st["y"].float()
    if st["post"] is not None:
        v = rms(v) * st["post"]
    if st["gate"] is not None:
        v = v * st["gate"].float()
    x = st["x"].float() + c["scale"] * v
    return {"x": x.to(st["x"].dtype), "h": (rms(x) * st["gain"]).to(DTYPES[c["h"]])}


# ------------------------------------------------------------- what a pass takes

def work(case):
    if case["op"] == "route":
        n, E = case["rows"], case["experts"]
        return {"bytes": n * E * BYTES[case["dtype"]] + n * case["k"] * 8 + (4 * E if case["bias"] else 0),
                "flops": 4 * n * E}
    if case["op"] == "norm":
        n, d = case["rows"], case["dim"]
        gate = {"none": 0, "row": n, "full": n * d}[case["gate"]] * BYTES[case["y"]]
        return {"bytes": n * d * (2 * BYTES[case["x"]] + BYTES[case["y"]] + BYTES[case["h"]]) + gate + 4 * d * (1 + case["post"]),
                "flops": n * d * (6 + 4 * case["post"] + (case["gate"] != "none"))}
    n, E, k = case["rows"] - case["pad"], case["experts"], case["k"]
    params = 3 * case["dim"] * case["ffn"]
    touched = E * (1.0 - (1.0 - k / E) ** n)  # experts that some row chose, evenly spread
    return {"bytes": int(2 * params * touched) + 2 * case["rows"] * case["dim"] * BYTES[case["dtype"]] + 8 * case["rows"] * k,
            "flops": 2 * params * n * k}


# ------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    d = _data(case, seed)
    if case["op"] == "route":
        return _exact_route(case, d)
    if case["op"] == "norm":
        n = {key: (None if t is None else t.double().cpu().numpy()) for key, t in d.items()}
        v = n["y"]
        if n["post"] is not None:
            v = v / np.sqrt(np.mean(v ** 2, axis=1, keepdims=True) + 1e-5) * n["post"]
        x = n["x"] + case["scale"] * (v if n["gate"] is None else n["gate"] * v)
        h = x / np.sqrt(np.mean(x ** 2, axis=1, keepdims=True) + 1e-5) * n["gain"]
        return {"x": torch.from_numpy(x), "h": torch.from_numpy(h)}
    x, ids, w = d["x"].double(), d["ids"], d["w"].double()
    out = torch.zeros_like(x)
    for e in range(case["experts"]):
        share = (w * (ids == e)).sum(1)
        rows = (ids == e).any(1).nonzero()[:, 0]
        if len(rows):
            a = torch.mm(d["gate"][e].double(), x[rows].T.contiguous())
            b = torch.mm(d["up"][e].double(), x[rows].T.contiguous())
            y = torch.mm(d["down"][e].double(), torch.sigmoid(a) * a * b)
            out[rows] += share[rows, None] * y.T
    return {"out": out}


def _exact_route(case, d):
    l = d["logits"].double().cpu().numpy()
    n, E = l.shape
    k, G = case["k"], case["groups"]
    with np.errstate(over="ignore"):
        if case["score"] == "softmax":
            s = np.exp(l - l.max(1, keepdims=True))
            s /= s.sum(1, keepdims=True)
        else:
            s = 1 / (1 + np.exp(-l))
    pick = s + (0.0 if d["bias"] is None else d["bias"].double().cpu().numpy())
    pick[np.isneginf(l)] = -np.inf
    if G > 1:
        parts = np.sort(pick.reshape(n, G, -1), axis=2)
        value = parts[:, :, -1].copy()
        if parts.shape[2] > 1:
            value += np.where(np.isneginf(parts[:, :, -2]), 0.0, parts[:, :, -2])
        rank = np.argsort(np.argsort(-value, axis=1, kind="stable"), axis=1)
        pick[np.repeat(rank >= case["top_groups"], E // G, axis=1)] = -np.inf
    ids = np.argsort(-pick, axis=1, kind="stable")[:, :k]
    w = np.take_along_axis(s, ids, 1)
    gone = np.isneginf(np.take_along_axis(pick, ids, 1))
    w[gone] = 0.0
    if case["renorm"]:
        w = w / w.sum(1, keepdims=True)
    return {"ids": torch.from_numpy(np.where(gone, -1, ids).astype(np.int32)), "weights": torch.from_numpy(w * case["scale"])}
