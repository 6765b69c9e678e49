"""The expert-layer operators against plain 64-bit implementations.

Tolerances (derived, not fitted).  u = half a step of a type (bf16 2^-8 / 2,
fp16 2^-11 / 2, fp32 2^-24 / 2 relative, written below as eps / 2).
* route: ids equal; weights are 64-bit values rounded once: u32 relative, twice
  that for the 64-bit functions' own last bits.
* block_norm: each output is rounded once (u of its type); before it a 32-bit
  chain of two sums of squares over dim terms (their relative error is at most
  (terms per thread + tree) 2^-24 and halves in the square root) and fewer than
  16 operations: 32 * 2^-24 of the largest term, |x| + |scale gate v|.
* experts: see ``bound``.
"""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def rnd(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


# ------------------------------------------------------------------- route

def route_ref(logits, k, score="softmax", bias=None, n_groups=1, top_groups=1, renorm=True, scale=1.0):
    """Row by row, from the definition."""
    L = logits.double().cpu().numpy()
    n, E = L.shape
    b = np.zeros(E) if bias is None else bias.double().cpu().numpy()
    ids = np.full((n, k), -1, dtype=np.int32)
    w = np.zeros((n, k))
    for t in range(n):
        live = [e for e in range(E) if L[t, e] > -math.inf]  # (False for NaN)
        l = {e: min(L[t, e], 3.402823466e38) for e in live}
        top = max(l.values(), default=0.0)
        if score == "softmax":
            z = {e: math.exp(l[e] - top) for e in live}
            tot = sum(z.values())
            s = {e: z[e] / tot for e in live}
        else:
            s = {e: 1.0 / (1.0 + math.exp(-l[e])) if l[e] > -700 else 0.0 for e in live}
        c = {e: s[e] + b[e] for e in live}
        S = E // n_groups
        value = {}
        for g in range(n_groups):
            best = sorted((c[e] for e in live if e // S == g), reverse=True)[:2]
            if best:
                value[g] = sum(best)
        keep = sorted(value, key=lambda g: (-value[g], g))[:top_groups]
        pick = sorted((e for e in live if e // S in keep), key=lambda e: (-c[e], e))[:k]
        tot = sum(s[e] for e in pick)
        for j, e in enumerate(pick):
            ids[t, j] = e
            w[t, j] = scale * (s[e] / tot if renorm and tot > 0 else s[e] if not renorm else 0.0)
    return ids, w


def check_route(hvd, logits, k, **kw):
    ids, w = hvd.route(logits, k, **kw)
    rid, rw = route_ref(logits, k, **kw)
    assert ids.dtype == torch.int32 and w.dtype == torch.float32
    np.testing.assert_array_equal(ids.cpu().numpy(), rid)
    got = w.double().cpu().numpy()
    assert np.all(np.abs(got - rw) <= 2.0 ** -23 * np.abs(rw) + 1e-45)
    return ids, w


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (8, 2), (63, 8), (64, 8), (65, 7), (128, 16), (160, 6), (256, 8), (511, 5),
                                 (512, 16)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows", [1, 5])
def test_route_sizes(hvd, E, k, score, rows):
    g = gen(E * 31 + k)
    check_route(hvd, rnd(g, rows, E, std=2.0), k, score=score, bias=rnd(g, E, std=0.1), renorm=rows == 1, scale=2.5)


@pytest.mark.parametrize("E,G,top,k", [(8, 8, 3, 3), (64, 2, 1, 8), (64, 8, 4, 8), (96, 3, 2, 6), (120, 5, 2, 7), (256, 8, 4, 8),
                                       (448, 7, 3, 9), (512, 64, 16, 16), (512, 64, 64, 2), (65, 13, 1, 5)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_groups(hvd, E, G, top, k, score):
    g = gen(E + G)
    check_route(hvd, rnd(g, 9, E, std=1.5), k, score=score, bias=rnd(g, E, std=0.05), n_groups=G, top_groups=top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("stride", [48, 49, 80])
def test_route_types_and_strides(hvd, dtype, stride):
    base = rnd(gen(5), 7 * stride + 3, dtype=dtype)
    check_route(hvd, torch.as_strided(base, (7, 48), (stride, 1), 3), 6)


def test_route_ties_take_the_lower_index(hvd):
    l = torch.zeros(3, 100, device="cuda")
    l[1, 50:] = 1.0
    l[2] = torch.arange(100, device="cuda") % 7
    for G, top in ((1, 1), (4, 2), (10, 3)):
        for score in ("softmax", "sigmoid"):
            check_route(hvd, l, 9, score=score, n_groups=G, top_groups=top)
    # 16-bit logits tie by themselves
    check_route(hvd, rnd(gen(8), 40, 256, dtype=torch.bfloat16), 8)


def test_route_masked_experts(hvd):
    g = gen(77)
    l = rnd(g, 12, 64)
    l[0] = -math.inf                      # nothing left
    l[1, 3:] = -math.inf                  # three left for eight places
    l[2] = math.nan
    l[3, ::2] = math.nan
    l[4, 10] = math.inf
    l[5, 10:20] = math.inf
    l[6] = torch.finfo(torch.float32).min  # the lowest finite value masks nothing
    l[7, 1:] = torch.finfo(torch.float32).min
    l[8, :32] = -math.inf                 # whole groups
    l[9, 1:64:8] = -math.inf
    l[10] = -math.inf
    l[10, 63] = -5.0
    for kw in (dict(), dict(renorm=False), dict(n_groups=8, top_groups=3), dict(bias=rnd(g, 64, std=0.1)),
               dict(n_groups=64, top_groups=8)):
        for score in ("softmax", "sigmoid"):
            ids, w = check_route(hvd, l, 8, score=score, **kw)
            assert (ids[0] == -1).all() and (w[0] == 0).all()


def test_route_sigmoid_that_vanishes(hvd):
    """Scores of 0 in 64 bits: weights 0, not NaN."""
    l = torch.full((2, 16), -1e30, device="cuda")
    ids, w = check_route(hvd, l, 4, score="sigmoid")
    assert (w == 0).all() and ids[0].tolist() == [0, 1, 2, 3]


def test_route_many_rows(hvd):
    l = rnd(gen(3), 3001, 72)
    l[100, 1] = math.nan
    ids, w = hvd.route(l, 4)
    s = torch.softmax(l.double().nan_to_num(-math.inf), 1)
    v, i = torch.sort(s, dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), i[:, :4])
    ref = v[:, :4] / v[:, :4].sum(1, keepdim=True)
    assert ((w.double() - ref).abs() <= 2.0 ** -23 * ref).all()


# ------------------------------------------------------------------- block norm

def norm_ref(x, y, gain, post, gate, scale, eps):
    rms = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    xd = x.double()
    add = torch.zeros_like(xd)
    if y is not None:
        v = y.double()
        if post is not None:
            v = rms(v) * post.double()
        add = scale * (v if gate is None else v * gate.double())
    xn = xd + add
    return xn, (rms(xn) * gain.double() if gain is not None else None), xd.abs() + add.abs()


def check_norm(hvd, x, y, gain=None, post=None, gate=None, scale=1.0, eps=1e-5, h_dtype=None, **kw):
    rx, rh, mag = norm_ref(x, y, gain, post, gate, scale, eps)
    xt = x.dtype
    gx, gh = hvd.block_norm(x, y, gain=gain, post_gain=post, gate=gate, scale=scale, eps=eps, h_dtype=h_dtype, **kw)
    u = lambda t: torch.finfo(t).eps / 2
    tiny = lambda t: torch.finfo(t).smallest_normal * u(t) * 2
    chain = 32 * 2.0 ** -24
    assert gx.dtype == xt
    if y is not None:
        assert ((gx.double() - rx).abs() <= u(xt) * rx.abs() + chain * mag + tiny(xt)).all()
    if gain is not None:
        ht = h_dtype or xt
        assert gh.dtype == ht
        ir = 1.0 / torch.sqrt((rx * rx).mean(1, keepdim=True) + eps)
        top = mag * ir * gain.double().abs()
        assert ((gh.double() - rh).abs() <= u(ht) * rh.abs() + 2 * chain * top + tiny(ht)).all()
    return gx, gh


TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dim", [1, 7, 8, 63, 64, 256, 511, 512, 513, 1024, 1031, 2048, 2056, 4096, 4099, 5120, 6144, 8191,
                                 8192, 8200, 16384])
def test_norm_widths(hvd, dim):
    g = gen(dim)
    x, y = rnd(g, 5, dim, std=3.0), rnd(g, 5, dim)
    check_norm(hvd, x, y, gain=rnd(g, dim), post=rnd(g, dim), gate=rnd(g, 5, dim), scale=0.25)
    check_norm(hvd, x, None, gain=rnd(g, dim))
    check_norm(hvd, x, y)


@pytest.mark.parametrize("dim", [2, 9, 519, 575, 576, 577, 1088, 1089, 2303, 2304, 2305, 4100, 4352, 4353, 6400, 6401, 8448, 8449,
                                 16383])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_leftover_columns(hvd, dim, dtype):
    """Widths around the steps' ends, where columns go one to a lane."""
    g = gen(dim + 1)
    x, y = rnd(g, 6, dim, dtype=dtype, std=2.0), rnd(g, 6, dim, dtype=dtype)
    check_norm(hvd, x, y, gain=rnd(g, dim), post=rnd(g, dim), gate=rnd(g, 6, dim, dtype=dtype), scale=0.5)
    check_norm(hvd, x, y, gain=rnd(g, dim), h_dtype=torch.float16)


@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("yt", TYPES)
@pytest.mark.parametrize("ht", TYPES)
def test_norm_types(hvd, xt, yt, ht):
    g = gen(11)
    x, y = rnd(g, 6, 321, dtype=xt), rnd(g, 6, 321, dtype=yt)
    check_norm(hvd, x, y, gain=rnd(g, 321), post=rnd(g, 321), gate=rnd(g, 6, 1, dtype=ht), h_dtype=ht, scale=-0.5)


@pytest.mark.parametrize("shape", [(1, 1), (9, 1), (1, 640), (640,), (9, 640), (1,)])
def test_norm_gate_broadcasts(hvd, shape):
    g = gen(4)
    check_norm(hvd, rnd(g, 9, 640), rnd(g, 9, 640), gain=rnd(g, 640), gate=rnd(g, *shape))


@pytest.mark.parametrize("dim,xs,ys,off", [(40, 41, 47, 1), (4099, 4099, 4100, 3), (128, 129, 128, 5)])
def test_norm_strides_and_alignment(hvd, dim, xs, ys, off):
    g = gen(dim)
    for t in TYPES:
        bx, by = rnd(g, 6 * xs + off, dtype=t), rnd(g, 6 * ys + off, dtype=t)
        before = bx.clone()
        x, y = torch.as_strided(bx, (6, dim), (xs, 1), off), torch.as_strided(by, (6, dim), (ys, 1), off)
        gx, _ = check_norm(hvd, x, y, gain=rnd(g, dim))
        # in place: between the rows nothing changes
        want, _ = hvd.block_norm(x, y, gain=rnd(g, dim), x_out=x)
        assert want.data_ptr() == x.data_ptr() and torch.equal(x, gx)
        torch.as_strided(before, (6, dim), (xs, 1), off).copy_(gx)
        assert torch.equal(bx, before)


def test_norm_of_zero_and_huge_rows(hvd):
    x = torch.zeros(3, 4096, device="cuda")
    x[1] = 1e15
    x[2, 0] = -1e-30
    gx, gh = check_norm(hvd, x, torch.zeros_like(x), gain=torch.ones(4096, device="cuda"), post=torch.ones(4096, device="cuda"))
    assert (gh[0] == 0).all()
    x[1] = math.nan
    _, h = hvd.block_norm(x, None, gain=torch.ones(4096, device="cuda"), h_dtype=torch.bfloat16)
    assert h[1].isnan().all() and not h[0].isnan().any() and not h[2].isnan().any()


def test_norm_many_rows(hvd):
    g = gen(2)
    check_norm(hvd, rnd(g, 70001, 136, dtype=torch.bfloat16), rnd(g, 70001, 136, dtype=torch.bfloat16), gain=rnd(g, 136))


# ------------------------------------------------------------------- experts

def make(g, E, D, F, dtype):
    wt = torch.float16 if dtype == torch.float32 else dtype
    return rnd(g, E, F, D, dtype=wt, std=D ** -0.5), rnd(g, E, F, D, dtype=wt, std=D ** -0.5), rnd(g, E, D, F, dtype=wt, std=F ** -0.5)


def experts_ref(W, x, ids, w):
    """(out, bound): 64-bit result and how far a 32-bit chain may be from it.

    Relative to the sums of magnitudes: a dot product of n terms accumulated in
    32 bits is within (n + 2) 2^-24 of its magnitude sum, plus the operands'
    own rounding (the pair keeps 2^-22 of x; 16-bit operands are exact).  The
    slope of silu is at most 1.1 and |silu(a)| <= |a|; its evaluation in 32 bits costs
    8 * 2^-24.  The product h is rounded to half a step u of its form (2^-22
    for the pair, 2^-25 absolute below fp16's normal range), and the outputs'
    sum over k and the weights cost (k + 1) 2^-24."""
    gate, up, down = (t.double() for t in W)
    E, D, F = gate.shape[0], gate.shape[2], gate.shape[1]
    xd, wd, k = x.double(), w.double(), ids.shape[1]
    out, bound = torch.zeros_like(xd), torch.zeros_like(xd)
    pair = x.dtype == torch.float32
    u = 2.0 ** -22 if pair else torch.finfo(x.dtype).eps / 2
    dx = 2.0 ** -22 if pair else 0.0
    for e in range(E):
        hit = ids == e
        rows = hit.any(1).nonzero()[:, 0]
        if not len(rows):
            continue
        v = xd[rows]
        mm = lambda p, q: torch.mm(p, q.t().contiguous())
        a, b = mm(v, gate[e]), mm(v, up[e])
        am, bm = mm(v.abs(), gate[e].abs()), mm(v.abs(), up[e].abs())
        s = a * torch.sigmoid(a)
        h = s * b
        rel = (D + 2) * 2.0 ** -24 + dx
        dh = 1.1 * rel * am * b.abs() + s.abs() * rel * bm + 1.1 * rel * rel * am * bm + (8 * 2.0 ** -24 + u) * h.abs()
        dh += 0.0 if x.dtype == torch.bfloat16 else 2.0 ** -25
        y, ym = mm(h, down[e]), mm(h.abs(), down[e].abs())
        dy = mm(dh, down[e].abs()) + ((F + 2) * 2.0 ** -24) * ym
        # a repeated id adds up
        share, mag = (wd * hit)[rows].sum(1, keepdim=True), (wd.abs() * hit)[rows].sum(1, keepdim=True)
        out[rows] += share * y
        bound[rows] += mag * (dy + (k + 1) * 2.0 ** -24 * y.abs())
    t = torch.finfo(x.dtype)
    return out, bound + t.eps / 2 * out.abs() + t.smallest_normal * t.eps


def check_experts(hvd, W, x, ids, w, out=None, layer=None):
    layer = layer or hvd.Experts(*W)
    got = layer.forward(x, ids, w, out=out)
    ref, bound = experts_ref(W, x, ids, w)
    assert got.dtype == x.dtype and got.shape == x.shape
    err = (got.double() - ref).abs()
    assert (err <= bound).all(), float((err / bound).max())
    # the bound adds worst cases; errors are random, so the whole comes to about a
    # step of the type (two independent roundings of u / sqrt(3): h and the output)
    norm = float(torch.linalg.vector_norm(got.double() - ref) / torch.linalg.vector_norm(ref).clamp_min(1e-300))
    lim = 2.0 ** -18 if x.dtype == torch.float32 else 1.5 * torch.finfo(x.dtype).eps / 2
    assert norm <= lim, norm
    return got, layer


def choose(g, T, E, k, skew=0.0):
    l = torch.randn(T, E, generator=g, device="cuda") + skew * torch.randn(E, generator=g, device="cuda")
    v, i = torch.topk(l, k, dim=1)
    return i.to(torch.int32).contiguous(), torch.softmax(v, 1).contiguous()


DT = [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [1, 2, 3, 8, 9, 15, 16, 17, 31, 32, 33, 40, 64, 65, 100, 129, 300])
def test_experts_rows(hvd, dtype, T):
    g = gen(T)
    W = make(g, 8, 256, 96, dtype)
    check_experts(hvd, W, rnd(g, T, 256, dtype=dtype), *choose(g, T, 8, 2))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("E,k,D,F", [(1, 1, 64, 32), (2, 2, 64, 32), (3, 1, 128, 64), (5, 3, 192, 160), (16, 16, 320, 32),
                                     (64, 8, 1024, 352), (128, 4, 64, 1024), (512, 8, 64, 32), (7, 2, 4096, 32), (4, 2, 5120, 96)])
@pytest.mark.parametrize("T", [1, 7, 48, 150])
def test_experts_shapes(hvd, dtype, E, k, D, F, T):
    g = gen(E * 7 + T)
    W = make(g, E, D, F, dtype)
    check_experts(hvd, W, rnd(g, T, D, dtype=dtype), *choose(g, T, E, k, 1.0))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [700, 2100])
def test_experts_many_rows(hvd, dtype, T):
    g = gen(T)
    W = make(g, 9, 512, 224, dtype)
    check_experts(hvd, W, rnd(g, T, 512, dtype=dtype), *choose(g, T, 9, 3, 1.5))


@pytest.mark.parametrize("T", [1, 6, 16, 20, 90, 600])
def test_experts_all_rows_on_one(hvd, T):
    g = gen(T)
    W = make(g, 6, 128, 64, torch.bfloat16)
    x = rnd(g, T, 128, dtype=torch.bfloat16)
    ids = torch.full((T, 1), 4, dtype=torch.int32, device="cuda")
    check_experts(hvd, W, x, ids, rnd(g, T, 1))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [1, 5, 16, 24, 64, 500])
def test_experts_empty_slots(hvd, dtype, T):
    """Ids outside the range add nothing, whatever weight (and x) is there;
    rows without an expert come out 0."""
    g = gen(T + 50)
    W = make(g, 6, 128, 64, dtype)
    x = rnd(g, T, 128, dtype=dtype)
    ids, w = choose(g, T, 6, 3)
    ids[T // 2:, 1] = -1
    w[T // 2:, 1] = math.nan
    ids[::3, 2] = 6
    ids[T - 1] = torch.tensor([-1, -(1 << 31), (1 << 31) - 1])
    got, layer = check_experts(hvd, W, x, ids, torch.where((ids >= 0) & (ids < 6), w, torch.zeros_like(w)))
    assert (got[T - 1] == 0).all()
    same = layer.forward(x, ids, w)
    assert torch.equal(same, got)
    x[T - 1] = math.nan  # a row of its own
    again = layer.forward(x, ids, w)
    assert torch.equal(again, got)
    none = layer.forward(x, torch.full_like(ids, -1), w)
    assert (none == 0).all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [1, 4, 16, 30, 200])
def test_experts_same_id_twice(hvd, dtype, T):
    g = gen(T + 9)
    W = make(g, 5, 128, 96, dtype)
    ids, w = choose(g, T, 5, 4)
    ids[:, 2] = ids[:, 0]
    ids[0] = 3
    check_experts(hvd, W, rnd(g, T, 128, dtype=dtype), ids, w)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("E,row", [(2, [1, 0, -1, 1, 5, 0, 1, 1, 0, 0, -7, 1, 0, 1, 2, 0]), (9, [-1, 8, 9, 0, -1, 4]), (1, [0] * 16),
                                   (300, [299, -1, 255, 0, 256, 64, 63, 300])])
def test_experts_one_row_with_empty_and_repeated_slots(hvd, dtype, E, row):
    g = gen(E)
    W = make(g, E, 128, 64, dtype)
    x, ids = rnd(g, 1, 128, dtype=dtype), torch.tensor([row], dtype=torch.int32, device="cuda")
    ok = (ids >= 0) & (ids < E)
    w = rnd(g, 1, len(row)).abs()
    got, layer = check_experts(hvd, W, x, ids, torch.where(ok, w, torch.zeros_like(w)))
    assert torch.equal(layer.forward(x, ids, torch.where(ok, w, torch.full_like(w, math.nan))), got)


@pytest.mark.parametrize("T", [3, 30, 300])
def test_experts_infinite_weights_stay_in_their_rows(hvd, T):
    """An expert with infinities in its matrices spoils only the rows that chose it."""
    g = gen(T)
    W = make(g, 4, 128, 64, torch.bfloat16)
    for t in W:
        t[2, 3] = math.inf
    x = rnd(g, T, 128, dtype=torch.bfloat16)
    ids = torch.arange(T, device="cuda").remainder(4).to(torch.int32)[:, None].contiguous()
    w = torch.ones(T, 1, device="cuda")
    got = hvd.Experts(*W).forward(x, ids, w)
    bad = ids[:, 0] == 2
    assert got[~bad].isfinite().all() and not got[bad].isfinite().all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [1, 11, 60, 400])
def test_experts_strides(hvd, dtype, T):
    """Rows apart by any multiple of 16 bytes; other rows are copied first.
    What lies between and behind the output rows stays as it was."""
    g = gen(T)
    W = make(g, 4, 192, 64, dtype)
    ids, w = choose(g, T, 4, 2)
    big = rnd(g, T + 2, 256, dtype=dtype)
    x = big[1:-1, 8:200]
    outb = torch.full((T + 2, 320), 7.0, dtype=dtype, device="cuda")
    got, layer = check_experts(hvd, W, x, ids, w, out=outb[1:-1, 16:208])
    keep = torch.ones_like(outb, dtype=torch.bool)
    keep[1:-1, 16:208] = False
    assert (outb[keep] == 7.0).all()
    odd = rnd(g, T + 1, 193, dtype=dtype)[:T, 1:]
    check_experts(hvd, W, odd, ids, w, layer=layer)


def test_experts_past_32_bits(hvd):
    """Expert outputs of more than 4 GiB; rows further apart than 2^31 elements."""
    g = gen(2)
    W = make(g, 8, 4096, 32, torch.bfloat16)
    T = 17000
    x = rnd(g, T, 4096, dtype=torch.bfloat16)
    ids = torch.randint(0, 8, (T, 16), generator=g, device="cuda", dtype=torch.int32)
    check_experts(hvd, W, x, ids, rnd(g, T, 16))
    del x
    far = torch.empty(8 * (1 << 29) + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(far, (9, 4096), (1 << 29, 1))
    x.copy_(rnd(g, 9, 4096))
    ids, w = choose(g, 9, 8, 2)
    got, layer = check_experts(hvd, W, x, ids, w)
    y, h = hvd.block_norm(x, got, gain=torch.ones(4096, device="cuda"))
    y2, h2 = hvd.block_norm(x.contiguous(), got, gain=torch.ones(4096, device="cuda"))
    assert torch.equal(y, y2) and torch.equal(h, h2)
    a, b = hvd.route(x[:, :64], 8), hvd.route(x[:, :64].contiguous(), 8)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_experts_many_small_rows(hvd):
    g = gen(6)
    W = make(g, 24, 64, 32, torch.float16)
    check_experts(hvd, W, rnd(g, 60001, 64, dtype=torch.float16), *choose(g, 60001, 24, 3, 2.0))


def test_experts_are_the_same_bits_again(hvd):
    g = gen(1)
    for dtype in DT:
        layer = hvd.Experts(*make(g, 16, 256, 128, dtype))
        for T in (1, 9, 40, 500):
            x = rnd(g, T, 256, dtype=dtype)
            ids, w = choose(g, T, 16, 4)
            a = layer.forward(x, ids, w)
            for _ in range(3):
                assert torch.equal(layer.forward(x, ids, w), a)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T,E,k,F", [(40, 6, 2, 512), (300, 40, 3, 512), (900, 30, 2, 96)])
def test_experts_shared_tiles_replayed(hvd, dtype, T, E, k, F):
    """Tiles whose K range several workgroups share: right, and the same bits
    from a graph replayed between eager calls."""
    g = gen(T + 3)
    W = make(g, E, 2048, F, dtype)
    xs = [rnd(g, T, 2048, dtype=dtype) for _ in range(2)]
    ids, w = choose(g, T, E, k, 0.5)
    want, layer = check_experts(hvd, W, xs[0], ids, w)
    other = layer.forward(xs[1], ids, w)
    buf = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = layer.forward(buf, ids, w)
    for i in range(5):
        buf.copy_(xs[i % 2])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, (want, other)[i % 2])
        assert torch.equal(layer.forward(xs[1 - i % 2], ids, w), (other, want)[i % 2])


def test_experts_refusals(hvd):
    g = gen(1)
    W = make(g, 4, 128, 64, torch.bfloat16)
    layer = hvd.Experts(*W)
    x = rnd(g, 3, 128, dtype=torch.bfloat16)
    ids, w = choose(g, 3, 4, 2)
    for bad in (lambda: layer.forward(x.float(), ids, w), lambda: layer.forward(x[:, :64], ids, w),
                lambda: layer.forward(x, ids.long(), w), lambda: layer.forward(x, ids, w.double()),
                lambda: layer.forward(x, ids[:2], w), lambda: layer.forward(x, ids, w[:, :1]),
                lambda: layer.forward(x, ids, w, out=torch.empty(3, 128, device="cuda")),
                lambda: layer.forward(x, ids, w, out=torch.empty(3, 129, dtype=x.dtype, device="cuda")[:, 1:]),
                lambda: layer.forward(x, torch.zeros(3, 17, dtype=torch.int32, device="cuda"), torch.zeros(3, 17, device="cuda")),
                lambda: layer.forward(x.cpu(), ids, w), lambda: hvd.Experts(W[0], W[1][:2], W[2]),
                lambda: hvd.Experts(W[0].half(), W[1], W[2]), lambda: hvd.Experts(*(t.float() for t in W)),
                lambda: layer.forward(x.clone().requires_grad_(), ids, w), lambda: hvd.route(rnd(g, 3, 8).requires_grad_(), 2),
                lambda: hvd.block_norm(rnd(g, 3, 8), rnd(g, 3, 8).requires_grad_()),
                lambda: hvd.route(rnd(g, 3, 8), 9), lambda: hvd.route(rnd(g, 3, 8), 2, bias=rnd(g, 7)),
                lambda: hvd.block_norm(rnd(g, 3, 8), rnd(g, 3, 7)), lambda: hvd.block_norm(rnd(g, 3, 8).t()),
                lambda: hvd.block_norm(rnd(g, 3, 8), rnd(g, 3, 8), gate=rnd(g, 2, 8))):
        with pytest.raises(hvd.HvdError):
            bad()
    with torch.no_grad():
        assert torch.equal(layer.forward(x.clone().requires_grad_(), ids, w), layer.forward(x, ids, w))
    assert layer.forward(x[:0], ids[:0], w[:0]).shape == (0, 128)
    assert hvd.route(rnd(g, 3, 8)[:0], 2)[0].shape == (0, 2)
    layer.close()
    with pytest.raises(hvd.HvdError):
        layer.forward(x, ids, w)


# ------------------------------------------------------------------- together

def test_gradients_are_refused_for_every_argument(hvd):
    """No backward pass: a gradient that would get lost is an error, whichever
    argument asks for it; without autograd the same calls run."""
    g = gen(3)
    x, y, gate, gain = rnd(g, 3, 128), rnd(g, 3, 128), rnd(g, 3, 128), rnd(g, 128)
    W = make(g, 4, 128, 64, torch.float16)
    layer = hvd.Experts(*W)
    ids, w = choose(g, 3, 4, 2)
    logits, bias = rnd(g, 3, 8), rnd(g, 8)
    p = lambda t: t.clone().requires_grad_()
    calls = [lambda: hvd.block_norm(p(x), gain=gain), lambda: hvd.block_norm(x, p(y), gain=gain),
             lambda: hvd.block_norm(x, gain=p(gain)), lambda: hvd.block_norm(x, y, post_gain=p(gain)),
             lambda: hvd.block_norm(x, y, gate=p(gate)), lambda: hvd.block_norm(x, y, gate=p(gate[:1, :1])),
             lambda: hvd.route(p(logits), 2), lambda: hvd.route(logits, 2, bias=p(bias)),
             lambda: layer.forward(p(x), ids, w), lambda: layer.forward(x, ids, p(w))]
    calls += [lambda i=i: hvd.Experts(*(p(t) if i == j else t for j, t in enumerate(W))) for i in range(3)]
    for i, call in enumerate(calls):
        with pytest.raises(hvd.HvdError, match="gradient"):
            call()
        with torch.no_grad():
            call()


def block(hvd, layer, x, gain, k):
    """The MLP block of an expert layer on a 32-bit residual stream."""
    _, h = hvd.block_norm(x, None, gain=gain)
    ids, w = hvd.route(h[:, :16], k)  # (logits of any kind)
    return hvd.block_norm(x, layer.forward(h, ids, w), gain=gain)


@pytest.mark.parametrize("T", [1, 9, 40, 200])
def test_a_block_eager_captured_and_on_another_stream(hvd, T):
    """The three operators as a layer uses them: the same bits eagerly, on
    another stream, and from two graphs replayed in turn over new inputs."""
    g = gen(T)
    layer = hvd.Experts(*make(g, 16, 256, 96, torch.float32))
    gain = rnd(g, 256)
    xs = [rnd(g, T, 256) for _ in range(4)]
    eager = [block(hvd, layer, x, gain, 4) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x, (a, b) in zip(xs, eager):
            p, q = block(hvd, layer, x, gain, 4)
            side.synchronize()
            assert torch.equal(p, a) and torch.equal(q, b)
    graphs = []
    for _ in range(2):
        buf = torch.zeros(T, 256, device="cuda")
        with torch.cuda.stream(side):
            block(hvd, layer, buf, gain, 4)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            res = block(hvd, layer, buf, gain, 4)
        graphs.append((gr, buf, res))
    for i in range(6):
        x, (a, b) = xs[i % 4], eager[i % 4]
        y, (c, d) = xs[(i + 1) % 4], eager[(i + 1) % 4]
        graphs[0][1].copy_(x)
        graphs[1][1].copy_(y)
        graphs[0][0].replay()
        graphs[1][0].replay()
        torch.cuda.synchronize()
        assert torch.equal(graphs[0][2][0], a) and torch.equal(graphs[0][2][1], b)
        assert torch.equal(graphs[1][2][0], c) and torch.equal(graphs[1][2][1], d)
        assert torch.equal(block(hvd, layer, x, gain, 4)[1], b)  # eager between the replays
