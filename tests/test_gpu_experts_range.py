"""32-bit activations of any size through the experts: the pair's 22 bits hold
relative to each row, not to fp16's range.

Limits (derived).  A row (of x, and of h = silu(gate) * up) is scaled by the power
of two that brings its largest magnitude to [2^14, 2^15) and held as the fp16 hi +
lo pair: an element is off by at most 2^-22 of itself (hi leaves half of 2^-10,
lo half of 2^-10 of that) and, where lo is below fp16's normal range, by 2^-25 of
the scale, 2^-39 of the row's largest.  The rest as for unscaled activations: a dot product
of n terms in 32 bits is within (n + 2) 2^-24 of its magnitude sum; silu has a slope
of at most 1.1, its evaluation costs 8 * 2^-24 and, through exp, 3 |a| 2^-24 of the
part of it that exp makes, 1 - sigmoid(a); the sum over k and the weights (k + 1) 2^-24.
No term is absolute.  Errors are random, so the 2-norm of the whole is below
2^-20 of the result's, four times one rounding of 2^-22."""

import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


def reference(W, x, ids, w):
    gate, up, down = (t.double() for t in W)
    E, F, D = gate.shape
    k = ids.shape[1]
    xd, wd = x.double(), w.double()
    out, bound = torch.zeros_like(xd), torch.zeros_like(xd)
    mm = lambda p, q: torch.mm(p, q.t().contiguous())
    for e in range(E):
        hit = ids == e
        rows = hit.any(1).nonzero()[:, 0]
        if not len(rows):
            continue
        v = xd[rows]
        dv = 2.0 ** -22 * v.abs() + 2.0 ** -39 * v.abs().amax(1, keepdim=True)
        a, b = mm(v, gate[e]), mm(v, up[e])
        da = (D + 2) * EPS * mm(v.abs(), gate[e].abs()) + mm(dv, gate[e].abs())
        db = (D + 2) * EPS * mm(v.abs(), up[e].abs()) + mm(dv, up[e].abs())
        s, rest = a * torch.sigmoid(a), torch.sigmoid(-a)
        h = s * b
        dh = 1.1 * da * b.abs() + s.abs() * db + 1.1 * da * db + (8 + 3 * a.abs() * rest) * EPS * h.abs()
        dh += 2.0 ** -22 * h.abs() + 2.0 ** -39 * h.abs().amax(1, keepdim=True)
        y, ym = mm(h, down[e]), mm(h.abs(), down[e].abs())
        dy = mm(dh, down[e].abs()) + (F + 2) * EPS * ym
        share, mag = (wd * hit)[rows].sum(1, keepdim=True), (wd.abs() * hit)[rows].sum(1, keepdim=True)
        out[rows] += share * y
        bound[rows] += mag * (dy + (k + 1) * EPS * ym)
    return out, bound + EPS * out.abs() + 2.0 ** -149


def check(hvd, W, x, ids, w):
    got = hvd.Experts(*W).forward(x, ids, w).double()
    ref, bound = reference(W, x, ids, w)
    assert got.isfinite().all()
    assert ((got - ref).abs() <= bound).all(), float(((got - ref).abs() / bound).max())
    far = torch.linalg.vector_norm(got - ref, dim=1) / torch.linalg.vector_norm(ref, dim=1).clamp_min(2.0 ** -126)
    assert float(far.max()) <= 2.0 ** -20, float(far.max())
    return got


def make(g, E, D, F, gain=1.0):
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") * gain * s[-1] ** -0.5).half()
    return r(E, F, D), r(E, F, D), r(E, D, F)


def choose(g, T, E, k):
    v, i = torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, dim=1)
    return i.to(torch.int32).contiguous(), torch.softmax(v, 1).contiguous()


# rows: one; the few-row form on one and two row tiles; 64-row tiles; 128-row tiles with
# few and with many rows per expert
FORMS = [(1, 8, 2, 1024, 512), (1, 3, 3, 64, 32), (9, 8, 2, 1024, 512), (16, 4, 4, 192, 96), (24, 8, 2, 1024, 512),
         (33, 64, 4, 256, 704), (64, 32, 2, 512, 1056), (20, 16, 16, 128, 64), (60, 16, 2, 320, 96), (300, 8, 2, 1024, 512)]


@pytest.mark.parametrize("std", [1e10, 1e4, 100.0, 1.0, 0.1, 1e-2, 1e-3, 1e-4, 1e-10])
@pytest.mark.parametrize("T,E,k,D,F", FORMS)
def test_rows_of_any_size(hvd, T, E, k, D, F, std):
    g = torch.Generator("cuda").manual_seed(T)
    W, x = make(g, E, D, F), torch.randn(T, D, generator=g, device="cuda") * std
    check(hvd, W, x, *choose(g, T, E, k))


@pytest.mark.parametrize("gain", [1e-3, 0.05, 30.0])
@pytest.mark.parametrize("T,E,k,D,F", FORMS)
def test_weights_of_any_size(hvd, T, E, k, D, F, gain):
    g = torch.Generator("cuda").manual_seed(T + 1)
    W, x = make(g, E, D, F, gain), torch.randn(T, D, generator=g, device="cuda")
    check(hvd, W, x, *choose(g, T, E, k))


@pytest.mark.parametrize("T,E,k,D,F", FORMS)
def test_every_row_has_a_size_of_its_own(hvd, T, E, k, D, F):
    """Rows of sizes from 1e-12 to 1e12 side by side, a zero row, and elements that
    differ as much within a row."""
    g = torch.Generator("cuda").manual_seed(T + 2)
    W, x = make(g, E, D, F), torch.randn(T, D, generator=g, device="cuda")
    x *= 10.0 ** torch.randint(-12, 13, (T, 1), generator=g, device="cuda")
    x[T // 2, ::2] *= 1e-9
    if T > 4:
        x[3] = 0.0
    got = check(hvd, W, x, *choose(g, T, E, k))
    if T > 4:
        assert (got[3] == 0).all()


@pytest.mark.parametrize("T,E,k,D,F", FORMS)
def test_rows_scale_by_powers_of_two(hvd, T, E, k, D, F):
    """Far below 1 silu(a) is a / 2: x / 2^40 and x / 2^42 give outputs a factor of 16
    apart, to the last bits."""
    g = torch.Generator("cuda").manual_seed(T + 3)
    layer, x = hvd.Experts(*make(g, E, D, F)), torch.randn(T, D, generator=g, device="cuda")
    ids, w = choose(g, T, E, k)
    a, b = (layer.forward(x * 2.0 ** -n, ids, w) for n in (40, 42))
    assert torch.allclose(a, b * 16, rtol=1e-6, atol=2.0 ** -30 * float(a.abs().max()))


@pytest.mark.parametrize("T", [1, 9, 24, 60, 300])
def test_a_padded_tail_and_empty_slots(hvd, T):
    """Slots without an expert, whatever their rows hold, and repeated ids."""
    g = torch.Generator("cuda").manual_seed(T + 4)
    E, k, D, F = 8, 4, 256, 96
    W, x = make(g, E, D, F), torch.randn(T, D, generator=g, device="cuda") * 1e-3
    ids, w = choose(g, T, E, k)
    ids[:, 1] = ids[:, 0]
    ids[T // 2:, 2] = -1
    w = torch.where(ids < 0, torch.zeros_like(w), w)
    got = check(hvd, W, x, ids, w)
    ids[T - 1] = E
    x[T - 1] = math.nan
    again = hvd.Experts(*W).forward(x, ids, w).double()
    assert (again[T - 1] == 0).all() and torch.equal(again[:-1], got[:-1])


@pytest.mark.parametrize("T", [1, 9, 24, 60, 300])
def test_captured_and_replayed(hvd, T):
    """Scales are found anew by every replay."""
    g = torch.Generator("cuda").manual_seed(T + 5)
    E, k, D, F = 8, 2, 256, 96
    layer = hvd.Experts(*make(g, E, D, F))
    ids, w = choose(g, T, E, k)
    xs = [torch.randn(T, D, generator=g, device="cuda") * s for s in (1.0, 1e-3, 1e4)]
    want = [layer.forward(x, ids, w) for x in xs]
    buf = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = layer.forward(buf, ids, w)
    for i in (1, 0, 2, 1, 2, 0):
        buf.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res, want[i])
        assert torch.equal(layer.forward(xs[i], ids, w), want[i])
