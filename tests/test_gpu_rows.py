"""The operators on a step's rows against plain 64-bit implementations (tolerances
are derived in tests/_rows.py, where these stand)."""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests._rows import Case, adjust_ref, append_ref, attend_ref, check_attend  # noqa: E402

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


# ------------------------------------------------------------------ append_kv

def check_append(hvd, c, dtype=F32, heads=None, rot=None, interleaved=False, positions=None, strided=False, theta=1e4):
    heads = c.H if heads is None else heads
    width = (heads + 2 * c.H) * c.D
    if strided:  # a fused projection's row, at an odd address and stride
        base = c.rnd(c.T * (width + 3) + 1).to(dtype).cuda()
        both = torch.as_strided(base, (c.T, heads + 2 * c.H, c.D), (width + 3, c.D, 1), 1)
        q, k, v = both.split((heads, c.H, c.H), dim=1)
    else:
        q, k, v = (c.rnd(c.T, h, c.D).to(dtype).cuda() for h in (heads, c.H, c.H))
    rot = c.D if rot is None else rot
    freqs = None
    if rot:
        freqs = torch.tensor([theta ** (-2 * j / rot) for j in range(rot // 2)], dtype=torch.float64, device="cuda")
    outs, tols = append_ref(c, k, v, q, freqs, interleaved, positions)
    got_q = hvd.append_kv(c.k_cache, c.v_cache, k, v, c.batch(hvd), q=q, freqs=freqs, interleaved=interleaved,
                          positions=None if positions is None else ints(positions))
    for name, got in (("k", c.k_cache), ("v", c.v_cache), ("q", got_q)):
        off = (got.double().cpu() - outs[name]).abs() - tols[name]
        assert float(off.max()) <= 0, (name, float(off.max()))
    return got_q


@pytest.mark.parametrize("dtype,cache", [(F32, F16), (F32, BF16), (F16, F16), (BF16, BF16), (BF16, F16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(8, 8), (64, 64), (72, 36), (80, 2), (96, 40), (128, 128), (128, 6), (256, 256), (64, 0)])
def test_append_types_and_rotations(hvd, dtype, cache, interleaved, D, rot):
    c = Case([(3, 14), (1, 0), (5, 31)], 2, D, dtype=cache, seed=D + rot, pad=2)
    check_append(hvd, c, dtype, 3, rot, interleaved, strided=D % 16 == 0)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_append_pages_and_layouts(hvd, page, layout):
    check_append(hvd, Case([(1, 0), (33, page - 7), (0, 5), (2, 3 * page)], 3, 64, page, seed=page, layout=layout), heads=6)


@pytest.mark.parametrize("tree", [False, True])
def test_append_many_rows(hvd, tree):
    c = Case([(60, 5), (64, 100), (1, 0)] * 9 + [(0, 3)], 2, 64, seed=4, tree=tree, pad=5)
    check_append(hvd, c, heads=2)


def test_append_far_positions(hvd):
    c = Case([(4, 0), (4, 7)], 1, 128, seed=8)
    check_append(hvd, c, positions=[0, 1, 999_999, 2_000_003, 1 << 30, (1 << 31) - 1, 131071, -5])
    long = Case([(5, 1_000_000)], 1, 64, 64, seed=9, spare=0)
    check_append(hvd, long, theta=5e5)


def test_append_many_sequences(hvd):
    check_append(hvd, Case([(1, s % 19) for s in range(300)], 1, 16, seed=10))
    check_append(hvd, Case([(s % 3, s % 5) for s in range(4096)], 1, 8, seed=11))


def test_append_without_a_place(hvd):
    """Keys on pages that the cache does not have, and past the table, are not
    written; their queries are rotated all the same."""
    c = Case([(20, 5), (40, 20), (3, 0)], 2, 32, seed=12, pad=1)
    c.pages[0, 1] = -1
    c.pages[1, 2] = c.n_pages
    c.pages = np.ascontiguousarray(c.pages[:, :3])
    check_append(hvd, c)
    c.lengths[2] = 1  # less than its rows: keys before the first
    k = c.rnd(c.T, 2, 32).cuda()
    before = c.k_cache.clone()
    hvd.append_kv(c.k_cache, c.v_cache, k, k, c.batch(hvd))
    page = int(c.pages[2, 0])
    assert torch.equal(c.k_cache[page, :, 1:], before[page, :, 1:])
    assert torch.equal(c.k_cache[page, :, 0], k[62].to(F16))


def test_append_writes_nothing_else(hvd):
    c = Case([(7, 12)], 2, 64, seed=13)
    kept = c.k_cache.clone()
    k = c.rnd(7, 2, 64).cuda()
    hvd.append_kv(c.k_cache, c.v_cache, k, k, c.batch(hvd))
    same = (c.k_cache == kept).all(-1).all(1)  # [page, token]
    for j in range(19):
        same[int(c.pages[0, j // 16]), j % 16] ^= j >= 12
    assert bool(same.all())


def test_append_copies_special_values(hvd):
    c = Case([(4, 0)], 1, 16, seed=14)
    k = torch.tensor([math.inf, -math.inf, math.nan, 70000.0], device="cuda").view(4, 1, 1).repeat(1, 1, 16)
    hvd.append_kv(c.k_cache, c.v_cache, k, k, c.batch(hvd))
    got = c.v_cache[int(c.pages[0, 0]), 0, :4, 0].float().cpu().numpy()
    np.testing.assert_array_equal(got, [np.inf, -np.inf, np.nan, np.inf])


# --------------------------------------------------------------------- attend

def check(hvd, c, heads, **kw):
    q = c.rnd(c.T, heads, c.D).to(c.dtype).cuda()
    ref_kw = dict(kw)
    call_kw = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), **call_kw)
    check_attend(c, got, q, **ref_kw)
    return q, got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [8, 64, 72, 96, 128, 200, 256])
@pytest.mark.parametrize("sizes", [[(1, 0)], [(1, 200)], [(40, 3), (1, 70), (0, 9), (13, 0)]])
def test_attend_dims(hvd, dtype, D, sizes):
    check(hvd, Case(sizes, 2, D, dtype=dtype, seed=D, pad=2), 6)


@pytest.mark.parametrize("H,G", [(1, 1), (1, 7), (2, 8), (3, 5), (1, 33), (8, 4)])
@pytest.mark.parametrize("rows", [1, 2, 9, 70])
def test_attend_heads(hvd, H, G, rows):
    check(hvd, Case([(rows, 45), (1, 3)], H, 64, seed=H + G), H * G)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 31, 63, 64, 65, 127, 500])
def test_attend_lengths(hvd, page, ctx):
    check(hvd, Case([(1, ctx), (2, ctx), (3, 0)], 1, 64, page, seed=ctx), 2)
    check(hvd, Case([(66, ctx)], 1, 64, page, seed=ctx), 2)


FEATURES = {
    "cap": dict(cap=3.0), "large cap": dict(cap=1e4), "window": dict(window=37), "window 1": dict(window=1),
    "scale": dict(scale=0.7), "scale 0": dict(scale=0.0), "negative scale": dict(scale=-0.3),
    "slopes": dict(slopes=True), "first": dict(first=True), "prefix": dict(prefix=True),
    "all": dict(cap=20.0, window=90, slopes=True, first=True, prefix=True),
}


@pytest.mark.parametrize("name", FEATURES)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("sizes", [[(1, 130), (1, 0), (2, 64)], [(50, 0), (64, 150), (33, 40)]])
@pytest.mark.parametrize("dtype,D", [(F16, 64), (BF16, 128), (F16, 256)])
def test_attend_features(hvd, name, tree, sizes, dtype, D):
    c = Case(sizes, 2, D, dtype=dtype, seed=len(name) + D, tree=tree, pad=1)
    kw = dict(FEATURES[name])
    rng = np.random.default_rng(3)
    if kw.get("slopes"):
        kw["slopes"] = torch.tensor([0.5, 0.25, 0.0, 1.5])
    if kw.get("first"):  # some rows' documents start behind them: they see nothing
        kw["first"] = torch.tensor(rng.integers(-3, 120, c.T), dtype=torch.int32)
    if kw.get("prefix"):
        kw["prefix"] = torch.tensor([0, 170, 1000], dtype=torch.int32)
    check(hvd, c, 4, **kw)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("G", [1, 4])
def test_attend_long_contexts_are_split(hvd, rows, G):
    check(hvd, Case([(rows, 3000), (1, 11), (2, 700)], 2, 64, 64, seed=rows + G), 2 * G, cap=30.0)


@pytest.mark.parametrize("seqs", [1, 2, 62, 63, 64, 65, 130])
@pytest.mark.parametrize("rows", [1, 40])
def test_attend_splits_of_few_and_many_sequences(hvd, seqs, rows):
    """The lengths of splits are chosen apart for up to 63 sequences and for more."""
    check(hvd, Case([(rows if s % 20 == 0 else 1, (s * 97) % 700 + 200 * (s == 0)) for s in range(seqs)], 1, 64, seed=seqs, pad=2), 3)


@pytest.mark.parametrize("G", [1, 3, 5, 32])
@pytest.mark.parametrize("window", [1, 63, 200, 450])
@pytest.mark.parametrize("prefix", [False, True])
def test_attend_windows_over_prompts(hvd, G, window, prefix):
    """What a tile of a windowed prompt can span, where its rows end between columns."""
    c = Case([(150, 500), (1, 300), (66, 0)], 1, 64, seed=G + window, pad=1)
    check(hvd, c, G, window=window, prefix=torch.tensor([600, 0, 20], dtype=torch.int32) if prefix else None)


@pytest.mark.parametrize("dtype,D", [(F16, 256), (BF16, 256), (F16, 128), (BF16, 64)])
@pytest.mark.parametrize("cap", [0.0, 20.0, 100.0])
def test_attend_tiles_of_many_keys(hvd, dtype, D, cap):
    """Tiles that are not split (as many as the card has places for), over more keys
    than one look at the page table gives.  The tolerance is attend_ref's."""
    n, ctx, G = 2085, 1203, 8
    c = Case([(n, ctx)], 2, D, dtype=dtype, seed=D)
    q = c.rnd(n, 2 * G, D).to(dtype).cuda()
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), cap=cap).double()
    L, u, scale = n + ctx, torch.finfo(dtype).eps / 2, D ** -0.5
    ids = torch.from_numpy(c.pages[0]).long().cuda()
    seen = torch.arange(L, device="cuda")[None, :] <= ctx + torch.arange(n, device="cuda")[:, None]
    for h in range(2 * G):
        K, V = (t[ids, h // G].reshape(-1, D)[:L].double() for t in (c.k_cache, c.v_cache))
        Q = q[:, h].double()
        x = torch.mm(Q, K.t().contiguous()) * scale
        big = torch.mm(Q.abs(), K.abs().t().contiguous()).masked_fill(~seen, 0).amax(1) * scale
        d = (D + 8) * 2.0 ** -23 * big
        if cap:
            x = cap * torch.tanh(x / cap)
            d = d + 8 * 2.0 ** -23 * big.clamp(min=cap)
        d = d + 8 * 2.0 ** -23 * x.masked_fill(~seen, 0).abs().amax(1)
        p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
        o, A = torch.mm(p, V), torch.mm(p, V.abs())
        keys = seen.sum(1)[:, None].double()
        tol = 1.02 * (u * o.abs() + (u + 2 * d[:, None] + keys * 2.0 ** -23) * A + keys * 2.0 ** -32 * V.abs().amax(0))
        over = (got[:, h] - o).abs() - tol
        assert float(over.max()) <= 0, (h, float(over.max()))


@pytest.mark.parametrize("rows,D", [(1, 64), (40, 128), (40, 256)])
@pytest.mark.parametrize("cap", [1e-30, 0.01, 64.0, 65.0])
def test_attend_small_and_usual_caps(hvd, rows, D, cap):
    check(hvd, Case([(rows, 100)], 1, D, seed=rows), 2, cap=cap)


@pytest.mark.parametrize("rows,D", [(1, 64), (40, 128), (40, 256)])
@pytest.mark.parametrize("cap", [1e6, 1e30, 3.4e38])
def test_attend_a_cap_far_above_the_scores_changes_nothing(hvd, rows, D, cap):
    """x (1 - (x / cap)^2 / 3 + ..) is x to 2^-24 where |x| < 2^-11 cap: the tolerance is
    that of no cap."""
    c = Case([(rows, 100)], 1, D, seed=rows + 1)
    q = c.rnd(c.T, 2, D).to(F16).cuda()
    check_attend(c, hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), cap=cap), q)


def test_attend_starts_that_leave_rows_out(hvd):
    """Rows before the first start, and starts that go back, are no sequence's or some
    sequence's: no place that does not exist is read for them, and the other
    rows have their results."""
    c = Case([(4, 900), (30, 50)], 2, 64, seed=41)
    q = c.rnd(c.T, 4, 64).to(F16).cuda()
    want = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd))
    c.starts[0], c.lengths[0] = 2, c.lengths[0]
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd))
    assert torch.equal(got[4:], want[4:])
    c.starts[:] = [0, 30, 3]
    assert hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd)).shape == q.shape


def test_attend_a_long_prompt(hvd):
    check(hvd, Case([(300, 0), (129, 77)], 1, 128, seed=5), 3)


def test_attend_many_sequences(hvd):
    check(hvd, Case([(1, s % 40) for s in range(300)], 1, 64, seed=6), 2)
    check(hvd, Case([(s % 2, s % 3) for s in range(4096)], 1, 8, seed=7), 1)


def test_attend_rows_that_see_nothing_are_zero(hvd):
    c = Case([(3, 20), (70, 5)], 1, 64, seed=8, pad=4)
    first = torch.full((c.T,), 1000, dtype=torch.int32)
    first[1] = 0
    _, got = check(hvd, c, 2, first=first)
    assert not got[0].any() and not got[2:].any() and got[1].any()
    empty = Case([(0, 5), (0, 0)], 1, 64, seed=9, pad=3)
    assert not check(hvd, empty, 1)[1].any()
    none = Case([], 1, 64, seed=10, pad=3)
    assert not check(hvd, none, 1)[1].any()
    c.lengths[:] = 0  # no key at all
    assert not hvd.attend(c.rnd(c.T, 2, 64).to(F16).cuda(), c.k_cache, c.v_cache, c.batch(hvd)).any()


@pytest.mark.parametrize("rows", [2, 60])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D", [64, 128, 200, 256])
def test_attend_hidden_places_do_not_reach_a_row(hvd, rows, dtype, what, D):
    """What lies behind a sequence, before a row's document or after the row may be
    anything; what a row sees reaches it and no other."""
    c = Case([(rows, 90), (rows, 30)], 2, D, dtype=dtype, seed=rows)
    for cache in (c.k_cache, c.v_cache):
        for s, (n, ctx) in enumerate(c.sizes):
            for j in range(n + ctx, c.pages.shape[1] * 16):
                if c.pages[s, j // 16] >= 0:
                    cache[int(c.pages[s, j // 16]), :, j % 16] = what
    first = torch.full((c.T,), 40, dtype=torch.int32)
    first[rows:] = 0
    for cache in (c.k_cache, c.v_cache):  # before the documents of the first sequence
        for j in range(40):
            cache[int(c.pages[0, j // 16]), :, j % 16] = what
    _, got = check(hvd, c, 4, first=first)
    assert bool(torch.isfinite(got).all())
    # the last key's value: only the last row sees it
    j = c.sizes[0][0] + c.sizes[0][1] - 1
    c.v_cache[int(c.pages[0, j // 16]), 1, j % 16, 5] = what
    _, got = check(hvd, c, 4, first=first)
    bad = ~torch.isfinite(got)
    assert bad.any() and bool(bad[rows - 1, 2:, 5].all()) and int(bad.sum()) == 2


def test_attend_infinite_scores(hvd):
    c = Case([(1, 40), (40, 10)], 1, 64, seed=21)
    c.k_cache[int(c.pages[0, 0]), 0, 3] = -math.inf
    q = torch.ones(c.T, 1, 64, dtype=F16, device="cuda")
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd))
    check_attend(c, got, q)
    for j in range(41):
        c.k_cache[int(c.pages[0, j // 16]), 0, j % 16] = -math.inf
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd))
    assert not got[0].any()  # all scores -inf: nothing is seen
    check_attend(c, got, q)


@pytest.mark.parametrize("rows", [3, 50])
@pytest.mark.parametrize("D", [64, 96, 128, 200, 256])
def test_attend_without_pages(hvd, rows, D):
    c = Case([(rows, 100), (rows, 60)], 1, D, seed=22)
    c.pages[0, 2] = -1
    c.pages[0, 5] = c.n_pages
    c.pages[1, 0] = 1 << 30
    check(hvd, c, 3)
    c.pages = np.ascontiguousarray(c.pages[:, :4])  # lengths past the table's end
    check(hvd, c, 3)


@pytest.mark.parametrize("layout", ["head", "token"])
def test_attend_strides(hvd, layout):
    c = Case([(5, 40), (60, 3)], 2, 64, seed=23, layout=layout)
    q = c.rnd(c.T, 10, 64).to(F16).cuda()
    b = c.batch(hvd)
    want = hvd.attend(q[:, 2:6].contiguous(), c.k_cache, c.v_cache, b)
    check_attend(c, want, q[:, 2:6])
    assert torch.equal(hvd.attend(q[:, 2:6], c.k_cache, c.v_cache, b), want)
    odd = torch.as_strided(c.rnd(c.T * 300 + 1).to(F16).cuda(), (c.T, 4, 64), (300, 67, 1), 1)
    odd.copy_(q[:, 2:6])
    assert torch.equal(hvd.attend(odd, c.k_cache, c.v_cache, b), want)
    out = torch.full((c.T, 6, 64), 7.0, dtype=F16, device="cuda")
    assert hvd.attend(q[:, 2:6], c.k_cache, c.v_cache, b, out=out[:, 1:5]).data_ptr() == out[:, 1:5].data_ptr()
    assert torch.equal(out[:, 1:5], want) and bool((out[:, 0] == 7).all()) and bool((out[:, 5] == 7).all())
    assert torch.equal(hvd.attend(q[:, 2:6], c.k_cache, c.v_cache, b, out=q[:, 2:6]), want)


def test_attend_past_32_bit_offsets(hvd):
    """Pages whose elements lie past 2^32 bytes and 2^31 elements of the cache."""
    c = Case([(2, 60), (40, 30)], 1, 64, seed=24)
    n = (1 << 31) // (16 * 64) + 64
    big = [torch.empty(n, 1, 16, 64, dtype=F16, device="cuda") for _ in range(2)]
    for t, old in zip(big, (c.k_cache, c.v_cache)):
        t[n - c.n_pages:] = old
    c.pages = np.where(c.pages >= 0, c.pages + (n - c.n_pages), -1).astype(np.int32)
    k = c.rnd(c.T, 1, 64).cuda()
    q = c.rnd(c.T, 2, 64).to(F16).cuda()
    hvd.append_kv(big[0], big[1], k, k, c.batch(hvd))
    got = hvd.attend(q, big[0], big[1], c.batch(hvd))
    c.pages = np.where(c.pages >= 0, c.pages - (n - c.n_pages), -1).astype(np.int32)
    hvd.append_kv(c.k_cache, c.v_cache, k, k, c.batch(hvd))
    assert torch.equal(c.k_cache, big[0][n - c.n_pages:])
    check_attend(c, got, q)


def test_attend_same_bits_every_time(hvd):
    c = Case([(1, 2500), (9, 800), (1, 3)], 2, 128, seed=25)
    q = c.rnd(c.T, 8, 128).to(F16).cuda()
    b = c.batch(hvd)
    want = hvd.attend(q, c.k_cache, c.v_cache, b)
    for _ in range(5):
        assert torch.equal(hvd.attend(q, c.k_cache, c.v_cache, b), want)


# -------------------------------------------------------------- adjust_logits

def penalties(rng, S, V, hist=50, n_bias=5):
    t = lambda a, d=np.float32: torch.from_numpy(np.asarray(a, d)).cuda()
    return dict(history=t(rng.integers(-2, V + 2, (S, hist)), np.int32), history_lengths=t(rng.integers(0, hist + 5, S), np.int32),
                prompt_lengths=t(rng.integers(0, hist, S), np.int32), repetition=t(rng.uniform(0.7, 1.6, S)),
                frequency=t(rng.uniform(-0.2, 0.8, S)), presence=t(rng.uniform(-0.5, 0.8, S)),
                bias_ids=t(rng.integers(-1, V + 1, (S, n_bias)), np.int32), bias=t(rng.normal(size=(S, n_bias)) * 3))


def same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def check_adjust(hvd, starts, logits, tree=None, **kw):
    b = hvd.RowBatch(ints(starts), tree=tree)
    out, best = hvd.adjust_logits(logits, b, **kw)
    ref, rbest = adjust_ref(starts, logits, tree, **kw)
    assert out.dtype == logits.dtype and best.dtype == torch.int32
    assert same(out.cpu(), torch.from_numpy(ref).to(logits.dtype))
    n = int(starts[-1])
    np.testing.assert_array_equal(best.cpu().numpy()[:n], rbest[:n])
    assert bool((best[n:] == -1).all()) and torch.equal(out[n:], logits[n:])
    none, only = hvd.adjust_logits(logits, b, write=False, **kw)
    assert none is None and torch.equal(only, best)
    return out, best


@pytest.mark.parametrize("V", [1, 7, 8, 33, 2047, 2048, 2049, 8192, 8200, 32003])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows", [(1,), (3, 0, 9)])
def test_adjust_sizes(hvd, V, dtype, rows):
    rng = np.random.default_rng(V + len(rows))
    starts = np.concatenate([[0], np.cumsum(rows)])
    T = int(starts[-1]) + 2
    l = torch.from_numpy(rng.normal(size=(T, V)).astype(np.float32) * 3).cuda().to(dtype)
    toks = torch.from_numpy(rng.integers(0, V, T).astype(np.int32)).cuda()
    allowed = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (T, (V + 31) // 32)).astype(np.int32)).cuda()
    check_adjust(hvd, starts, l, tokens=toks, allowed=allowed, **penalties(rng, len(rows), V))


KEYS = [(), ("repetition",), ("frequency",), ("presence",), ("bias", "bias_ids"), ("allowed",), ("tokens", "frequency"),
        ("history", "history_lengths", "repetition"), ("history", "history_lengths", "prompt_lengths", "presence", "frequency"),
        ("tokens", "history", "history_lengths"), ("tokens", "repetition", "bias", "bias_ids", "allowed")]


@pytest.mark.parametrize("keys", KEYS, ids="-".join)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("rows", [(2, 3), (40, 64, 1, 30)])
def test_adjust_parts(hvd, keys, tree, rows):
    rng = np.random.default_rng(len(keys) * 3 + tree)
    V, starts = 301, np.concatenate([[0], np.cumsum(rows)])
    T = int(starts[-1])
    kw = penalties(rng, len(rows), V)
    kw["tokens"] = torch.from_numpy(rng.integers(0, 40, T).astype(np.int32)).cuda()
    kw["allowed"] = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (1, 10)).astype(np.int32)).cuda()
    masks = None
    if tree:
        c = Case([(n, 0) for n in rows], 1, 8, seed=1, tree=True)
        masks = torch.from_numpy(c.tree).cuda()
    l = torch.from_numpy(rng.normal(size=(T, V)).astype(np.float32)).cuda()
    check_adjust(hvd, starts, l, masks, **{k: kw[k] for k in keys})


def test_adjust_many_rows_of_long_histories(hvd):
    rng = np.random.default_rng(5)
    rows = (64, 1, 0, 33, 50, 17)
    starts = np.concatenate([[0], np.cumsum(rows)])
    T, V = int(starts[-1]) + 1, 20011
    l = torch.from_numpy(rng.normal(size=(T, V)).astype(np.float32)).cuda()
    toks = torch.from_numpy((rng.random(T) ** 3 * V).astype(np.int32)).cuda()
    check_adjust(hvd, starts, l, tokens=toks, **penalties(rng, len(rows), V, 5000, 300))


def test_adjust_ties_masks_and_special_values(hvd):
    V, inf = 100, math.inf
    l = torch.zeros(8, V, device="cuda")
    l[0, 50:] = 1.0
    l[1] = -inf
    l[2] = math.nan
    l[3, 9] = inf
    l[4, 70] = -0.0
    l[4, :70] = -1.0
    l[4, 71:] = 0.0  # both zeros are the largest: the lower one
    l[5, 3] = math.nan
    l[6] = -inf
    l[6, 99] = -3.4e38
    l[7, 5] = 2.0
    allowed = torch.full((8, 4), -1, dtype=torch.int32, device="cuda")
    allowed[7] = 0
    out, best = check_adjust(hvd, [0, 8], l, allowed=allowed)
    assert best.tolist() == [50, -1, -1, 9, 70, 0, 99, -1]
    assert bool((out[7] == -inf).all())


def test_adjust_counts_a_path_once_per_row(hvd):
    l = torch.zeros(4, 10, device="cuda")
    toks, one = ints([3, 3, 3, 5]), torch.ones(1, device="cuda")
    chain, _ = hvd.adjust_logits(l, hvd.RowBatch(ints([0, 4])), tokens=toks, frequency=one)
    assert chain[:, 3].tolist() == [-1, -2, -3, -3] and chain[:, 5].tolist() == [0, 0, 0, -1]
    tree = ints([1, 3, 5, 9], torch.int64)
    t, _ = hvd.adjust_logits(l, hvd.RowBatch(ints([0, 4]), tree=tree), tokens=toks, frequency=one)
    assert t[:, 3].tolist() == [-1, -2, -2, -1] and t[:, 5].tolist() == [0, 0, 0, -1]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_adjust_strides_and_places(hvd, dtype):
    rng = np.random.default_rng(8)
    base = torch.from_numpy(rng.normal(size=6 * 1003 + 1).astype(np.float32)).cuda().to(dtype)
    l = torch.as_strided(base, (6, 1001), (1003, 1), 1)
    kw = penalties(rng, 2, 1001)
    out, best = check_adjust(hvd, [0, 2, 6], l, **kw)
    b = hvd.RowBatch(ints([0, 2, 6]))
    room = torch.full((6, 1100), 5.0, dtype=dtype, device="cuda")
    got, gbest = hvd.adjust_logits(l, b, out=room[:, 7:1008], **kw)
    assert same(got, out) and torch.equal(gbest, best)
    assert bool((room[:, :7] == 5).all()) and bool((room[:, 1008:] == 5).all())
    hvd.adjust_logits(l, b, out=l, **kw)
    assert same(l, out) and float(base[0]) == float(base[0])


# ------------------------------------------------------------------- together

def test_a_step_of_all_three(hvd):
    """Chains and trees appended, attended and adjusted as a decoder would, the
    logits from a plain product in between."""
    for tree in (False, True):
        c = Case([(9, 40), (1, 5), (33, 100)], 2, 64, seed=31, tree=tree)
        V, heads = 500, 8
        k, v, q = (c.rnd(c.T, h, 64).cuda() for h in (2, 2, heads))
        freqs = torch.tensor([1e4 ** (-j / 32) for j in range(32)], dtype=torch.float64, device="cuda")
        outs, _ = append_ref(c, k, v, q, freqs)
        b = c.batch(hvd)
        rq = hvd.append_kv(c.k_cache, c.v_cache, k, v, b, q=q, freqs=freqs)
        o = hvd.attend(rq, c.k_cache, c.v_cache, b, cap=50.0)
        check_attend(c, o, rq, cap=50.0)
        head = c.rnd(heads * 64, V).cuda()
        logits = o.float().reshape(c.T, -1) @ head
        toks = torch.from_numpy(np.random.default_rng(1).integers(0, V, c.T).astype(np.int32)).cuda()
        kw = penalties(np.random.default_rng(2), 3, V)
        out, best = hvd.adjust_logits(logits, b, tokens=toks, **kw)
        ref, rbest = adjust_ref(c.starts, logits, b.tree, tokens=toks, **kw)
        assert same(out.cpu(), torch.from_numpy(ref))
        np.testing.assert_array_equal(best.cpu().numpy(), rbest)


def test_a_captured_step_follows_its_tensors(hvd):
    """One graph for the steps of a growing batch: lengths, pages' contents and
    inputs change between replays, and each replay is the eager result."""
    c = Case([(1, 300), (4, 20), (1, 0)], 2, 64, seed=32, max_pages=32)
    need = 32 * 3
    c.n_pages = need
    c.pages = np.random.default_rng(4).permutation(need).astype(np.int32).reshape(3, 32)
    kc, vc = (torch.zeros(need, 2, 16, 64, dtype=F16, device="cuda").normal_() for _ in range(2))
    b = c.batch(hvd)
    T, V = c.T, 1000
    k, v, q = (torch.empty(T, h, 64, device="cuda") for h in (2, 2, 8))
    l, toks = torch.empty(T, V, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    hist = torch.zeros(3, 400, dtype=torch.int32, device="cuda")
    hlen = b.lengths.clone()
    freqs = torch.tensor([1e4 ** (-j / 32) for j in range(32)], dtype=torch.float64, device="cuda")
    pen = torch.full((3,), 1.3, device="cuda")

    def step():
        rq = hvd.append_kv(kc, vc, k, v, b, q=q, freqs=freqs)
        o = hvd.attend(rq, kc, vc, b)
        return rq, o, *hvd.adjust_logits(l, b, tokens=toks, history=hist, history_lengths=hlen, repetition=pen, frequency=pen)

    def fill(seed):
        g = torch.Generator("cuda").manual_seed(seed)
        for t in (k, v, q, l):
            t.normal_(generator=g)
        hist.random_(0, V, generator=g)
        toks.random_(0, V, generator=g)

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(5):
        fill(i + 1)
        b.lengths += i
        hlen += i
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("D,rows", [(256, 70), (128, 70), (64, 1), (72, 2), (256, 1)])
def test_a_captured_attention_alone(hvd, D, rows):
    c = Case([(rows, 300), (1, 40)], 1, D, seed=D)
    q = c.rnd(c.T, 4, D).to(F16).cuda()
    b = c.batch(hvd)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = hvd.attend(q, c.k_cache, c.v_cache, b)
    for _ in range(3):
        q.copy_(c.rnd(c.T, 4, D).to(F16))
        graph.replay()
        torch.cuda.synchronize()
        check_attend(c, got, q)
        assert torch.equal(got, hvd.attend(q, c.k_cache, c.v_cache, b))


def test_one_batch_for_caches_of_two_page_sizes(hvd):
    """What a call needs depends on how many keys the table can hold."""
    small = Case([(1, 100), (2, 60)], 1, 64, 16, seed=39, max_pages=7)
    large = Case([(1, 100), (2, 60)], 1, 64, 1024, seed=39, max_pages=7, spare=30)
    large.pages, large.lengths = small.pages, np.array([101, 62], np.int32)
    b = small.batch(hvd)
    q = small.rnd(small.T, 2, 64).to(F16).cuda()
    for c in (small, large, small):
        check_attend(c, hvd.attend(q, c.k_cache, c.v_cache, b), q)


def test_two_graphs_at_once(hvd):
    """Each graph has a workspace of its own."""
    c = Case([(1, 2000), (5, 300)], 2, 128, seed=37)
    b = c.batch(hvd)
    qs = [c.rnd(c.T, 8, 128).to(F16).cuda() for _ in range(2)]
    graphs, got = [], []
    for q in qs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(hvd.attend(q, c.k_cache, c.v_cache, b))
    want = [hvd.attend(q, c.k_cache, c.v_cache, b) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_inference_mode(hvd):
    c = Case([(1, 20), (5, 30)], 2, 64, seed=38)
    b = c.batch(hvd)
    with torch.inference_mode():
        k, q = c.rnd(c.T, 2, 64).cuda(), c.rnd(c.T, 4, 64).to(F16).cuda()
        hvd.append_kv(c.k_cache, c.v_cache, k, k, b)
        out = hvd.attend(q, c.k_cache, c.v_cache, b, out=torch.empty_like(q))
        check_attend(c, out, q)
        l = torch.zeros(c.T, 100, device="cuda")
        assert hvd.adjust_logits(l, b, out=l)[1].tolist() == [0] * c.T


def test_streams_other_than_the_tensors(hvd):
    c = Case([(1, 900), (5, 30)], 2, 64, seed=33)
    q = c.rnd(c.T, 8, 64).to(F16).cuda()
    b = c.batch(hvd)
    want = hvd.attend(q, c.k_cache, c.v_cache, b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(hvd.attend(q, c.k_cache, c.v_cache, b))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)


def test_no_rows(hvd):
    c = Case([], 2, 64, seed=34)
    b = c.batch(hvd)
    e = torch.empty(0, 2, 64, dtype=F16, device="cuda")
    assert hvd.append_kv(c.k_cache, c.v_cache, e, e, b, q=e).shape == e.shape
    assert hvd.attend(e, c.k_cache, c.v_cache, b).shape == e.shape
    out, best = hvd.adjust_logits(torch.empty(0, 9, device="cuda"), b)
    assert out.shape == (0, 9) and best.shape == (0,)


def test_gradients_and_tangents_are_refused(hvd):
    c = Case([(2, 3)], 1, 64, seed=35)
    b = c.batch(hvd)
    q = torch.zeros(2, 1, 64, dtype=F16, device="cuda", requires_grad=True)
    l = torch.zeros(2, 9, device="cuda", requires_grad=True)
    for call in (lambda: hvd.attend(q, c.k_cache, c.v_cache, b), lambda: hvd.append_kv(c.k_cache, c.v_cache, q, q, b),
                 lambda: hvd.adjust_logits(l, b)):
        with pytest.raises(hvd.HvdError):
            call()
        with torch.no_grad():
            call()
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level():
        d = fwd.make_dual(q.detach().float(), torch.ones(2, 1, 64, device="cuda"))
        with pytest.raises(hvd.HvdError):
            hvd.append_kv(c.k_cache, c.v_cache, d, d, b)


def test_caches_count_as_written(hvd):
    c = Case([(2, 3)], 1, 64, seed=36)
    k = torch.zeros(2, 1, 64, dtype=F16, device="cuda")
    was = c.k_cache._version, c.v_cache._version
    hvd.append_kv(c.k_cache, c.v_cache, k, k, c.batch(hvd))
    assert c.k_cache._version > was[0] and c.v_cache._version > was[1]


@pytest.mark.parametrize("dim", range(4))
def test_keys_and_values_in_one_buffer(hvd, dim):
    """Keys beside values, page by page, head by head or token by token."""
    c = Case([(3, 40), (60, 3)], 2, 64, seed=61)
    shape = (c.n_pages, 2, 16, 64)
    c.k_cache, c.v_cache = c.rnd(*shape[:dim], 2, *shape[dim:]).to(F16).cuda().unbind(dim)
    check_append(hvd, c, heads=4)
    check(hvd, c, 4)


@pytest.mark.parametrize("dim", range(3))
def test_queries_and_results_in_one_buffer(hvd, dim):
    c = Case([(3, 40), (60, 3)], 2, 64, seed=62, pad=1)
    shape = (c.T, 4, 64)
    both = c.rnd(*shape[:dim], 2, *shape[dim:]).to(F16).cuda()
    q, out = both.unbind(dim)
    b, kept = c.batch(hvd), q.clone()
    hvd.attend(q, c.k_cache, c.v_cache, b, out=out)
    assert torch.equal(q, kept)
    check_attend(c, out, kept)
    moved = torch.empty(c.T + 1, 4, 64, dtype=F16, device="cuda")
    moved[:-1] = kept
    with pytest.raises(hvd.HvdError, match="shares memory"):
        hvd.attend(moved[:-1], c.k_cache, c.v_cache, b, out=moved[1:])
    assert torch.equal(moved[:-1], kept)


def test_logits_and_results_in_one_buffer(hvd):
    both = torch.randn(7, 2, 100, device="cuda")
    l, out = both.unbind(1)
    b, one = hvd.RowBatch(ints([0, 6])), torch.ones(1, device="cuda")
    want, best = hvd.adjust_logits(l, b, tokens=ints([0, 5, 5, 99, 3, 3, 3]), frequency=one)
    assert torch.equal(hvd.adjust_logits(l, b, tokens=ints([0, 5, 5, 99, 3, 3, 3]), frequency=one, out=out)[1], best)
    assert torch.equal(out, want)
    kept = both.clone()
    with pytest.raises(hvd.HvdError, match="shares memory"):
        hvd.adjust_logits(l[1:], hvd.RowBatch(ints([0, 6])), out=l[:-1])
    assert torch.equal(both, kept)


@pytest.mark.parametrize("rows,ctx,heads", [(1, 40, 2), (1, 3000, 2), (9, 40, 2), (70, 300, 6), (40, 2500, 4)])
@pytest.mark.parametrize("D,dtype", [(64, F16), (128, BF16), (256, F16)])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 9, 2.0 ** 17, 2.0 ** 22, 2.0 ** 40, 2.0 ** 110, -2.0 ** 22])
@pytest.mark.parametrize("biased", [False, True])
def test_attend_scores_of_any_size(hvd, rows, ctx, heads, D, dtype, scale, biased):
    """Small whole numbers, so that every score is exact (up to 2^122): its place below the
    row's largest is what counts, however large both are.  Tolerance: half a step of the type for
    a weight and for the result; 2^-12 for two base-2 maxima of up to 2^12 that are rounded
    before they are taken off (half a step of numbers in [2^11, 2^12) is 2^-13; larger ones
    are taken off exactly); 2^-23 for each of the sums' operations; and three
    roundings of an exponent of up to 2^7 (smaller weights are nothing)."""
    c = Case([(rows, ctx)], 2, D, dtype=dtype, seed=rows + D)
    c.k_cache.copy_(torch.randint(-8, 9, c.k_cache.shape, generator=c.g))
    q = torch.randint(-8, 9, (rows, heads, D), generator=c.g).to(dtype).cuda()
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), scale=scale,
                     slopes=torch.zeros(heads, device="cuda") if biased else None).double()
    L, u = rows + ctx, torch.finfo(dtype).eps / 2
    ids = torch.from_numpy(c.pages[0]).long().cuda()
    seen = torch.arange(L, device="cuda")[None, :] <= ctx + torch.arange(rows, device="cuda")[:, None]
    for h in range(heads):
        K, V = (t[ids, h * 2 // heads].reshape(-1, D)[:L].double() for t in (c.k_cache, c.v_cache))
        x = torch.mm(q[:, h].double(), K.t().contiguous()) * scale
        p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
        o, A = torch.mm(p, V), torch.mm(p, V.abs())
        d = 2.0 ** -12 + 3 * 2.0 ** -24 * 2 ** 7 + L * 2.0 ** -23
        tol = 1.02 * (u * o.abs() + (u + 2 * d) * A + L * 2.0 ** -32 * V.abs().amax(0))
        over = (got[:, h] - o).abs() - tol
        assert bool((over <= 0).all()), (h, float(over.max()))
@pytest.mark.parametrize("rows,D", [(1, 64), (40, 128), (40, 256)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_attend_the_largest_scale(hvd, rows, D, sign, cap):
    """Queries of 2^-14 in one place and keys up to 2^-22 leave scores of up to 2^91 at
    a scale of 2^127: one-hot weights, or a cap reached, by both forms."""
    c = Case([(rows, 100)], 1, D, dtype=BF16, seed=rows)
    c.k_cache.mul_(2.0 ** -24)
    q = torch.zeros(c.T, 2, D, dtype=BF16, device="cuda")
    q[..., 3] = 2.0 ** -14
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), scale=sign * 2.0 ** 127, cap=cap)
    assert bool(torch.isfinite(got).all())
    ids = torch.from_numpy(c.pages[0]).long().cuda()
    K, V = (t[ids, 0].reshape(-1, D).double() for t in (c.k_cache, c.v_cache))
    for r in range(rows):
        n = 100 + r + 1
        x = sign * K[:n, 3] * 2.0 ** 113
        p = torch.softmax(cap * torch.tanh(x / cap) if cap else x, 0)
        o, A = p @ V[:n], p @ V[:n].abs()
        # a score is one product, exact; half a step for a weight and for the result, the cap's 8 roundings
        tol = 1.02 * (2.0 ** -8 * (o.abs() + A) + (2 * 8 * 2.0 ** -23 * cap + n * 2.0 ** -22) * A)
        assert bool(((got[r].double() - o).abs() <= tol).all())
    for bad in (1.8e38, -2.4e38, math.inf, math.nan):
        with pytest.raises(hvd.HvdError, match="scale"):
            hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), scale=bad)


def test_attend_a_cap_that_32_bits_do_not_hold(hvd):
    """Rounded to 0 it would be none; the least that there is makes all weights equal."""
    c = Case([(2, 20)], 1, 64, seed=63)
    q = c.rnd(c.T, 2, 64).to(F16).cuda()
    b = c.batch(hvd)
    for cap in (1e-46, 1e-300, -1e-46):
        with pytest.raises(hvd.HvdError, match="cap"):
            hvd.attend(q, c.k_cache, c.v_cache, b, cap=cap)
    for cap in (2.0 ** -149, 1e-40, 2.0 ** -126):
        check_attend(c, hvd.attend(q, c.k_cache, c.v_cache, b, cap=cap), q, cap=cap)


@pytest.mark.parametrize("rows", [3, 60])
@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 8])
def test_attend_a_window_wider_than_any_distance(hvd, rows, window):
    """Hides nothing, from rows before the first key either (a length less than the rows),
    which see a prefix."""
    c = Case([(rows, 40), (rows, 0)], 1, 64, seed=64)
    q = c.rnd(c.T, 2, 64).to(F16).cuda()
    check_attend(c, hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), window=window), q)
    c.lengths[:] = [2, 1]
    prefix = ints([2, 1])
    want = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), prefix=prefix)
    assert want.any(-1).all()
    assert torch.equal(hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), prefix=prefix, window=window), want)


# ------------------------------------------------- many keys, by whole matrices

def check_long(c, got, q, cap=0.0, first=None):
    """attend_ref for chains over many keys, by matrices of 64 bits, with its tolerance
    (cap as in test_attend_tiles_of_many_keys).  A weight of a value that is not finite
    counts as one wherever it is not 0; a score that is a NaN makes its row one."""
    g, u, scale = got.double(), torch.finfo(q.dtype).eps / 2, c.D ** -0.5
    ids = torch.from_numpy(c.pages).long().cuda()
    for s, (n, ctx) in enumerate(c.sizes):
        if n == 0:
            continue
        L, a = n + ctx, int(c.starts[s])
        j = torch.arange(L, device="cuda")
        page = ids[s][j // c.page]
        there = (page >= 0) & (page < c.n_pages)
        at = torch.where(there, page, 0)
        seen = (j[None, :] <= ctx + torch.arange(n, device="cuda")[:, None]) & there
        if first is not None:
            seen &= j[None, :] >= first[a:a + n, None]
        for h in range(q.shape[1]):
            K, V = (t[at, h * c.H // q.shape[1], j % c.page].double() for t in (c.k_cache, c.v_cache))
            Q = q[a:a + n, h].double()
            x = (torch.mm(Q, K.t().contiguous()) * scale).masked_fill(~seen, 0)
            big = (torch.mm(Q.abs(), K.abs().t().contiguous()) * scale).masked_fill(~seen, 0).nan_to_num(0).amax(1)
            nan_row = x.isnan().any(1, keepdim=True)
            d = (c.D + 8) * 2.0 ** -23 * big
            if cap:
                x = cap * torch.tanh(x / cap)
                d = d + 8 * 2.0 ** -23 * big.clamp(min=cap)
            x = x.nan_to_num(0)
            d = d + 8 * 2.0 ** -23 * x.abs().amax(1)
            p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
            plain = torch.where(V.isfinite(), V, 0.0)
            o, A = torch.mm(p, plain), torch.mm(p, plain.abs())
            up, down, bad = (torch.mm((p > 0).double(), w.double()) > 0 for w in (V == math.inf, V == -math.inf, V.isnan()))
            bad = bad | (up & down) | nan_row
            want = torch.where(up, math.inf, torch.where(down, -math.inf, o))
            keys = seen.sum(1)[:, None].double()
            tol = 1.02 * (u * o.abs() + (u + 2 * d[:, None] + keys * 2.0 ** -23) * A + keys * 2.0 ** -32 * plain.abs().amax(0))
            mine = g[a:a + n, h]
            assert torch.equal(mine.isnan(), bad), (s, h)
            fine = ~(up | down | bad)
            assert torch.equal(mine[(up | down) & ~bad], want[(up | down) & ~bad]), (s, h)
            over = ((mine - o).abs() - tol)[fine]
            assert over.numel() == 0 or float(over.max()) <= 0, (s, h, float(over.max()))


@pytest.mark.parametrize("D,dtype,long", [(64, F16, 9000), (128, BF16, 9000), (72, F16, 4700), (256, BF16, 4500), (256, F16, 2200)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_attend_tokens_over_many_keys_in_one_piece(hvd, D, dtype, long, cap):
    """A token each of so many sequences that no keys are split: a wave looks at the page
    table again and again, pages without a place among those it finds there."""
    sizes = [(1, (s * 7) % 50) for s in range(100)]
    sizes[0], sizes[41], sizes[99] = (1, long), (1, long - 333), (1, long // 2 + 77)
    c = Case(sizes, 16, D, dtype=dtype, seed=D)
    for k in (0, 70, 129, 140, 141, 142, 200, 256, 270):
        if k * 16 < long:
            c.pages[0, k] = -1 if k % 2 else c.n_pages + k
    q = c.rnd(c.T, 16, D).to(dtype).cuda()
    check_long(c, hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), cap=cap), q, cap)


@pytest.mark.parametrize("seqs,rows,H,G", [(8, 40, 8, 8), (3, 9, 8, 4), (5, 64, 2, 4), (20, 3, 4, 4), (62, 1, 8, 1), (70, 2, 8, 2)])
def test_attend_splits_of_many_lengths(hvd, seqs, rows, H, G):
    c = Case([(rows, 4000 + 61 * (s % 17) if s % 3 else 900 + s) for s in range(seqs)], H, 64, seed=seqs)
    q = c.rnd(c.T, H * G, 64).to(F16).cuda()
    check_long(c, hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd)), q)


@pytest.mark.parametrize("rows", [1, 5, 60])
@pytest.mark.parametrize("D,dtype", [(64, F16), (128, BF16), (200, F16), (256, BF16)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_attend_what_is_not_finite_in_some_splits(hvd, rows, D, dtype, cap):
    """Infinities and NaNs among 3000 keys, seen and hidden, of which most splits see none."""
    c = Case([(rows, 3000), (rows, 2000)], 2, D, dtype=dtype, seed=rows + D)
    inf, nan = math.inf, math.nan

    def put(t, s, head, key, dim, v):
        t[int(c.pages[s, key // 16]), head, key % 16, dim] = v

    for key in range(64):  # before the first sequence's documents
        put(c.k_cache, 0, 0, key, slice(None), nan)
        put(c.v_cache, 0, 0, key, slice(None), inf if key % 2 else nan)
    put(c.v_cache, 0, 0, 100, 3, inf)
    put(c.v_cache, 0, 0, 2500, 3, -inf)  # both signs, apart: a NaN
    put(c.v_cache, 0, 0, 1500, 4, nan)
    put(c.v_cache, 0, 0, 2900, 5, inf)
    put(c.v_cache, 0, 0, 200, 6, -inf)
    put(c.v_cache, 0, 0, 2800, 6, -inf)
    put(c.v_cache, 0, 0, 3000 + rows - 1, 7, inf)  # the last row's own
    put(c.k_cache, 0, 1, 1000, 0, nan)  # a score: all rows of this head
    put(c.k_cache, 1, 1, 2000 + rows - 1, 0, nan)  # the last row's of this one
    first = torch.full((c.T,), 64, dtype=torch.int32, device="cuda")
    q = c.rnd(c.T, 4, D).to(dtype).cuda()
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), cap=cap, first=first)
    check_long(c, got, q, cap, first)
    assert int(got.isfinite().sum()) == got.numel() - 2 * (4 * rows + 1) - 2 * rows * D - 2 * D


@pytest.mark.parametrize("rows,ctx", [(1, 60), (1, 5000), (60, 30), (150, 2500)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("power", [96, -96])
def test_attend_values_of_any_size(hvd, rows, ctx, D, power):
    """Powers of two scale bfloat16 results exactly, with a bias that has the maximum rise
    from tile to tile."""
    c = Case([(rows, ctx)], 2, D, dtype=BF16, seed=rows + D)
    q, slopes = c.rnd(c.T, 4, D).to(BF16).cuda(), torch.tensor([0.5, 0.25, 0.02, 0.0], device="cuda")
    want = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), slopes=slopes)
    c.v_cache.mul_(2.0 ** power)
    got = hvd.attend(q, c.k_cache, c.v_cache, c.batch(hvd), slopes=slopes)
    assert torch.equal(got.double(), want.double() * 2.0 ** power)


@pytest.mark.parametrize("rows,ctx", [(2, 60), (5, 2500), (60, 30), (60, 2500)])
@pytest.mark.parametrize("D,dtype", [(64, F16), (128, BF16), (200, F16), (256, BF16)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_attend_hidden_places_leave_every_bit(hvd, rows, ctx, D, dtype, cap):
    """Rows have the same bits whatever lies before their documents, on other branches of
    their tree or behind them, and however large the scores of other rows are."""
    c = Case([(rows, ctx), (rows, 40)], 2, D, dtype=dtype, seed=rows + D, tree=rows < 65)
    b = c.batch(hvd)
    first = torch.full((c.T,), 33, dtype=torch.int32, device="cuda")
    q = c.rnd(c.T, 6, D).to(dtype).cuda()
    want = hvd.attend(q, c.k_cache, c.v_cache, b, cap=cap, first=first)
    for cache, what in ((c.v_cache, math.nan), (c.v_cache, -math.inf), (c.k_cache, math.nan), (c.k_cache, math.inf), (c.k_cache, 3e4)):
        for j in range(33):
            cache[int(c.pages[0, j // 16]), :, j % 16] = what
        assert torch.equal(hvd.attend(q, c.k_cache, c.v_cache, b, cap=cap, first=first), want)
    # the last row's own value and key, which no other row sees
    for cache, what in ((c.v_cache, math.inf), (c.k_cache, 3e4), (c.k_cache, math.nan)):
        j = ctx + rows - 1
        cache[int(c.pages[0, j // 16]), :, j % 16] = what
        got = hvd.attend(q, c.k_cache, c.v_cache, b, cap=cap, first=first)
        assert torch.equal(got[:rows - 1], want[:rows - 1]) and torch.equal(got[rows:], want[rows:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [(1, 3), (2, 60)])
def test_adjust_in_place_of_strided_logits_writes_nothing_else(hvd, dtype, rows):
    rng = np.random.default_rng(9)
    T, V = sum(rows) + 2, 9001
    base = torch.from_numpy(rng.normal(size=T * (V + 2) + 3).astype(np.float32)).cuda().to(dtype)
    l = torch.as_strided(base, (T, V), (V + 2, 1), 1)
    kw = penalties(rng, 2, V)
    starts = [0, rows[0], sum(rows)]
    out, best = check_adjust(hvd, starts, l, **kw)
    kept = base.clone()
    again, gbest = hvd.adjust_logits(l, hvd.RowBatch(ints(starts)), out=l, **kw)
    assert again.data_ptr() == l.data_ptr() and torch.equal(gbest, best) and same(l, out)
    torch.as_strided(kept, (T, V), (V + 2, 1), 1).copy_(out)
    assert torch.equal(base, kept)


@pytest.mark.parametrize("starts", [[0, 30, 3], [2, 4, 34], [0, 1000, -5], [-7, 40, 34], [34, 34, 0], [1 << 30, -1 << 30, 9]])
@pytest.mark.parametrize("lengths", [[904, 80], [3, -1], [(1 << 31) - 1, -1 << 31]])
@pytest.mark.parametrize("tree", [False, True])
def test_batches_that_are_none_reach_no_other_memory(hvd, starts, lengths, tree):
    """Starts that go back or leave the rows, and lengths of anything: rows, keys and
    pages that do not exist are neither read nor written."""
    c = Case([(4, 900), (30, 50)], 2, 64, seed=65, tree=tree)
    mine = sorted(set(c.pages[c.pages >= 0].tolist()))
    q, k = c.rnd(c.T, 4, 64).to(F16).cuda(), c.rnd(c.T, 2, 64).cuda()
    c.starts[:], c.lengths[:] = starts, lengths
    b = c.batch(hvd)
    room = torch.full((c.T + 6, 6, 64), 7.0, dtype=F16, device="cuda")
    out = room[3:-3, 1:5]
    hvd.attend(q, c.k_cache, c.v_cache, b, out=out)
    edge = room.clone()
    edge[3:-3, 1:5] = 7
    assert bool((edge == 7).all())
    kept = c.k_cache.clone(), c.v_cache.clone()
    hvd.append_kv(c.k_cache, c.v_cache, k, k, b, q=q.float())
    others = [i for i in range(c.n_pages) if i not in mine]
    for new, old in zip((c.k_cache, c.v_cache), kept):
        assert torch.equal(new[others], old[others])
        # (no more places than rows)
        assert int((new != old).any(-1).any(1).sum()) <= c.T
    wide = torch.full((c.T + 6, 110), 7.0, device="cuda")
    hvd.adjust_logits(torch.randn(c.T, 100, device="cuda"), b, tokens=torch.full((c.T,), 5, dtype=torch.int32, device="cuda"),
                      frequency=torch.ones(2, device="cuda"), out=wide[3:-3, 5:105])
    wide[3:-3, 5:105] = 7
    assert bool((wide == 7).all())


# ------------------------------------------------------------------- the limits

def test_the_longest_sequence(hvd):
    """2^29 keys on 2^19 pages.  Equal scores: every result is a count over a count, both
    exact in 32 bits."""
    n_pages, page = 1 << 19, 1024
    L = n_pages * page
    ids = torch.randperm(n_pages, device="cuda").to(torch.int32)
    kc, vc = (torch.zeros(n_pages, 1, page, 8, dtype=F16, device="cuda") for _ in range(2))
    vc[ids[n_pages // 4 * 3:].long(), ..., 0] = 1.0
    vc[ids[:2].long(), ..., 1] = 1.0
    b = hvd.RowBatch(ints([0, 2]), ints([L]), ids[None])
    new = torch.zeros(2, 1, 8, device="cuda")
    new[:, :, 2] = 1.0
    freqs = torch.tensor([0.25], dtype=torch.float64, device="cuda")
    hvd.append_kv(kc, vc, new, new, b, freqs=freqs)
    at = int(ids[-1])
    assert torch.equal(vc[at, 0, -2:], new[:, 0].to(F16)) and torch.equal(kc[at, 0, -2:], new[:, 0].to(F16))
    assert not kc[at, 0, -3].any() and not kc[:, 0, 0].any()
    q = torch.zeros(2, 2, 8, dtype=F16, device="cuda")
    got = hvd.attend(q, kc, vc, b)
    for row in range(2):
        seen = L - 1 + row
        count = torch.tensor([L // 4 - 2, 2 * page, 1 + row], dtype=torch.float64)
        want = torch.where(count / seen < 2.0 ** -25, 0.0, count / seen).half().cuda()
        assert torch.equal(got[row, :, :3], want.expand(2, 3)), (got[row, :, :3], want)
    got = hvd.attend(q, kc, vc, b, window=7)
    want = torch.tensor([[6 / 7, 0, 1 / 7], [5 / 7, 0, 2 / 7]], dtype=torch.float64).half().cuda()
    assert torch.equal(got[:, 0, :3], want)
    got = hvd.attend(q, kc, vc, b, first=ints([0, L - 3]))
    assert torch.equal(got[1, 0, :3], torch.tensor([1 / 3, 0, 2 / 3], dtype=torch.float64).half().cuda())


def test_the_most_rows(hvd):
    """2^20 rows of 4096 sequences."""
    S, n, D = 4096, 256, 8
    T = S * n
    g = torch.Generator("cuda").manual_seed(1)
    k, v, q = (torch.randn(T, 1, D, generator=g, device="cuda").to(BF16) for _ in range(3))
    kc, vc = (torch.full((S * n // 16, 1, 16, D), 9.0, dtype=BF16, device="cuda") for _ in range(2))
    pages = torch.randperm(S * n // 16, generator=g, device="cuda").to(torch.int32).view(S, n // 16)
    b = hvd.RowBatch(torch.arange(0, T + 1, n, dtype=torch.int32, device="cuda"), torch.full((S,), n, dtype=torch.int32, device="cuda"), pages)
    hvd.append_kv(kc, vc, k, v, b)
    assert torch.equal(kc[pages.flatten().long()].view(T, 1, D), k) and torch.equal(vc[pages.flatten().long()].view(T, 1, D), v)
    got = hvd.attend(q, kc, vc, b).view(S, n, D).double()
    u, seen = 2.0 ** -8, torch.ones(n, n, device="cuda", dtype=torch.bool).tril()
    for s in range(0, S, 512):
        K, V, Q = (t.view(S, n, D)[s:s + 512].double() for t in (k, v, q))
        KT = K.transpose(1, 2).contiguous()
        x = torch.bmm(Q, KT) * D ** -0.5
        big = (torch.bmm(Q.abs(), KT.abs()) * D ** -0.5).masked_fill(~seen, 0).amax(2, keepdim=True)
        d = (D + 8) * 2.0 ** -23 * big + 8 * 2.0 ** -23 * x.masked_fill(~seen, 0).abs().amax(2, keepdim=True)
        p = torch.softmax(x.masked_fill(~seen, -math.inf), 2)
        o, A = torch.bmm(p, V), torch.bmm(p, V.abs())
        tol = 1.02 * (u * o.abs() + (u + 2 * d + n * 2.0 ** -23) * A + n * 2.0 ** -32 * V.abs().amax(1, keepdim=True))
        assert bool(((got[s:s + 512] - o).abs() <= tol).all())
    T, V = 65536, 35
    l = torch.randn(T, V, generator=g, device="cuda")
    toks = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    # a sequence of all rows: each token counts for the rows after it
    out, best = hvd.adjust_logits(l, hvd.RowBatch(ints([0, T])), tokens=toks, frequency=torch.full((1,), 2.0 ** -10, device="cuda"))
    want = l - torch.nn.functional.one_hot(toks.long(), V).cumsum(0).float() * 2.0 ** -10
    assert torch.equal(out, want) and torch.equal(best.long(), want.argmax(1))
