"""Products past the range of the type that holds them: infinite in every form of a
call, not NaN in those that hold hi + lo pairs, and only where they are."""

import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# rows: one; the few-row form on one and two row tiles; tiles of few and of many rows per expert
ROWS = [1, 5, 16, 24, 60, 300]


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


def setup(T, dtype, size, E=8, D=128, F=96, column=37):
    """Expert 3's product at `column` is about size^2 (x[:, 0] = 1), with the sign of
    x[:, 1]; the rest is of ordinary size."""
    g = torch.Generator("cuda").manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    wt = torch.float16 if dtype == torch.float32 else dtype
    gate, up, down = r(E, F, D) * D ** -0.5, r(E, F, D) * D ** -0.5, r(E, D, F) * F ** -0.5
    gate[3, column] = up[3, column] = 0.0
    gate[3, column, 0] = up[3, column, 1] = size
    down[:, :, column] = torch.where(down[:, :, column] < 0, -0.5, 0.5)
    x = r(T, D)
    x[:, 0], x[:, 1] = 1.0, torch.where(x[:, 1] < 0, -1.0, 1.0)
    ids = torch.stack([torch.arange(T, device="cuda") % 2 * 3, torch.full((T,), 5, device="cuda")], 1).to(torch.int32).contiguous()
    if T == 1:
        ids[0, 0] = 3
    return [t.to(wt) for t in (gate, up, down)], x.to(dtype), ids, torch.full((T, 2), 0.5, device="cuda")


@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("dtype,size", [(torch.float16, 300.0), (torch.bfloat16, 1e20)])
def test_products_past_the_range(hvd, T, dtype, size):
    W, x, ids, w = setup(T, dtype, size)
    got = hvd.Experts(*W).forward(x, ids, w).float()
    hit = ids[:, 0] == 3
    want = x[:, 1].float()[:, None] * W[2][3, :, 37].float()[None, :].sign() * math.inf
    assert torch.equal(got[hit], want[hit])
    assert got[~hit].isfinite().all()


@pytest.mark.parametrize("T", ROWS)
def test_products_past_the_range_of_32_bits(hvd, T):
    """Scaled pairs: finite past fp16's range, infinite past the 32-bit range."""
    W, x, ids, w = setup(T, torch.float32, 300.0)
    layer = hvd.Experts(*W)
    hit = ids[:, 0] == 3
    assert layer.forward(x, ids, w).isfinite().all()
    calm = layer.forward(x, ids, w)[~hit]
    x[hit, :2] *= 1e18
    got = layer.forward(x, ids, w)
    want = x[:, 1][:, None].sign() * W[2][3, :, 37].float()[None, :].sign() * math.inf
    assert torch.equal(got[hit], want[hit]) and torch.equal(got[~hit], calm)


@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_rows_with_infinities_spoil_no_others(hvd, T, dtype, what):
    W, x, ids, w = setup(T, dtype, 1.0)
    layer = hvd.Experts(*W)
    calm = layer.forward(x, ids, w)
    x[T // 2, 7] = what
    got = layer.forward(x, ids, w)
    keep = torch.arange(T, device="cuda") != T // 2
    assert torch.equal(got[keep], calm[keep]) and not got[T // 2].isfinite().any()
