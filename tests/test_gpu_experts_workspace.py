"""hvd_experts_workspace: one buffer for the most rows serves every call of fewer,
whatever form a call takes."""

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

CASES = [(64, 8, 256, 96, torch.bfloat16), (8, 2, 64, 2048, torch.bfloat16), (256, 16, 64, 1024, torch.float16),
         (3, 16, 64, 32, torch.float16), (40, 1, 128, 160, torch.float32), (16, 2, 1024, 512, torch.float32)]


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


@pytest.mark.parametrize("E,k,D,F,dtype", CASES)
def test_one_workspace_for_all_row_counts(hvd, E, k, D, F, dtype):
    g = torch.Generator("cuda").manual_seed(E)
    wt = torch.float16 if dtype == torch.float32 else dtype
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    layer = hvd.Experts(*((r(*s) * s[-1] ** -0.5).to(wt) for s in ((E, F, D), (E, F, D), (E, D, F))))
    code = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}[dtype]
    lib, h = layer.lib, layer.handle
    size = lambda T: lib.hvd_experts_workspace(h, T, k, code)
    sizes = [size(T) for T in range(1, 1200)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    pair = 16 * E // k  # about the rows from which the product is one 16-bit value
    N = max(700, pair + 40)
    work = torch.empty(size(N), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    for T in sorted({1, 2, 15, 16, 17, 31, 32, 33, 34, 100, 300, pair - 1, pair, pair + 1, N} - {0, -1}):
        x = r(T, D).to(dtype)
        ids = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
        w = r(T, k).abs()
        out = torch.empty_like(x)
        assert lib.hvd_experts_forward(h, T, k, x.data_ptr(), code, D, ids.data_ptr(), w.data_ptr(), out.data_ptr(), D,
                                       work.data_ptr(), work.numel(), s) == 0, (T, lib.hvd_last_error())
        assert torch.equal(out, layer.forward(x, ids, w)), T
    assert lib.hvd_experts_forward(h, N, k, x.data_ptr(), code, D, ids.data_ptr(), w.data_ptr(), out.data_ptr(), D,
                                   work.data_ptr(), 255, s) != 0  # too small
    assert size(0) > 0 and size(-1) == 0


def test_no_partial_sums_where_no_tile_is_shared(hvd):
    """Calls of few rows per expert: slots, products and outputs, without the 32 MiB
    of partial sums that 128-row tiles share."""
    E, k, D, F = 64, 8, 64, 1024
    layer = hvd.Experts(*(torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((E, F, D), (E, F, D), (E, D, F))))
    for T in (33, 64, 127):
        need = layer.lib.hvd_experts_workspace(layer.handle, T, k, 0)
        few = 2 * E * 16 * F * 2  # (the largest few-row call)
        assert need <= max(few, T * k * (2 * 4 + 2 * F * 2 + D * 4)) + 16384, (T, need)
    assert layer.lib.hvd_experts_workspace(layer.handle, 128, k, 0) > 32 << 20
