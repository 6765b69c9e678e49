"""The torch binding of the expert-layer operators on the GPU: calls whose result
would be silently wrong are refused."""

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def hvd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_01019_amd as h
    return h


def weights(E=4, D=128, F=64):
    g = torch.Generator("cuda").manual_seed(3)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).half()
    return r(E, F, D), r(E, F, D), r(E, D, F)


@pytest.mark.parametrize("which", range(3))
def test_packed_weights_keep_their_need_of_a_gradient(hvd, which):
    """Packed without autograd, called with it: the gradient would get lost."""
    W = [torch.nn.Parameter(w) if i == which else w for i, w in enumerate(weights())]
    x, ids, w = torch.ones(3, 128, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, 1, device="cuda")
    with torch.no_grad():
        layer = hvd.Experts(*W)
        want = layer.forward(x, ids, w)
    with pytest.raises(hvd.HvdError, match="gradient"):
        layer.forward(x, ids, w)
    with torch.no_grad():
        assert torch.equal(layer.forward(x, ids, w), want)
    assert torch.equal(hvd.Experts(*(t.detach() for t in W)).forward(x, ids, w), want)


def test_tangents_of_the_experts_arguments(hvd):
    import torch.autograd.forward_ad as fwd
    W = weights()
    x, ids, w = torch.ones(3, 128, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, 1, device="cuda")
    layer = hvd.Experts(*W)
    want = layer.forward(x, ids, w)
    with fwd.dual_level():
        p = lambda t: fwd.make_dual(t, torch.ones_like(t))
        calls = [lambda: layer.forward(p(x), ids, w), lambda: layer.forward(x, ids, p(w)), lambda: layer.forward(x, ids, w, out=p(x))]
        calls += [lambda i=i: hvd.Experts(*(p(t) if i == j else t for j, t in enumerate(W))) for i in range(3)]
        for call in calls:
            with pytest.raises(hvd.HvdError, match="tangent"):
                call()
        assert torch.equal(hvd.Experts(*W).forward(x, ids, w), want)


def test_an_output_that_is_given_counts_as_changed(hvd):
    """A backward pass that saved the output's buffer notices that it was written."""
    layer = hvd.Experts(*weights())
    x, ids, w = torch.ones(3, 128, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, 1, device="cuda")
    for write in (lambda o: layer.forward(x, ids, w, out=o), lambda o: hvd.block_norm(x, x, x_out=o)):
        out, a = torch.zeros(3, 128, device="cuda"), torch.ones(3, 128, device="cuda", requires_grad=True)
        z = (a * out).sum()
        write(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()
