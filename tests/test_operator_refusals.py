"""What the expert-layer operators refuse (CPU: every refusal comes from the
host's checks, before anything is enqueued; the addresses are never read)."""

import ctypes

import pytest

import paper_2606_01019_amd as hvd
from paper_2606_01019_amd import operators as ops
from paper_2606_01019_amd.hvd import HVD_ERR_ARG, HVD_OK

A = 1 << 20  # an aligned address nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return hvd.load_library()


def route_cfg(**kw):
    d = dict(n_experts=64, top_k=8, score=0, n_groups=1, top_groups=1, renorm=1, scale=1.0)
    d.update(kw)
    return ops.RouteConfig(*[d[f] for f, _ in ops.RouteConfig._fields_])


@pytest.mark.parametrize("kw", [
    dict(n_experts=0), dict(n_experts=513), dict(top_k=0), dict(top_k=17), dict(n_experts=4), dict(score=2),
    dict(n_groups=0), dict(n_groups=5), dict(n_experts=130, n_groups=65), dict(n_groups=4, top_groups=5),
    dict(n_groups=4, top_groups=0), dict(n_groups=16, top_groups=1), dict(scale=float("nan")),
    dict(scale=float("inf"))])
def test_route_config(lib, kw):
    assert lib.hvd_route(ctypes.byref(route_cfg(**kw)), 1, A, 2, 512, None, A, A, None) == HVD_ERR_ARG
    assert lib.hvd_last_error()


@pytest.mark.parametrize("rows,logits,dtype,stride,bias,ids,w", [
    (-1, A, 2, 64, None, A, A), ((1 << 23) + 1, A, 2, 64, None, A, A), (1, None, 2, 64, None, A, A), (1, A, 3, 64, None, A, A), (1, A, -1, 64, None, A, A),
    (2, A, 2, 63, None, A, A), (1, A + 2, 2, 64, None, A, A), (1, A + 1, 0, 64, None, A, A), (1, A, 2, 64, A + 1, A, A),
    (1, A, 2, 64, None, None, A), (1, A, 2, 64, None, A, None), (1, A, 2, 64, None, A + 2, A)])
def test_route_arguments(lib, rows, logits, dtype, stride, bias, ids, w):
    assert lib.hvd_route(ctypes.byref(route_cfg()), rows, logits, dtype, stride, bias, ids, w, None) == HVD_ERR_ARG


def test_no_rows_is_nothing(lib):
    assert lib.hvd_route(ctypes.byref(route_cfg()), 0, None, 2, 64, None, None, None, None) == HVD_OK
    assert lib.hvd_route(None, 0, None, 2, 64, None, None, None, None) == HVD_ERR_ARG
    assert lib.hvd_block_norm(ctypes.byref(ops.BlockNormArgs()), 0, 8, None) == HVD_OK
    assert lib.hvd_block_norm(None, 0, 8, None) == HVD_ERR_ARG


@pytest.mark.parametrize("E,D,F,dtype", [(0, 64, 32, 0), (513, 64, 32, 0), (4, 0, 32, 0), (4, 96, 32, 0), (4, 64, 0, 0),
                                         (4, 64, 48, 0), (4, 64, 32, 2), (4, 64, 32, 3), (4, 1 << 21, 32, 0)])
def test_experts_config(lib, E, D, F, dtype):
    cfg = ops.ExpertsConfig(E, D, F, dtype)
    h = ctypes.c_void_p()
    assert lib.hvd_experts_bytes(ctypes.byref(cfg)) == 0
    assert lib.hvd_experts_load(ctypes.byref(cfg), A, A, A, A, 1 << 40, None, ctypes.byref(h)) == HVD_ERR_ARG
    assert h.value is None


def test_experts_load_arguments(lib):
    cfg = ops.ExpertsConfig(4, 64, 32, 1)
    n = lib.hvd_experts_bytes(ctypes.byref(cfg))
    assert n == 3 * 4 * 64 * 32 * 2
    h = ctypes.c_void_p()
    for g, u, d, b, m in ((None, A, A, A, n), (A, None, A, A, n), (A, A, None, A, n), (A + 8, A, A, A, n),
                          (A, A, A, A + 8, n), (A, A, A, A, n - 1)):
        assert lib.hvd_experts_load(ctypes.byref(cfg), g, u, d, b, m, None, ctypes.byref(h)) == HVD_ERR_ARG
    assert lib.hvd_experts_load(ctypes.byref(cfg), A, A, A, A, n, None, None) == HVD_ERR_ARG
    lib.hvd_experts_free(None)
    assert lib.hvd_experts_workspace(None, 1, 1, 1) == 0
    assert lib.hvd_experts_forward(None, 1, 1, A, 1, 64, A, A, A, 64, A, 1 << 40, None) == HVD_ERR_ARG


def norm_args(**kw):
    a = ops.BlockNormArgs(x=A, x_stride=64, x_dtype=2, y=A, y_stride=64, y_dtype=1, x_out=A, x_out_stride=64, gain=A,
                          h=A, h_stride=64, h_dtype=0, scale=1.0, eps=1e-5)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(x_out=None, h=None, gain=None), dict(gain=None), dict(h=None), dict(y=None, gate=A),
    dict(y=None, post_gain=A), dict(x_dtype=3), dict(y_dtype=-1), dict(h_dtype=9), dict(x=A + 2), dict(y=A + 1),
    dict(h=A + 1), dict(x_stride=63), dict(y_stride=63), dict(h_stride=63), dict(x_out_stride=63),
    dict(x_out_stride=65), dict(gate=A, gate_dtype=4), dict(gate=A + 1, gate_dtype=1),
    dict(gate=A, gate_col_stride=2), dict(gate=A, gate_row_stride=-1), dict(gain=A + 2), dict(post_gain=A + 1),
    dict(eps=-1.0), dict(eps=float("nan"))])
def test_block_norm_arguments(lib, kw):
    assert lib.hvd_block_norm(ctypes.byref(norm_args(**kw)), 2, 64, None) == HVD_ERR_ARG


@pytest.mark.parametrize("rows,dim", [(-1, 64), (1, 0), (1, 16385), ((1 << 23) + 1, 64)])
def test_block_norm_sizes(lib, rows, dim):
    assert lib.hvd_block_norm(ctypes.byref(norm_args()), rows, dim, None) == HVD_ERR_ARG


def test_tensors_on_the_host_are_refused():
    import torch
    x = torch.zeros(2, 64)
    with pytest.raises(hvd.HvdError):
        hvd.route(x, 2)
    with pytest.raises(hvd.HvdError):
        hvd.Experts(torch.zeros(2, 32, 64), torch.zeros(2, 32, 64), torch.zeros(2, 64, 32))
    with pytest.raises(hvd.HvdError):
        hvd.block_norm(x, x)
