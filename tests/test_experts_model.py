"""Decoders with expert layers, on the CPU: what their loading refuses, and the
oracle's own invariants."""

import ctypes

import numpy as np
import pytest

import oracle
import paper_2606_01019_amd as hvd
from paper_2606_01019_amd.hvd import HVD_ERR_ARG, Config, MoeConfig, tensor_names
from tests._experts import GROUPED, GROUPED_MOE, SMALL, SMALL_MOE, weights
from workloads import tokens as wt


@pytest.fixture(scope="module")
def lib():
    return hvd.load_library()


def change(m, **kw):
    c = MoeConfig.from_moe_config(m)
    for k, v in kw.items():
        setattr(c.route if hasattr(c.route, k) else c, k, v)
    return c


@pytest.mark.parametrize("kw", [dict(first_layer=-1), dict(first_layer=3), dict(ffn_dim=0), dict(ffn_dim=48),
                                dict(ffn_dim=1 << 18), dict(out_scale=float("nan")), dict(n_experts=0), dict(n_experts=513),
                                dict(top_k=0), dict(top_k=17), dict(n_groups=3), dict(n_groups=4, top_groups=5),
                                dict(score=7), dict(scale=float("inf"))])
def test_refused_configs(lib, kw):
    c, m = Config.from_model_config(SMALL), change(SMALL_MOE, **kw)
    assert lib.hvd_model_bytes_moe(ctypes.byref(c), ctypes.byref(m)) == 0
    assert lib.hvd_kv_bytes_moe(ctypes.byref(c), ctypes.byref(m), 1, 8) == 0
    ptrs = (ctypes.c_void_p * 64)(*[1 << 20] * 64)
    h = ctypes.c_void_p()
    assert lib.hvd_model_load_moe(ctypes.byref(c), ctypes.byref(m), ptrs, 1 << 20, 1 << 40, None, ctypes.byref(h)) == HVD_ERR_ARG


def test_sizes(lib):
    c, m = Config.from_model_config(SMALL), change(SMALL_MOE)
    for f, args in (("hvd_model_bytes", ()), ("hvd_kv_bytes", (2, 32))):
        dense = getattr(lib, f)(ctypes.byref(c), *args)
        assert getattr(lib, f + "_moe")(ctypes.byref(c), None, *args) == dense
    assert lib.hvd_kv_bytes_moe(ctypes.byref(c), ctypes.byref(m), 2, 32) > lib.hvd_kv_bytes(ctypes.byref(c), 2, 32)
    expert = 3 * SMALL_MOE.n_experts * SMALL_MOE.ffn_dim * SMALL.d_model * 2
    dense = 3 * SMALL.ffn_dim * SMALL.d_model * 2
    got = lib.hvd_model_bytes_moe(ctypes.byref(c), ctypes.byref(m)) - lib.hvd_model_bytes(ctypes.byref(c))
    assert 2 * (expert - dense) < got < 2 * (expert - dense) + (1 << 19)  # and the routers


def test_null_tensors(lib):
    """Every tensor is needed, but for the bias and a post_norm that is off."""
    c, m = Config.from_model_config(SMALL), change(SMALL_MOE)
    names = tensor_names(SMALL.n_layers, SMALL_MOE.first_layer)
    assert len(names) == 3 + 9 + 2 * 12
    h = ctypes.c_void_p()
    for post in (0, 1):
        m.post_norm = post
        for i, n in enumerate(names):
            ptrs = (ctypes.c_void_p * len(names))(*[1 << 20] * len(names))
            ptrs[i] = None
            if n.endswith("router_bias") or (n.endswith("post_norm") and not post):
                continue
            # (too small a buffer: refused before anything is read either way)
            assert lib.hvd_model_load_moe(ctypes.byref(c), ctypes.byref(m), ptrs, 1 << 20, 1, None, ctypes.byref(h)) == HVD_ERR_ARG
            assert b"null tensor" in lib.hvd_last_error(), n
        ptrs = (ctypes.c_void_p * len(names))(*[None if n.endswith("router_bias") else 1 << 20 for n in names])
        assert lib.hvd_model_load_moe(ctypes.byref(c), ctypes.byref(m), ptrs, 1 << 20, 1, None, ctypes.byref(h)) == HVD_ERR_ARG
        assert b"dev_buf" in lib.hvd_last_error()


@pytest.mark.parametrize("cfg,moe,bias", [(SMALL, SMALL_MOE, False), (GROUPED, GROUPED_MOE, True)])
def test_oracle(cfg, moe, bias):
    w = weights(cfg, moe, bias=bias)
    om = oracle.OracleExpertsModel(cfg, w, moe)
    toks = wt.uniform_context(wt.rng_for("context", 5), 12, cfg.vocab)
    st = oracle.prefill(om, toks)
    got, _ = oracle.greedy_decode(om, st, 3)
    want, rows = oracle.brute_force_greedy(om, toks, 3)
    assert got == want
    # the rows' routing is their own: verified together or one by one, the same
    r = oracle.verify(om, st, got)
    assert np.abs(r.logits[:3] - rows).max() < 1e-9 and r.accepted == 3
    # and it matters (far more than the tolerance of the GPU tests)
    import dataclasses
    other = oracle.OracleExpertsModel(cfg, w, dataclasses.replace(moe, out_scale=0.0))
    assert np.abs(oracle.verify(other, oracle.prefill(other, toks), got).logits - r.logits).max() > 0.2
    once = oracle.OracleExpertsModel(cfg, w, dataclasses.replace(moe, top_k=moe.top_k - 1))
    assert np.abs(oracle.verify(once, oracle.prefill(once, toks), got).logits - r.logits).max() > 0.06


def test_oracle_of_one_expert_is_the_dense_mlp():
    from workloads.configs import MoeConfig as Shape
    moe = Shape(n_experts=1, top_k=1, ffn_dim=SMALL.ffn_dim)
    w = weights(SMALL, moe)
    for l in range(SMALL.n_layers):
        p = f"layers.{l}."
        w[p + "wg"], w[p + "wu"], w[p + "wd"] = (w[p + "experts_" + n][0] for n in ("gate", "up", "down"))
    toks = wt.uniform_context(wt.rng_for("context", 6), 9, SMALL.vocab)
    a, b = oracle.OracleExpertsModel(SMALL, w, moe), oracle.OracleModel(SMALL, w)
    la, lb = (oracle.verify(m, oracle.prefill(m, toks), []).logits for m in (a, b))
    assert np.abs(la - lb).max() < 1e-12
