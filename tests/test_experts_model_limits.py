"""Decoders with more layers than the library counts: refused, not an exception at
the C entry."""

import ctypes

import pytest

import paper_2606_01019_amd as hvd
from paper_2606_01019_amd.hvd import HVD_ERR_ARG, Config, MoeConfig
from tests._experts import SMALL, SMALL_MOE


@pytest.mark.parametrize("layers", [(1 << 16) + 1, 1 << 28, (1 << 31) - 1])
def test_layers(layers):
    lib = hvd.load_library()
    c, m = Config.from_model_config(SMALL), MoeConfig.from_moe_config(SMALL_MOE)
    c.n_layers = 1 << 16
    assert lib.hvd_model_bytes_moe(ctypes.byref(c), ctypes.byref(m)) > 0
    c.n_layers = layers
    assert lib.hvd_model_bytes_moe(ctypes.byref(c), ctypes.byref(m)) == 0
    assert lib.hvd_kv_bytes_moe(ctypes.byref(c), ctypes.byref(m), 1, 8) == 0
    ptrs = (ctypes.c_void_p * 8)(*[1 << 20] * 8)
    h = ctypes.c_void_p()
    assert lib.hvd_model_load_moe(ctypes.byref(c), ctypes.byref(m), ptrs, 1 << 20, 1 << 40, None, ctypes.byref(h)) == HVD_ERR_ARG
    assert b"n_layers" in lib.hvd_last_error()
