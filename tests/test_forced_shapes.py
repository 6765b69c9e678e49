"""Forced GEMM shapes (mid_plan.h, through the host-only build): families that
cannot be forced -- an expert layer's router -- have none, and read no other's."""

import ctypes
import os

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_01019_amd")


@pytest.mark.parametrize("family", list(range(12)) + [-1])
def test_families_without_an_option(family):
    path = os.path.join(PKG, "libhvd_host.so")
    if not os.path.exists(path):
        from paper_2606_01019_amd.build import build
        build()
    out = (ctypes.c_int32 * 2)(7, 7)
    ctypes.CDLL(path).hvdh_forced_shape(family, out)
    assert tuple(out) == ((10 * family + 1, 10 * family + 2) if 0 <= family < 5 else (0, 0))
