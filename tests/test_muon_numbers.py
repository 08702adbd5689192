"""Orthogonalised momentum without a GPU: step sizes and the like that 64 bits hold and 32 do not."""
import ctypes

import pytest

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb

SMALLEST = 2.0 ** -149   # of 32 bits


@pytest.fixture(scope="module")
def step():
    darb_build.build()
    L = darb.lib()
    none, plan = (ctypes.c_void_p * 1)(), ctypes.c_void_p()
    side = (ctypes.c_int64 * 1)(0)   # a matrix without elements needs no device
    assert L.darb_muon_create(1, side, side, none, none, None, darb.F32, ctypes.byref(plan), None) == darb.OK
    yield lambda lr=1e-3, beta=0.9, decay=0.01, eps=1e-7: L.darb_muon_step(plan, none, None, lr, beta, decay, eps, 1, None)
    L.darb_muon_destroy(plan)


@pytest.mark.parametrize("kw", [dict(eps=1e-46), dict(eps=5e-324), dict(eps=1e39), dict(lr=1e39), dict(lr=1e300, decay=1e300), dict(lr=1e30, decay=1e30),
                                dict(decay=float("inf"))])
def test_refused_as_they_are_rounded(step, kw):
    assert step(**kw) == darb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [{}, dict(eps=SMALLEST), dict(eps=1e38), dict(lr=0.0), dict(lr=1e30, decay=0.0), dict(lr=0.0, decay=1e300)])
def test_taken(step, kw):
    assert step(**kw) == darb.OK
