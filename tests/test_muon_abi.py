"""Updates with orthogonalised momentum without a GPU: arguments that are refused before any CUDA work."""
import ctypes
import math

import numpy as np
import pytest

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb
from tests.muon_reference import orthogonalise

INVALID, UNSUPPORTED, OK, OOM = darb.ERR_INVALID_ARG, darb.ERR_UNSUPPORTED, darb.OK, darb.ERR_OOM
X, Y, Z = 1 << 24, 2 << 24, 3 << 24   # addresses that no accepted call here dereferences


@pytest.fixture(scope="module")
def L():
    darb_build.build()
    return darb.lib()


def create(L, n=2, rows=(10, 30), cols=(20, 7), p=(X, X + 65536), m=(Y, Y + 65536), c=None, dt=0):
    arr = lambda a, t: None if a is None else (t * len(a))(*a)  # noqa: E731
    out = ctypes.c_void_p(77)
    st = L.darb_muon_create(n, arr(rows, ctypes.c_int64), arr(cols, ctypes.c_int64), arr(p, ctypes.c_void_p), arr(m, ctypes.c_void_p),
                            arr(c, ctypes.c_void_p), dt, ctypes.byref(out), None)
    return st, out.value


def test_create_refusals(L, monkeypatch):
    for kw in (dict(n=0), dict(rows=None), dict(cols=None), dict(p=None), dict(m=None), dict(dt=2), dict(rows=(10, -1)), dict(p=(X, None)),
               dict(m=(None, Y)), dict(p=(X, X + 796)), dict(m=(X, Y)), dict(p=(X + 2, X + 65536)), dict(c=(X, None)), dict(c=(Z, Z + 398)),
               dict(c=(Z + 1, None))):
        assert create(L, **kw) == (INVALID, None), kw
    assert create(L, rows=(10, 32769)) == (UNSUPPORTED, None) and create(L, cols=(1 << 40, 1)) == (UNSUPPORTED, None)
    monkeypatch.setenv("DARB_FAIL_ALLOC", "1")
    assert create(L) == (OOM, None)
    assert L.darb_muon_create(1, None, None, None, None, None, 0, None, None) == INVALID


def test_step_refusals(L):
    st, plan = create(L, rows=(0, 5), cols=(4, 0), p=(None, None), m=(None, None))   # matrices without elements need no device
    assert st == OK
    g = (ctypes.c_void_p * 2)()
    hyper = (1e-3, 0.9, 0.0, 1e-7)
    call = lambda h, grads=g, scale=None, plan=plan: L.darb_muon_step(plan, grads, scale, *h, 1, None)  # noqa: E731
    assert call(hyper) == OK
    assert call(hyper, None) == INVALID and call(hyper, scale=X + 2) == INVALID
    for i, bad in ((0, -1.0), (0, math.inf), (1, 1.0), (1, -0.1), (2, -1e-9), (2, math.nan), (3, 0.0), (3, math.nan)):
        h = list(hyper)
        h[i] = bad
        assert call(h) == INVALID, (i, bad)
    assert L.darb_muon_sync_status(plan, None) == OK
    assert L.darb_muon_destroy(plan) == OK
    assert call(hyper) == INVALID and L.darb_muon_destroy(plan) == INVALID and L.darb_muon_sync_status(plan, None) == INVALID
    assert L.darb_muon_destroy(None) == OK


@pytest.mark.parametrize("rows,cols", [(12, 12), (5, 40), (33, 6), (1, 9)])
def test_reference_pulls_singular_values_to_one(rows, cols):
    """What the five iterations are for: singular values of the direction end in a band around 1, its vectors stay."""
    u = np.random.default_rng(rows).standard_normal((rows, cols))
    x = orthogonalise(u)
    s = np.linalg.svd(x, compute_uv=False)
    assert s.min() > 0.3 and s.max() < 1.3
    np.testing.assert_allclose((u.T @ x), (u.T @ x).T, atol=1e-10 * np.abs(u).max() ** 2 * rows)
