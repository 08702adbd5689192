"""The scoring and training calls without a GPU: arguments that are refused before any CUDA work."""
import ctypes

import numpy as np
import pytest

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb

INVALID, UNSUPPORTED, OK, OOM = darb.ERR_INVALID_ARG, darb.ERR_UNSUPPORTED, darb.OK, darb.ERR_OOM
X, Y, Z = 1 << 20, 2 << 20, 3 << 20   # addresses that no accepted call here dereferences


@pytest.fixture(scope="module")
def L():
    darb_build.build()
    return darb.lib()


def test_token_logprobs_refusals(L):
    base = dict(x=X, dt=0, lay=0, n=4, v=100, ld=100, tg=Y, k=0, lp=Z, en=None, lse=None, tl=None, ti=None)

    def call(**kw):
        a = dict(base, **kw)
        return L.darb_token_logprobs(a["x"], a["dt"], a["lay"], a["n"], a["v"], a["ld"], a["tg"], a["k"], a["lp"], a["en"], a["lse"],
                                     a["tl"], a["ti"], None)

    for kw in (dict(x=None), dict(dt=2), dict(lay=2), dict(n=-1), dict(v=0), dict(ld=99), dict(lay=1, ld=3), dict(tg=None), dict(lp=None),
               dict(k=33), dict(k=-1), dict(v=5, ld=5, k=6), dict(k=2), dict(k=2, tl=Z + 4096), dict(x=X + 2), dict(x=X + 1, dt=1),
               dict(lp=Z + 2), dict(tg=Y + 4), dict(lp=X), dict(lse=Z), dict(en=Y)):
        assert call(**kw) == INVALID, kw
    assert call(n=0) == OK and call(n=0, x=None, tg=None, lp=None) == OK
    assert call(n=(1 << 27) + 1) == UNSUPPORTED and call(v=1 << 31, ld=1 << 31) == UNSUPPORTED
    assert call(ld=1 << 62) == UNSUPPORTED


def test_token_logprobs_grad_refusals(L):
    base = dict(x=X, dt=0, lay=0, n=4, v=100, ld=100, tg=Y, lse=Y + 4096, en=None, da=Y + 8192, db=None, dx=Z, ldg=100)

    def call(**kw):
        a = dict(base, **kw)
        return L.darb_token_logprobs_grad(a["x"], a["dt"], a["lay"], a["n"], a["v"], a["ld"], a["tg"], a["lse"], a["en"], a["da"], a["db"],
                                          a["dx"], a["ldg"], None)

    for kw in (dict(x=None), dict(dx=None), dict(lse=None), dict(tg=None), dict(db=Y), dict(ld=99), dict(ldg=99), dict(dx=X + 4),
               dict(dx=X, ldg=101), dict(dx=Y), dict(dx=Z + 1), dict(dt=-1), dict(lay=3), dict(lay=1, ld=4, ldg=3), dict(v=0), dict(n=-2)):
        assert call(**kw) == INVALID, kw
    assert call(n=0) == OK
    assert call(ld=1 << 62, dx=X) == UNSUPPORTED


def test_layer_norm_refusals(L):
    base = dict(x=X, dt=0, lay=0, s=1, n=4, f=100, ld=100, g=None, b=None, eps=1e-5, y=Y, ldy=100, mean=None, rstd=None)

    def call(**kw):
        a = dict(base, **kw)
        return L.darb_layer_norm(a["x"], a["dt"], a["lay"], a["s"], a["n"], a["f"], a["ld"], a["g"], a["b"], a["eps"], a["y"], a["ldy"],
                                 a["mean"], a["rstd"], None)

    for kw in (dict(x=None), dict(y=None), dict(dt=9), dict(lay=-1), dict(s=2), dict(s=-1, lay=1), dict(f=0), dict(ld=99), dict(ldy=99),
               dict(eps=-1e-5), dict(eps=float("nan")), dict(y=X + 4), dict(y=X, ldy=200, ld=100), dict(mean=Y), dict(mean=Z, rstd=Z),
               dict(g=X + 2), dict(lay=1, ld=4, ldy=3), dict(g=Y)):
        assert call(**kw) == INVALID, kw
    assert call(n=0) == OK and call(lay=1, s=0) == OK
    assert call(f=(1 << 24) + 1, ld=1 << 25, ldy=1 << 25) == UNSUPPORTED and call(ld=1 << 61) == UNSUPPORTED


def test_layer_norm_grad_refusals(L):
    need = ctypes.c_int64()
    assert L.darb_layer_norm_grad_work(0, 1, 4, 100, ctypes.byref(need)) == OK and need.value > 0
    assert L.darb_layer_norm_grad_work(0, 1, 4, 100, None) == INVALID
    assert L.darb_layer_norm_grad_work(0, 2, 4, 100, ctypes.byref(need)) == INVALID
    W = 64 << 20
    base = dict(dy=X, ldd=100, x=Y, ld=100, dt=0, lay=0, s=1, n=4, f=100, g=None, mean=Z, rstd=Z + 4096, dx=4 << 20, ldo=100,
                dg=5 << 20, db=6 << 20, work=W)

    def call(**kw):
        a = dict(base, **kw)
        return L.darb_layer_norm_grad(a["dy"], a["ldd"], a["x"], a["ld"], a["dt"], a["lay"], a["s"], a["n"], a["f"], a["g"], a["mean"],
                                      a["rstd"], a["dx"], a["ldo"], a["dg"], a["db"], a["work"], None)

    for kw in (dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dg=None), dict(db=None),
               dict(work=W + 4), dict(dx=Y), dict(dx=X, ldo=101), dict(dg=6 << 20), dict(dg=X), dict(work=X), dict(ldd=99), dict(ldo=99),
               dict(f=-1), dict(s=0x7FFFFFFF)):
        assert call(**kw) == INVALID, kw
    assert call(n=0, dg=None, db=None, work=None) == OK
    assert call(n=0, db=5 << 20) == INVALID


def _adamw(L, n=2, numel=(10, 300), p=(X, X + 65536), m=(Y, Y + 65536), v=(Z, Z + 65536), ms=None, vs=None, c=None, dt=0):
    arr = lambda a: None if a is None else (ctypes.c_void_p * len(a))(*a)
    out = ctypes.c_void_p(77)
    st = L.darb_adamw_create(n, None if numel is None else (ctypes.c_int64 * len(numel))(*numel), arr(p), arr(m), arr(v), arr(ms), arr(vs),
                             arr(c), dt, ctypes.byref(out), None)
    return st, out.value


def test_adamw_refusals(L, monkeypatch):
    S, S2 = (5 << 20, (5 << 20) + 4096), (6 << 20, (6 << 20) + 4096)
    for kw in (dict(n=0), dict(numel=None), dict(p=None), dict(m=None), dict(v=None), dict(dt=3), dict(numel=(10, -1)), dict(ms=S),
               dict(p=(X, None)), dict(m=(None, Y)), dict(p=(X, X + 36)), dict(m=(X, Y)), dict(p=(X + 2, X + 65536)),
               dict(ms=S, vs=(6 << 20, None)), dict(ms=S, vs=S), dict(c=(X, None)), dict(c=(7 << 20, (7 << 20) + 1))):
        assert _adamw(L, **kw) == (INVALID, None), kw
    assert _adamw(L, numel=(10, 1 << 50)) == (UNSUPPORTED, None)
    assert _adamw(L, numel=(10, 1 << 45), p=(X, 1 << 50), m=(Y, 1 << 51), v=(Z, 1 << 52)) == (UNSUPPORTED, None)
    monkeypatch.setenv("DARB_FAIL_ALLOC", "1")
    assert _adamw(L) == (OOM, None)
    assert L.darb_adamw_create(1, None, None, None, None, None, None, None, 0, None, None) == INVALID
    # tensors without elements need no device
    st, plan = _adamw(L, numel=(0, 0), p=(None, None), m=(None, None), v=(None, None))
    assert st == OK
    g = (ctypes.c_void_p * 2)()
    hyper = (1e-3, 0.9, 0.999, 1e-8, 0.0)
    assert L.darb_adamw_step(plan, g, None, 1, 0, *hyper, None) == OK
    assert L.darb_adamw_step(plan, g, None, 0, 0, *hyper, None) == INVALID
    assert L.darb_adamw_step(plan, None, None, 1, 0, *hyper, None) == INVALID
    for i, bad in ((0, -1.0), (0, np.inf), (1, 1.0), (2, np.nan), (3, -1e-8), (4, np.nan)):
        h = list(hyper)
        h[i] = float(bad)
        assert L.darb_adamw_step(plan, g, None, 1, 0, *h, None) == INVALID
    assert L.darb_adamw_sync_status(plan, None) == OK
    assert L.darb_adamw_destroy(plan) == OK
    assert L.darb_adamw_sync_status(plan, None) == INVALID
    assert L.darb_adamw_step(plan, g, None, 1, 0, *hyper, None) == INVALID and L.darb_adamw_destroy(plan) == INVALID
    assert L.darb_adamw_destroy(None) == OK
