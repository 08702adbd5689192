"""The gated recurrence without a GPU: arguments that are refused before any CUDA work, and the formulas of the
backward pass against automatic differentiation."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb
from tests.scan_reference import back, forward

INVALID, UNSUPPORTED, OK = darb.ERR_INVALID_ARG, darb.ERR_UNSUPPORTED, darb.OK
A, B, C, D, E, F, G = (i << 24 for i in range(1, 8))   # addresses that no accepted call here dereferences


@pytest.fixture(scope="module")
def L():
    darb_build.build()
    return darb.lib()


def scan(L, **kw):
    a = dict(gate=A, ldg=10, sg=50, x=B, ldx=10, sx=50, dt=0, gates=0, outer=5, steps=7, inner=10, h0=None, h=C, ldh=10, sh=50, last=None)
    a.update(kw)
    return L.darb_gated_scan(a["gate"], a["ldg"], a["sg"], a["x"], a["ldx"], a["sx"], a["dt"], a["gates"], 1, a["outer"], a["steps"],
                             a["inner"], a["h0"], a["h"], a["ldh"], a["sh"], a["last"], None)


def grad(L, **kw):
    a = dict(dh=A, gate=B, x=C, h=D, dg=E, dx=F, dt=0, gates=0, outer=5, steps=7, inner=10, h0=None, dl=None, d0=None, ld={}, st={})
    a.update(kw)
    op = lambda k: (a[k], a["ld"].get(k, 10), a["st"].get(k, 50))  # noqa: E731
    return L.darb_gated_scan_grad(*op("dh"), *op("gate"), *op("x"), *op("h"), a["dt"], a["gates"], 1, a["outer"], a["steps"], a["inner"],
                                  a["h0"], a["dl"], *op("dg"), *op("dx"), a["d0"], None)


def test_scan_refusals(L):
    for kw in (dict(gate=None), dict(x=None), dict(h=None), dict(dt=2), dict(gates=2), dict(outer=-1), dict(steps=-1), dict(inner=-3),
               dict(ldg=9), dict(sx=49), dict(sh=-50), dict(ldh=-10), dict(x=B + 2), dict(x=B + 1, dt=1), dict(h0=D + 2), dict(last=D + 1),
               dict(h=A), dict(h=B, sh=60), dict(h=B + 4), dict(last=C), dict(last=A + 40), dict(h0=D, last=D + 4), dict(h0=C, last=C),
               dict(last=B), dict(gate=A, h=A, ldh=10)):
        assert scan(L, **kw) == INVALID, kw
    assert scan(L, outer=0) == OK and scan(L, inner=0, h=None, x=None, gate=None) == OK
    assert scan(L, steps=0, h=None, x=None, gate=None) == OK and scan(L, steps=0, h0=D, last=D) == OK
    for kw in (dict(steps=(1 << 30) + 1), dict(outer=1 << 16, inner=1 << 15, ldg=1 << 15), dict(sg=1 << 50)):
        assert scan(L, **kw) == UNSUPPORTED, kw


def test_slices_that_meet(L):
    """Slices of one buffer that share bytes with an input (those that share none are in test_gpu_scan.py)."""
    two = dict(outer=2, steps=3, inner=4)
    for kw in (dict(gate=A, x=A + 16, h=A + 20, ldg=36, sg=12, ldx=36, sx=12, ldh=36, sh=12, **two),
               dict(gate=A, x=A + 400, h=A + 404, ldg=1000, sg=4, ldx=1000, sx=4, ldh=1000, sh=4, **two),
               dict(gate=A, x=A + 400, h=A, ldg=1000, sg=4, ldx=1000, sx=4, ldh=1000, sh=4, **two),
               dict(gate=A, x=A + 4, h=A + 12, outer=6, steps=50, inner=1, ldg=300, sg=3, ldx=300, sx=3, ldh=300, sh=3),
               dict(gate=A, x=A + 4, h=A + 8, outer=6, steps=50, inner=1, ldg=300, sg=3, ldx=300, sx=3, ldh=300, sh=2)):
        assert scan(L, **kw) == INVALID, kw


def test_scan_grad_refusals(L):
    for kw in (*(({k: None}) for k in ("dh", "gate", "x", "h", "dg", "dx")), dict(dt=7), dict(gates=-1), dict(inner=-1),
               dict(ld={"h": 9}), dict(st={"dg": 49}), dict(dg=C), dict(dx=B), dict(dg=A), dict(dx=A), dict(dx=D), dict(dg=E, dx=E),
               dict(dg=B, st={"dg": 60}), dict(dg=B + 4), dict(d0=E), dict(d0=B), dict(dg=B, d0=B), dict(d0=G, dl=G + 4), dict(h0=G, d0=G),
               dict(h0=E), dict(dl=F + 8), dict(d0=G + 2)):
        assert grad(L, **kw) == INVALID, kw
    assert grad(L, outer=0) == OK and grad(L, steps=0, dl=G, d0=G) == OK
    assert grad(L, st={"dx": 1 << 50}) == UNSUPPORTED


@pytest.mark.parametrize("shape,strides,dim,want", [
    ((7, 5, 10), (50, 10, 1), 0, (1, 7, 50, -1, 0)), ((7, 5, 10), (60, 12, 1), 0, (5, 7, 10, 1, 0)),
    ((5, 7, 10), (70, 10, 1), 1, (5, 7, 10, 0, 1)), ((5, 7, 10), (140, 20, 1), -2, (5, 7, 10, 0, 1)),
    ((5, 7, 1), (7, 1, 1), 1, (5, 7, 1, 0, 1)), ((1, 7, 10), (999, 20, 1), 1, (1, 7, 10, -1, 1)),
    ((5, 10, 7), (70, 7, 1), 2, (50, 7, 1, 1, 2)), ((7, 10), (10, 1), 0, (1, 7, 10, -1, 0)), ((10, 7), (7, 1), 1, (10, 7, 1, 0, 1)),
    ((1, 7, 1), (9, 3, 2), 1, (1, 7, 1, -1, 1)), ((5, 1, 10), (10, 10, 1), 1, (1, 1, 50, -1, 1))])
def test_channels_of_a_tensor(shape, strides, dim, want):
    assert darb._channel_axes(shape, (strides, strides), dim, "call") == want


def test_channels_that_do_not_fit():
    shape, dense = (7, 5, 10), (50, 10, 1)
    with pytest.raises(darb.DarbError):
        darb._channel_axes(shape, (dense,), 3, "call")
    with pytest.raises(darb.DarbError):
        darb._channel_axes(shape, ((100, 20, 2), (100, 30, 2)), 0, "call")
    # one of the tensors is a slice: all go by two axes
    assert darb._channel_axes(shape, (dense, (100, 20, 1)), 0, "call") == (5, 7, 10, 1, 0)


@pytest.mark.parametrize("logits", [True, False])
@pytest.mark.parametrize("coupled", [True, False])
def test_reference_gradients(logits, coupled):
    """The formulas that the GPU tests go by, against automatic differentiation and differences."""
    gen = torch.Generator().manual_seed(3)
    gate, x, dh = (torch.randn(6, 4, generator=gen, dtype=torch.float64) for _ in range(3))
    h0, d_last = (torch.randn(4, generator=gen, dtype=torch.float64) for _ in range(2))
    leaves = [t.clone().requires_grad_() for t in (gate, x, h0)]

    def loss(gate, x, h0):
        state, total = h0, 0.0
        for t in range(6):
            a = torch.sigmoid(gate[t]) if logits else gate[t]
            state = a * state + ((1 - a) * x[t] if coupled else x[t])
            total = total + (state * dh[t]).sum()
        return total + (state * d_last).sum()

    loss(*leaves).backward()
    arrays = [t.numpy() for t in (gate, x, h0)]
    h = forward(*arrays, logits, coupled)[0]
    got = back(dh.numpy(), arrays[0], arrays[1], h, arrays[2], d_last.numpy(), logits, coupled)
    for g, leaf in zip(got[:3], leaves):
        np.testing.assert_allclose(g, leaf.grad.numpy(), rtol=1e-12, atol=1e-13)
    step = 1e-6
    for k in range(3):   # a difference of one element of each leaf; the second derivative's part is below 1e-11
        moved = [t.clone() for t in (gate, x, h0)]
        moved[k].view(-1)[2] += step
        up = loss(*moved)
        moved[k].view(-1)[2] -= 2 * step
        assert abs((up - loss(*moved)) / (2 * step) - got[k].reshape(-1)[2]) < 1e-8
