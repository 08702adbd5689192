"""The policy loss without a GPU: arguments that are refused before any CUDA work, and the reference's gradients."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb
from tests.policy_reference import policy

INVALID, UNSUPPORTED, OK = darb.ERR_INVALID_ARG, darb.ERR_UNSUPPORTED, darb.OK
A, B, C, D, E, F, G, H, I, J, W = (i << 24 for i in range(1, 12))   # addresses that no accepted call here dereferences


@pytest.fixture(scope="module")
def L():
    darb_build.build()
    return darb.lib()


def call(L, **kw):
    a = dict(n=6000, s=9, lp=A, old=B, ref=C, ent=D, mask=E, adv=F, off=G, low=0.2, high=0.2, kl=0.1, bonus=0.1, ratio=0, mean=0, stats=H,
             dlp=I, dent=J, work=W)
    a.update(kw)
    return L.darb_policy_loss(a["n"], a["s"], a["lp"], a["old"], a["ref"], a["ent"], a["mask"], a["adv"], a["off"], a["low"], a["high"],
                              a["kl"], a["bonus"], a["ratio"], a["mean"], a["stats"], a["dlp"], a["dent"], a["work"], None)


def test_refusals(L):
    nan, inf = math.nan, math.inf
    for kw in (*({k: None} for k in ("lp", "old", "ref", "ent", "adv", "off", "stats", "dlp")), dict(n=-1), dict(s=-1), dict(low=-0.1),
               dict(low=1.1), dict(low=nan), dict(high=-0.1), dict(high=nan), dict(kl=inf), dict(bonus=nan), dict(ratio=2), dict(mean=-1),
               dict(ent=None, bonus=0.0), dict(lp=A + 2), dict(off=G + 4), dict(work=W + 8), dict(adv=F + 1), dict(dlp=A), dict(dlp=A + 400),
               dict(dent=I + 100), dict(stats=F + 8), dict(dlp=E), dict(dent=D), dict(stats=I + 40), dict(work=I), dict(work=B + 16),
               dict(dent=G)):
        assert call(L, **kw) == INVALID, kw
    assert call(L, n=(1 << 27) + 1, lp=1 << 40, old=2 << 40, ref=3 << 40) == UNSUPPORTED and call(L, s=(1 << 27) + 1) == UNSUPPORTED


def test_work_sizes(L):
    need = ctypes.c_int64()
    assert L.darb_policy_loss_work(4096, ctypes.byref(need)) == OK and need.value == 0
    assert L.darb_policy_loss_work(4097, ctypes.byref(need)) == OK and 12 * 4097 <= need.value < 13 * 4097
    assert L.darb_policy_loss_work(1 << 27, ctypes.byref(need)) == OK
    assert L.darb_policy_loss_work(-1, ctypes.byref(need)) == INVALID and L.darb_policy_loss_work(5, None) == INVALID
    assert L.darb_policy_loss_work((1 << 27) + 1, ctypes.byref(need)) == UNSUPPORTED


@pytest.mark.parametrize("ratio", [0, 1])
@pytest.mark.parametrize("mean", [0, 1])
def test_reference_gradients(ratio, mean):
    """The formulas that the GPU tests go by, against automatic differentiation and differences."""
    g = np.random.default_rng(4)
    offsets = np.array([1, 1, 6, 14, 14, 30])
    n = 33
    lp, old, ref = (-g.random(n) * 2 for _ in range(3))
    ent, adv, mask = g.random(n), g.standard_normal(5), g.random(n) < 0.8

    def loss(lp, ent):
        total, tokens, sequences = 0.0, 0, 0
        for s in range(5):
            i = [t for t in range(offsets[s], offsets[s + 1]) if mask[t]]
            if not i:
                continue
            tokens, sequences = tokens + len(i), sequences + 1
            d = lp[i] - torch.tensor(old[i])
            r = (d.mean().expand(len(i)) if ratio else d).exp()
            gain = torch.minimum(r * adv[s], r.clamp(0.8, 1.3) * adv[s])
            x = torch.tensor(ref[i]) - lp[i]
            part = (-gain + 0.07 * (x.exp() - 1 - x) - 0.02 * ent[i]).sum()
            total = total + (part / len(i) if mean else part)
        return total / (sequences if mean else tokens)

    leaves = [torch.tensor(v, requires_grad=True) for v in (lp, ent)]
    value = loss(*leaves)
    value.backward()
    (stats, d_lp, d_ent), _, _ = policy(lp, old, adv, offsets, ref, ent, mask, 0.2, 0.3, 0.07, 0.02, ratio, mean)
    assert abs(stats[0] - value.item()) < 1e-13
    np.testing.assert_allclose(d_lp, leaves[0].grad.numpy(), rtol=1e-11, atol=1e-15)
    np.testing.assert_allclose(d_ent, leaves[1].grad.numpy(), rtol=1e-11, atol=1e-15)
    for i in (3, 9, 20):   # differences (no ratio here is within 1e-4 of a border)
        up, down = lp.copy(), lp.copy()
        up[i] += 1e-6
        down[i] -= 1e-6
        slope = (loss(torch.tensor(up), leaves[1]) - loss(torch.tensor(down), leaves[1])).item() / 2e-6
        assert abs(slope - d_lp[i]) < 1e-8
