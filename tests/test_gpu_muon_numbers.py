"""Orthogonalised momentum at the ends of what 32 bits hold (the refusals: test_muon_numbers.py)."""
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.muon_reference import COEFFICIENTS, step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("eps", [2.0 ** -149, 1e-40, 1e-7, 1e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_zero_gradients_at_any_eps(dtype, eps):
    """X = 0: the decay alone, of which 1 - lr decay and the product are rounded."""
    p = [torch.randn(r, c, device="cuda") for r, c in ((40, 70), (65, 64))]
    keep = [t.clone() for t in p]
    with darb.darb_muon_create(p, [torch.zeros_like(t) for t in p], grad_dtype=dtype) as plan:
        darb.darb_muon_step(plan, [torch.zeros_like(t, dtype=dtype) for t in p], 0.1, weight_decay=0.5, eps=eps)
        darb.darb_muon_sync_status(plan)
    for t, k in zip(p, keep):
        assert bool(((t.double() - 0.95 * k.double()).abs() <= 2 * U * k.double().abs()).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size,eps", [(2e38, 1e-7), (2e38, 3e38), (1e38, 3e38)])
def test_a_norm_past_32_bits(dtype, size, eps):
    """The norm of numbers that 32 bits hold, and its sum with eps, may be past their range.

    The matrix has one number in a row, none in a column twice: all of its singular values are the same s, X keeps its
    form, and every product has one term.  So a step is s' = a s + b s^3 + c s^5, whose terms have up to five factors
    that are off by e relative to themselves: 2^-12 (bf16 gradients: one fp16 number) or 2^-21 (two of them).  What a
    step is off by goes through the derivatives of the steps after it; s at the start, by 5 e."""
    n = 600
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = torch.zeros(n, n + 7, device="cuda", dtype=dtype)
    g[torch.arange(n, device="cuda"), torch.randperm(n + 7, generator=gen, device="cuda")[:n]] = size
    p, m = [torch.zeros(n, n + 7, device="cuda")], [torch.zeros(n, n + 7, device="cuda")]
    with darb.darb_muon_create(p, m, grad_dtype=dtype) as plan:
        darb.darb_muon_step(plan, [g], 0.1, weight_decay=0.0, eps=eps)
        darb.darb_muon_sync_status(plan)
    _, _, x = step(np.zeros(g.shape), np.zeros(g.shape), g.double().cpu().numpy(), 0.1, eps=eps)
    got = p[0].double().cpu().numpy() / -(0.1 * 0.2 * math.sqrt(max(g.shape)))
    a, b, c = COEFFICIENTS
    u = g.max().item() * 0.05 * 1.95
    s = u / (math.sqrt(n) * u + eps)
    off, e = 5 * s, 2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -21
    for _ in range(5):
        off = abs(a + 3 * b * s ** 2 + 5 * c * s ** 4) * off + 5 * (a * s + abs(b) * s ** 3 + c * s ** 5)
        s = a * s + b * s ** 3 + c * s ** 5
    assert abs(np.abs(x).max() - s) < 1e-9 and off * 2.0 ** -12 < 0.1 * s   # (the bound tells X from 0)
    assert np.abs(got - x).max() <= off * e


def test_a_gradient_of_another_shape_is_refused():
    """As many numbers, side by side, but other rows: the transpose's, a vector's.  Nothing is written."""
    p = [torch.randn(8, 6, device="cuda"), torch.randn(5, 5, device="cuda")]
    keep, m = [t.clone() for t in p], [torch.zeros_like(t) for t in p]
    g = [torch.randn_like(t) for t in p]
    with darb.darb_muon_create(p, m) as plan:
        for bad in (g[0].t().contiguous(), g[0].view(-1), g[0].view(4, 12), g[0].view(1, 8, 6)):
            with pytest.raises(darb.DarbError):
                darb.darb_muon_step(plan, [bad, g[1]], 0.1)
            with pytest.raises(darb.DarbError):
                darb.darb_muon_step(plan, [bad, None], 0.1)
        darb.darb_muon_sync_status(plan)
        assert all(torch.equal(t, k) for t, k in zip(p, keep)) and not any(t.any() for t in m)
        darb.darb_muon_step(plan, g, 0.1)
        assert not torch.equal(p[0], keep[0])
