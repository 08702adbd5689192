"""Orthogonalised momentum at the ends of what 32 bits hold (the refusals: test_muon_numbers.py)."""
import pytest
import torch

from paper_1911_08020_gb300 import darb

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
