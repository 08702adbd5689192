"""Scores of tokens whose distribution is one entry, on the GPU: an entropy is never below 0 and a log
probability never above it, so that a caller may take the logarithm of one and the exponential of the other."""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.test_gpu_logprobs import DTYPES, LAYOUTS, U, place

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(2000, 40), (60, 5003), (3, 130000)])
def test_signs(n, v, dtype, layout):
    g = np.random.default_rng(v)
    x = np.full((n, v), -np.inf, np.float32)
    at = g.integers(0, v, n)
    x[np.arange(n), at] = g.uniform(-40.0, 40.0, n)
    x[n // 2, at[n // 2]] = 1e6
    near = np.arange(n) % 3 == 1                     # others there, with next to no probability
    x[near] = np.where(np.isfinite(x[near]), x[near], -90.0)
    t, dim = place(x, layout, dtype)
    got = darb.darb_token_logprobs(t, torch.from_numpy(at).cuda(), min(v, 4), dim=dim)
    assert got.entropy.ge(0).all() and got.logprob.le(0).all() and got.top_logprob.le(0).all()
    # (by the definition: exp(-50) of others at most, and 8 roundings of numbers up to 60)
    assert got.entropy.le(512 * U).all() and got.logprob.ge(-512 * U).all()
    assert torch.equal(got.top_index[:, 0].cpu().long(), torch.from_numpy(at))


@pytest.mark.parametrize("layout", LAYOUTS)
def test_nan_stays(layout):
    t, dim = place(np.array([[0.0, np.nan], [np.inf, 1.0]], np.float32), layout, "f32")
    got = darb.darb_token_logprobs(t, torch.zeros(2, dtype=torch.int64, device="cuda"), 2, dim=dim)
    assert got.entropy.isnan().all() and got.logprob.isnan().all() and got.top_logprob.isnan().all()
