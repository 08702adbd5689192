"""What a call of the binding does not compute is not in what it returns, although a buffer for it was given."""
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def test_scores_into_buffers_kept_from_an_earlier_call():
    x = torch.randn(6, 50, device="cuda")
    targets = torch.arange(6, device="cuda")
    out = darb.TokenLogprobs.empty(6, 3)
    full = darb.darb_token_logprobs(x, targets, 3, out=out)
    assert all(a is b for a, b in zip(full, out))
    y = torch.randn(6, 50, device="cuda")
    got = darb.darb_token_logprobs(y, None, 0, out=out)
    assert got.logprob is None and got.top_logprob is None and got.top_index is None
    assert got.lse is out.lse and got.entropy is out.entropy
    assert torch.allclose(got.lse, torch.logsumexp(y, 1), rtol=0, atol=1e-5)
    got = darb.darb_token_logprobs(y, targets, 0, out=darb.TokenLogprobs.empty(6, 0))
    assert got.logprob is not None and got.top_index.shape == (6, 0)
