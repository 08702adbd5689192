"""One step's gradients of the prune-retrain loop against automatic differentiation in 64 bits."""
import pytest
import torch

from paper_1911_08020_gb300 import darb, retrain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("vocab,features,block,tokens", [(300, 64, 8, 200), (97, 48, 4, 33)])
def test_gradients_are_those_of_the_pruned_layer(monkeypatch, vocab, features, block, tokens):
    head = retrain.Head(vocab, features, block, states="f32", seed=3)
    try:
        head.gamma.normal_(1.0, 0.3)
        head.beta.normal_(0.0, 0.3)
        h, words = retrain.data(tokens, vocab, features, seed=5)
        W = head.stored.double()
        taken = []
        monkeypatch.setattr(darb, "darb_adamw_step", lambda plan, grads, *a, **k: taken.extend(g.double() for g in grads))
        logprob = head.train(h, words).double()
    finally:
        head.close()
    # the layer that was multiplied: of every block of a row the weight of largest magnitude
    blocks = W.abs().view(vocab, features // block, block)
    kept = torch.zeros_like(blocks).scatter_(2, blocks.argmax(dim=2, keepdim=True), 1.0).view(vocab, features)
    W.requires_grad_(True)
    gamma, beta = (t.double().requires_grad_(True) for t in (head.gamma, head.beta))
    through = W + (W * kept - W).detach()      # its value is the pruned one's, its gradient the dense one's
    x = h.double()
    x = (x - x.mean(0)) / torch.sqrt(x.var(0, unbiased=False) + 1e-5)
    logp = torch.log_softmax(through @ (x * gamma[:, None] + beta[:, None]), dim=0)[words, torch.arange(tokens, device="cuda")]
    (-logp.mean()).backward()
    # fp32 sums of at most 300 terms, u = 2^-24: 300 u = 2e-5 of the terms, which exceed their sums by some times
    assert (logprob - logp).abs().max() < 1e-4
    for got, want in zip(taken, (W.grad, gamma.grad, beta.grad)):
        assert (got - want).norm() <= 2e-4 * want.norm(), float((got - want).norm() / want.norm())
