"""A small prune-retrain loop of a language model's output layer, on synthetic data.

Run ``python -m paper_1911_08020_gb300.retrain``.  Hidden states (features x tokens, as the steps write
them) go through layer norm and the pruned output layer; the given words are scored, the gradient comes
back, one AdamW step updates the dense weights, and the layer is encoded again:

    darb_layer_norm -> darb_spmm -> darb_token_logprobs -> darb_token_logprobs_grad
      -> darb_layer_norm_grad -> darb_adamw_step -> darb_reencode

(``states="muon"``: the weights take darb_muon_step, whose momentum is orthogonalised, and AdamW the vectors.)
The products of the backward pass are plain dense ones (library calls).  The gradient of the layer's input
is that of the pruned layer, whose dense form is the product with the identity.  The gradient of the weights
passes the pruning straight through: that of a pruned weight is that of the weight at its place, so that
the best weight of a block can change from one encode to the next.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import darb


class Head:
    """Layer norm and a pruned output layer, trained with AdamW (states in 8 bits, or fp32), or the weights with
    orthogonalised momentum."""

    def __init__(self, vocab: int, features: int, block: int, lr: float = 2e-3, states: str = "e4m3", seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.W = torch.randn(vocab, features, generator=gen, device="cuda") / math.sqrt(features)
        self.eye = torch.eye(features, device="cuda")
        self.gamma, self.beta = torch.ones(features, device="cuda"), torch.zeros(features, device="cuda")
        self.stored = self.W.to(torch.bfloat16)   # what is encoded
        self.handle = darb.darb_encode(self.stored, np.full(vocab, block, np.int32))
        params, copies, self.muon = [self.W, self.gamma, self.beta], [self.stored, None, None], None
        if states == "muon":
            self.muon = darb.darb_muon_create(params[:1], [torch.zeros_like(self.W)], copies=copies[:1])
            params, copies = params[1:], None
        if states == "e4m3":
            def codes(p):
                return torch.zeros(p.numel(), device=p.device).to(torch.float8_e4m3fn)

            def scales(p):
                return torch.zeros(-(-p.numel() // darb.ADAMW_BLOCK), device=p.device)

            moments = [[codes(p) for p in params] for _ in range(2)] + [[scales(p) for p in params] for _ in range(2)]
        else:
            moments = [[torch.zeros_like(p) for p in params] for _ in range(2)]
        self.plan = darb.darb_adamw_create(params, *moments, copies=copies)
        self.lr, self.step = lr, 0

    def forward(self, h):
        """(normalised states, their statistics, logits vocab x tokens) of hidden states h (features x tokens)."""
        x, mean, rstd = darb.darb_layer_norm(h, self.gamma, self.beta, dim=0)
        return x, (mean, rstd), darb.darb_spmm(self.handle, x)

    def score(self, h, words, k: int = 0) -> darb.TokenLogprobs:
        """Log probability of the given words, entropy and the k best alternatives."""
        return darb.darb_token_logprobs(self.forward(h)[2], words, k, dim=0)

    def train(self, h, words) -> torch.Tensor:
        """One step on the mean negative log probability of `words`; returns the log probabilities before it."""
        x, (mean, rstd), logits = self.forward(h)
        scores = darb.darb_token_logprobs(logits, words, dim=0)
        d_logprob = torch.full_like(scores.logprob, -1.0 / h.shape[1])
        d_logits = darb.darb_token_logprobs_grad(logits, words, scores.lse, d_logprob, dim=0, out=logits)
        dW, dx = d_logits @ x.t(), darb.darb_spmm(self.handle, self.eye).t() @ d_logits
        _, d_gamma, d_beta = darb.darb_layer_norm_grad(dx, h, self.gamma, mean, rstd, dim=0, dx=dx)
        self.step += 1
        if self.muon is not None:
            darb.darb_muon_step(self.muon, [dW], self.lr)
        darb.darb_adamw_step(self.plan, [d_gamma, d_beta] if self.muon is not None else [dW, d_gamma, d_beta], self.step, self.lr)
        darb.darb_reencode(self.handle, self.stored)
        return scores.logprob

    def close(self):
        darb.darb_adamw_destroy(self.plan)
        darb.darb_muon_destroy(self.muon)
        darb.darb_destroy(self.handle)


def data(tokens: int, vocab: int, features: int, seed: int):
    """Hidden states (features x tokens) and words that a fixed random layer finds likely for them."""
    gen = torch.Generator(device="cuda").manual_seed(1234)
    truth = torch.randn(vocab, features, generator=gen, device="cuda")
    gen.manual_seed(seed)
    h = torch.randn(features, tokens, generator=gen, device="cuda")
    return h, (truth @ h / math.sqrt(features) * 4.0).argmax(dim=0)


def retrain(steps: int = 200, vocab: int = 2000, features: int = 256, tokens: int = 512, block: int = 8, states: str = "e4m3"):
    """(perplexity before, perplexity after) on held-out tokens."""
    head = Head(vocab, features, block, states=states)
    try:
        held_out = data(4 * tokens, vocab, features, seed=99)
        perplexity = lambda: math.exp(-head.score(*held_out).logprob.mean().item())  # noqa: E731
        before = perplexity()
        for i in range(steps):
            head.train(*data(tokens, vocab, features, seed=i))
        return before, perplexity()
    finally:
        head.close()


if __name__ == "__main__":
    for kind in ("f32", "e4m3", "muon"):
        print("states %s: perplexity %.1f -> %.1f" % ((kind,) + retrain(states=kind)))
