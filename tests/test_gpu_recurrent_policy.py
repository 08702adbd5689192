"""A pruned recurrent layer and a pruned output layer, trained by the loss of words that were drawn: the calls together,
as a program makes them, against automatic differentiation in 64 bits and the update's formula."""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb, retrain
from tests.muon_reference import step
from tests.scan_reference import forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def pruned(W, block):
    """The dense form of an encoded matrix: of every block of a row the weight of largest magnitude."""
    blocks = W.abs().view(W.shape[0], -1, block)
    return W * torch.zeros_like(blocks).scatter_(2, blocks.argmax(dim=2, keepdim=True), 1.0).view(W.shape)


def near(got, want, what):
    # fp32 sums of at most 400 terms, 2^-24 each: 400 u = 2.4e-5 of the terms, which exceed their sums by some times; the
    # probabilities are off by 2^-16 = 1.5e-5 through lse
    off = float((got.double() - want).norm() / want.norm())
    assert off <= 2e-4, (what, off)


@pytest.mark.parametrize("T,B,F,I,V", [(40, 3, 32, 48, 60), (1, 5, 16, 32, 33), (130, 1, 24, 16, 50)])
def test_one_training_step(T, B, F, I, V):
    gen = torch.Generator(device="cuda").manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    Wg, Wo, X, h0 = rand(2 * F, I) / 4, rand(V, F) / 2, rand(I, T * B), rand(F, B)
    words = torch.randint(V, (T * B,), generator=gen, device="cuda")
    # the tokens of a product lie step after step: a word of each stream in turn; B answers would be strided, so that an
    # answer here is a step's words
    offsets = torch.arange(T + 1, device="cuda") * B
    adv, mask = rand(T), torch.rand(T * B, generator=gen, device="cuda") < 0.9
    gates, out = (darb.darb_encode(W, np.full(W.shape[0], 4, np.int32)) for W in (Wg, Wo))
    try:
        Y = darb.darb_spmm(gates, X)
        gate, x = Y.view(2, F, T, B)
        h, h_last = darb.darb_gated_scan(gate, x, h0, dim=1)
        logits = darb.darb_spmm(out, h.view(F, T * B))
        s = darb.darb_token_logprobs(logits, words, dim=0)
        old = s.logprob + 0.2 * rand(T * B)
        ref = s.logprob + 0.3 * rand(T * B)
        o = darb.darb_policy_loss(s.logprob, old, adv, offsets, ref, s.entropy, mask, kl_coef=0.1, entropy_coef=0.05,
                                  ratio=darb.PER_SEQUENCE, mean=darb.PER_SEQUENCE)
        d_logits = darb.darb_token_logprobs_grad(logits, words, s.lse, o.d_logprob, s.entropy, o.d_entropy, dim=0)
        hv = h.view(F, T * B)
        dWo, dh = d_logits @ hv.t(), (pruned(Wo, 4).t() @ d_logits).view(F, T, B)
        dY = torch.empty_like(Y)
        dg, dx = dY.view(2, F, T, B)
        _, _, d_h0 = darb.darb_gated_scan_grad(dh, gate, x, h, h0, dim=1, d_gate=dg, d_x=dx)
        dWg = dY @ X.t()
    finally:
        darb.darb_destroy(gates), darb.darb_destroy(out)

    # the same in 64 bits; the gradient of the weights goes straight through the pruning
    straight = lambda W: (lambda D: D + (pruned(D, 4) - D).detach())(W)  # noqa: E731
    leaves = [t.double().requires_grad_() for t in (Wg, Wo, h0)]
    g64, x64 = (straight(leaves[0]) @ X.double()).view(2, F, T, B)
    state, states = leaves[2], []
    for t in range(T):
        a = torch.sigmoid(g64[:, t])
        state = a * state + (1 - a) * x64[:, t]
        states.append(state)
    logp = (straight(leaves[1]) @ torch.stack(states, 1).reshape(F, T * B)).log_softmax(0)
    lp, ent = logp.gather(0, words[None])[0], -(logp.exp() * logp).sum(0)
    on = mask.double()
    ids = torch.arange(T, device="cuda").repeat_interleave(B)
    count = torch.zeros(T, dtype=torch.float64, device="cuda").index_add(0, ids, on)
    ratio = torch.zeros(T, dtype=torch.float64, device="cuda").index_add(0, ids, (lp - old.double()) * on) / count.clamp(min=1)
    w = on / (count.clamp(min=1) * (count > 0).sum())[ids]
    r, A, k = ratio.exp()[ids], adv.double()[ids], ref.double() - lp
    loss = (w * (-torch.minimum(r * A, r.clamp(0.8, 1.2) * A) + 0.1 * (k.exp() - 1 - k) - 0.05 * ent)).sum()
    loss.backward()
    assert abs(o.stats[0].item() - loss.item()) <= 2e-5 * max(1.0, abs(loss.item()))
    for got, leaf, what in ((dWg, leaves[0], "gates"), (dWo, leaves[1], "output"), (d_h0, leaves[2], "state")):
        near(got, leaf.grad, what)
    # the carried state and the last one written are two sums for one state, each off by its bound
    arrays = [t.detach().cpu().numpy().transpose(1, 0, 2).reshape(T, F * B) for t in (gate.double(), x.double())]
    bound = forward(*arrays, h0.double().cpu().numpy().reshape(-1), True, True)[1][-1]
    assert (np.abs((h_last - h[:, -1]).double().cpu().numpy().reshape(-1)) <= 2 * bound).all()

    # and both matrices take a step
    p, m = [Wg.clone(), Wo.clone()], [torch.zeros_like(Wg), torch.zeros_like(Wo)]
    copies = [torch.empty_like(t, dtype=torch.bfloat16) for t in p]
    with darb.darb_muon_create(p, m, copies) as plan:
        darb.darb_muon_step(plan, [dWg, dWo], 0.02)
        darb.darb_muon_sync_status(plan)
    for before, after, g, c in zip((Wg, Wo), p, (dWg, dWo), copies):
        want = step(before.double().cpu().numpy(), np.zeros(before.shape), g.double().cpu().numpy(), 0.02)[0]
        # the direction is off by 1.3e-5 of its norm at most (test_gpu_muon.py), the parameter by two roundings
        moved = np.linalg.norm(want - before.double().cpu().numpy() * (1 - 0.02 * 0.01))
        assert np.linalg.norm(after.double().cpu().numpy() - want) <= 1.3e-5 * moved + 2.0 ** -22 * np.linalg.norm(want)
        assert torch.equal(c, after.bfloat16())


def test_the_loop_with_orthogonalised_momentum(monkeypatch):
    """One step of the prune-retrain loop: the weights move by the formula, and what is encoded is what they became."""
    head = retrain.Head(100, 32, 4, states="muon")
    try:
        taken = []
        real = darb.darb_muon_step
        monkeypatch.setattr(darb, "darb_muon_step", lambda plan, grads, *a, **k: (taken.extend(g.clone() for g in grads), real(plan, grads, *a, **k)))
        before, offset = head.W.double().cpu().numpy(), head.beta.clone()
        h, words = retrain.data(64, 100, 32, 0)
        head.train(h, words)
        want = step(before, np.zeros(before.shape), taken[0].double().cpu().numpy(), head.lr)[0]
        moved = np.linalg.norm(want - before * (1 - head.lr * 0.01))
        assert np.linalg.norm(head.W.double().cpu().numpy() - want) <= 1.3e-5 * moved + 2.0 ** -22 * np.linalg.norm(want)
        assert torch.equal(head.stored, head.W.bfloat16()) and not torch.equal(head.beta, offset)
        fresh = darb.darb_encode(head.stored, darb.darb_export(head.handle)[3])
        for a, b in zip(darb.darb_export(head.handle), darb.darb_export(fresh)):
            assert (a == b).all()
        darb.darb_destroy(fresh)
    finally:
        head.close()


def test_the_loop_runs():
    before, after = retrain.retrain(steps=3, vocab=60, features=32, tokens=64, states="muon")
    assert np.isfinite(before) and np.isfinite(after)
