"""The clipped policy loss and its gradients on the GPU, against the formulas in 64 bits (bounds: policy_reference.py)."""
import itertools
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.policy_reference import SEQUENCE, TOKEN, policy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def put(a, shift=0):
    """On the GPU, `shift` elements past an aligned address."""
    if a is None:
        return None
    t = torch.zeros(len(a) + shift, dtype=torch.bool if a.dtype == bool else torch.int64 if a.dtype == np.int64 else torch.float32, device="cuda")
    t[shift:] = torch.from_numpy(np.ascontiguousarray(a))
    return t[shift:]


def lengths(n, sequences, g, lead=0, tail=0):
    """Offsets of ragged sequences, some of them empty."""
    cut = np.sort(g.integers(lead, n - tail + 1, sequences - 1)) if sequences > 1 else np.zeros(0, int)
    return np.concatenate([[lead], cut, [n - tail]]).astype(np.int64)


def values(n, sequences, seed):
    g = np.random.default_rng(seed)
    lp = -np.log(g.random(n).clip(1e-9)) ** 2 * 0.5
    lp, old, ref = ((-np.abs(v)).astype(np.float32) for v in (lp, lp + 0.15 * g.standard_normal(n), lp + 0.4 * g.standard_normal(n)))
    return g, lp, old, ref, g.random(n).astype(np.float32) * 3, g.standard_normal(sequences).astype(np.float32)


def check(lp, old, adv, offsets, ref, ent, mask, kw, shift=0, work=True):
    n = len(lp)
    want, bound, ids = policy(lp, old, adv, offsets, ref, ent, mask, kw["clip_low"], kw["clip_high"], kw["kl_coef"], kw["entropy_coef"], kw["ratio"], kw["mean"])
    out = darb.PolicyLoss.empty(n, "cuda", entropy=ent is not None)
    if shift or not work:
        out = out._replace(d_logprob=torch.empty(n + shift, device="cuda")[shift:], work=out.work if work else None)
    for t in out[:3]:
        if t is not None:
            t.fill_(float("nan"))
    got = darb.darb_policy_loss(put(lp, shift), put(old, shift), put(adv), put(offsets), put(ref, shift), put(ent, shift), put(mask, shift), out=out, **kw)
    assert got is out
    stats = out.stats.double().cpu().numpy()
    assert (np.abs(stats - want[0]) <= bound[0]).all(), (stats, want[0], bound[0])
    for t, w, b in ((out.d_logprob, want[1], bound[1]), (out.d_entropy, want[2], bound[2])):
        if t is None:
            continue
        v = t.double().cpu().numpy()
        assert np.isnan(v[ids < 0]).all()                 # tokens of no sequence are left as they were
        bad = ~(np.abs(v - w) <= b + 2.0 ** -140) & (ids >= 0)
        assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], v[bad][:3], w[bad][:3])
    return out


KW = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, entropy_coef=0.01, ratio=TOKEN, mean=TOKEN)
FORMS = list(itertools.product((TOKEN, SEQUENCE), (TOKEN, SEQUENCE)))
SIZES = [(1, 1), (7, 3), (300, 8), (2048, 2), (4095, 4095), (4096, 1), (4097, 1), (5000, 40), (6144, 3), (30011, 1), (30011, 300), (30011, 29000),
         (200000, 17), (9000, 20000), (100, 70000)]


@pytest.mark.parametrize("ratio,mean", FORMS)
@pytest.mark.parametrize("n,sequences", SIZES)
def test_sizes(n, sequences, ratio, mean):
    g, lp, old, ref, ent, adv = values(n, sequences, n + sequences)
    offsets = lengths(n, sequences, g, lead=min(3, n // 3), tail=min(70, n // 4))
    check(lp, old, adv, offsets, ref, ent, g.random(n) < 0.9, dict(KW, ratio=ratio, mean=mean))


def test_more_chunks_than_a_cta_adds_up():
    """A sequence of more than a million masked tokens among them."""
    n = 2048 * 4100 + 5
    g, lp, old, ref, ent, adv = values(n, 500, 9)
    offsets = lengths(n, 500, g)
    mask = g.random(n) < 0.9
    mask[offsets[100] - 1000000:offsets[100] + 1000000] = False
    for ratio, mean in ((TOKEN, SEQUENCE), (SEQUENCE, TOKEN)):
        check(lp, old, adv, offsets, ref, ent, mask, dict(KW, ratio=ratio, mean=mean))


@pytest.mark.parametrize("ratio,mean", FORMS)
@pytest.mark.parametrize("n", [200, 20000])
@pytest.mark.parametrize("with_ref,with_ent,with_mask", [(False, False, False), (True, False, True), (False, True, False)])
def test_terms_left_out(n, ratio, mean, with_ref, with_ent, with_mask):
    g, lp, old, ref, ent, adv = values(n, 11, n)
    kw = dict(KW, ratio=ratio, mean=mean, kl_coef=0.3 if with_ref else 0.0, entropy_coef=0.2 if with_ent else 0.0)
    check(lp, old, adv, lengths(n, 11, g), ref if with_ref else None, ent if with_ent else None, g.random(n) < 0.5 if with_mask else None, kw)


@pytest.mark.parametrize("shift", [1, 4])
@pytest.mark.parametrize("n", [513, 9999])
def test_addresses(n, shift):
    g, lp, old, ref, ent, adv = values(n, 20, n + shift)
    check(lp, old, adv, lengths(n, 20, g), ref, ent, g.random(n) < 0.9, dict(KW, ratio=SEQUENCE, mean=SEQUENCE), shift=shift)
    check(lp, old, adv, lengths(n, 20, g), ref, ent, g.random(n) < 0.9, KW, shift=shift, work=False)


@pytest.mark.parametrize("ratio,mean", FORMS)
@pytest.mark.parametrize("n", [3000, 40000])
def test_masks_that_leave_nothing(n, ratio, mean):
    """Sequences without a token, whole chunks without one, nothing at all; what stands there is not looked at."""
    g, lp, old, ref, ent, adv = values(n, 6, n)
    offsets = np.array([0, n // 10, n // 10, n // 2, n // 2 + 1, n - 5, n - 5], np.int64)
    mask = g.random(n) < 0.7
    mask[:n // 10] = False                        # all of the first sequence
    mask[n // 10:n // 10 + n // 3] = False        # the first chunks of the third
    mask[n // 2] = False
    for a, bad in ((lp, np.nan), (old, np.inf), (ref, -np.inf), (ent, np.nan)):
        a[~mask] = bad
        a[n - 5:] = bad
    kw = dict(KW, ratio=ratio, mean=mean)
    check(lp, old, adv, offsets, ref, ent, mask, kw)
    out = check(lp, old, adv, offsets, ref, ent, np.zeros(n, bool), kw)
    assert not out.stats.any() and not out.d_logprob[:n - 5].any()
    assert not check(lp, old, adv, np.zeros(7, np.int64), ref, ent, mask, kw).stats.any()


def test_one_token_that_counts_among_many_chunks():
    n = 50000
    g, lp, old, ref, ent, adv = values(n, 3, 5)
    mask = np.zeros(n, bool)
    mask[[49000, 12]] = True
    for ratio, mean in FORMS:
        check(lp, old, adv, np.array([0, 10, 11, n], np.int64), ref, ent, mask, dict(KW, ratio=ratio, mean=mean))


def test_nothing_at_all():
    none = torch.empty(0, device="cuda")
    offsets = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = darb.darb_policy_loss(none, none, none, offsets)
    assert not out.stats.any() and out.d_logprob.numel() == 0
    lp = torch.randn(5, device="cuda")
    out = darb.darb_policy_loss(lp, lp, none, offsets)
    assert not out.stats.any() and not out.d_logprob.any()


def test_borders():
    """Differences that only their exact value tells from a border, on both sides of it."""
    low, high = 0.2, 0.28
    lp, old, sign = [], [], []
    for border, s in ((math.log1p(high), 1.0), (math.log1p(-low), -1.0)):
        near = np.float32(border)
        for o in (0.0, -1e-5, -0.3, -3e-8, 7e-9):
            for k in range(-3, 4):
                v = near + np.float32(o)
                for _ in range(abs(k)):
                    v = np.nextafter(v, np.float32(np.inf if k > 0 else -np.inf))
                lp.append(v), old.append(np.float32(o)), sign.append(s)
    lp, old, adv = (np.array(v, np.float32) for v in (lp, old, sign))
    n = len(lp)
    assert 5 < sum(float(a) - float(b) > math.log1p(high) for a, b in zip(lp, old)) < n - 5
    out = check(lp, old, adv, np.arange(n + 1, dtype=np.int64), None, None, None, dict(KW, kl_coef=0.0, entropy_coef=0.0))
    assert 0.2 < out.stats[4].item() < 0.8


def test_clips_that_are_open_and_extreme_ratios():
    n = 4000
    g, lp, old, ref, ent, adv = values(n, 9, 1)
    old[::7] -= 30
    old[::11] += 60
    ref[::5] -= 20
    offsets = lengths(n, 9, g)
    check(lp, old, adv, offsets, ref, ent, None, dict(KW, clip_low=1.0, clip_high=math.inf))
    check(lp, old, adv, offsets, ref, ent, None, dict(KW, clip_low=0.0, clip_high=0.0))
    # a log probability of -inf now is a ratio of 0
    lp[5] = -np.inf
    out = darb.darb_policy_loss(put(lp), put(old), put(np.abs(adv)), put(offsets))
    assert bool(out.stats.isfinite().all()) and out.d_logprob[5] == 0 and bool(out.d_logprob.isfinite().all())
    # a NaN that counts reaches the loss and its own gradient, of one ratio a sequence its sequence's
    lp[5] = np.nan
    out = darb.darb_policy_loss(put(lp), put(old), put(adv), put(offsets), ratio=SEQUENCE)
    hit = out.d_logprob.isnan().cpu().numpy()
    s = int(np.searchsorted(offsets, 5, side="right")) - 1
    assert hit[offsets[s]:offsets[s + 1]].all() and hit.sum() == offsets[s + 1] - offsets[s] and out.stats[0].isnan()


def test_small_divergences():
    """ref next to logprob: the KL term is the square of a small difference."""
    n = 3000
    g, lp, old, _, ent, adv = values(n, 4, 2)
    ref = lp + (10.0 ** g.uniform(-7, 0, n) * np.sign(g.standard_normal(n))).astype(np.float32)
    check(lp, old, adv, lengths(n, 4, g), ref, ent, None, dict(KW, kl_coef=1.0))


@pytest.mark.parametrize("n", [300, 60000])
def test_graphs_and_streams(n):
    g, lp, old, ref, ent, adv = values(n, 30, n)
    args = [put(v) for v in (lp, old, adv, lengths(n, 30, g), ref, ent, g.random(n) < 0.9)]
    call = lambda out=None: darb.darb_policy_loss(*args, out=out, **dict(KW, ratio=SEQUENCE, mean=SEQUENCE))  # noqa: E731
    want = call()
    assert all(torch.equal(a, b) for a, b in zip(call()[:3], want[:3]))
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for st in streams:
        out = darb.PolicyLoss.empty(n, "cuda", entropy=True)
        out.d_logprob.zero_(), out.d_entropy.zero_()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            call(out)
        graphs.append(gr), outs.append(out)
    for _ in range(3):
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    other = darb.darb_policy_loss(*args, **dict(KW, ratio=SEQUENCE, mean=SEQUENCE), stream=streams[0])
    streams[0].synchronize()
    assert all(torch.equal(a, b) for out in (*outs, other) for a, b in zip(out[:3], want[:3]))


def test_from_logits_to_their_gradient():
    """Scores, loss and gradient in a row, against automatic differentiation in 64 bits."""
    n, v = 500, 300
    gen = torch.Generator(device="cuda").manual_seed(8)
    logits = torch.randn(n, v, generator=gen, device="cuda")
    words = torch.randint(v, (n,), generator=gen, device="cuda")
    offsets = torch.tensor([0, 120, 120, 333, 490], device="cuda")
    adv = torch.tensor([1.0, -1.0, -0.5, 0.7], device="cuda")
    scores = darb.darb_token_logprobs(logits, words)
    old = scores.logprob + 0.2 * torch.randn(n, generator=gen, device="cuda")
    out = darb.darb_policy_loss(scores.logprob, old, adv, offsets, scores.logprob.flip(0).contiguous(), scores.entropy, kl_coef=0.01, entropy_coef=0.02)
    d = darb.darb_token_logprobs_grad(logits, words, scores.lse, out.d_logprob, scores.entropy, out.d_entropy)
    x = logits.double().requires_grad_()
    logp = x.log_softmax(1)
    lp, ent = logp.gather(1, words[:, None])[:, 0], -(logp.exp() * logp).sum(1)
    ids = torch.repeat_interleave(torch.arange(4, device="cuda"), offsets.diff())
    r, a = (lp - old.double())[:490].exp(), adv.double()[ids]
    k = scores.logprob.flip(0).double()[:490] - lp[:490]
    loss = (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.01 * (k.exp() - 1 - k) - 0.02 * ent[:490]).mean()
    loss.backward()
    assert abs(out.stats[0].item() - loss.item()) < 2e-6
    # a probability is off by 2^-16 at most relative to itself through lse, and so are the terms of the gradient
    size = (out.d_logprob.abs() + out.d_entropy.abs() * (1 + scores.entropy + logp.abs().max(1).values)).double()[:, None] * (logp.exp() + (logp == lp[:, None]))
    assert bool(((d.double() - x.grad).abs() <= 2.0 ** -15 * size + 1e-12).all())
    assert not d[490:].any()


def test_refusals():
    lp = torch.zeros(10, device="cuda")
    adv, off = torch.zeros(2, device="cuda"), torch.tensor([0, 4, 10], device="cuda")
    for args, kw in (((lp.double(), lp, adv, off), {}), ((lp, lp[:9], adv, off), {}), ((lp, lp, adv, off[:2]), {}), ((lp, lp, adv, off.int()), {}),
                     ((lp, lp, adv, off), dict(kl_coef=0.1)), ((lp, lp, adv, off), dict(entropy_coef=0.1)), ((lp, lp, adv, off), dict(mask=lp)),
                     ((lp, lp, adv.cpu(), off), {}), ((lp, lp, adv, off), dict(out=darb.PolicyLoss.empty(9))), ((lp, lp, adv, off), dict(clip_low=2.0)),
                     ((lp, lp, adv, off), dict(out=darb.PolicyLoss.empty(10)._replace(d_logprob=lp))),
                     ((lp, lp, adv, off), dict(out=darb.PolicyLoss.empty(10)._replace(stats=None)))):
        with pytest.raises(darb.DarbError):
            darb.darb_policy_loss(*args, **kw)
    big = torch.zeros(5000, device="cuda")
    with pytest.raises(darb.DarbError):
        darb.darb_policy_loss(big, big, adv, off, out=darb.PolicyLoss.empty(5000)._replace(work=torch.zeros(10, device="cuda")))
