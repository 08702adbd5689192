"""Log probabilities and their gradient of tokens whose logits are large in magnitude, on the GPU.

Every bound is a token's own, from its differences d = x - max, never from the size of its logits or of its
masked entries.  With u = 2^-24, a sum of v terms in chains of at most v / 64 + 64 and an exponential of
relative error 2^-22 give s a relative error of rel = 2^-22 + u (log2 v + v / 64 + 64); a log probability
is off by rel and by four roundings at its own size and that of log2 v; the entropy by (2 + log2 v) rel and as
many roundings.  The gradient is p times differences of these.  Where the gradient uses one fp32 number for
log sum exp, which it may while that is below 512, half a unit in its last place is 2^-16.
"""
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.test_gpu_logprobs import DTYPES, LAYOUTS, U, place, same, stored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def logits(n, v, seed):
    """Tokens of every magnitude, each followed by an ordinary one."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((n, v)).astype(np.float32)
    centres = (-1e9, -3e38, 1e5, -1e5, 1e6, -1e6, 400.0, -600.0, 1000.0, 1e4, -2e4, 2e38, -1e7)
    for i in range(0, n, 2):
        c = centres[i // 2 % len(centres)]
        x[i] = np.float32(c) if abs(c) >= 1e7 else np.float32(c) + x[i]
        if i % 3 == 2:
            x[i, g.random(v) < 0.5] = -np.inf
        if i % 5 == 4:
            x[i, : v // 3] = -1e9 if c > -1e8 else -3.2e38
    return x


def formula(x):
    """(p, log p, entropy, lse) in 64 bits of tokens that each have an entry."""
    m = x.max(axis=1, keepdims=True)
    d = x - m
    s = np.exp(d).sum(axis=1, keepdims=True)
    logp = d - np.log(s)
    p = np.exp(logp)
    logp = np.where(p > 0, logp, 0.0)
    return p, logp, -(p * logp).sum(axis=1), (m + np.log(s))[:, 0]


def rel_s(v):
    return 2.0 ** -22 + U * (math.log2(v) + v / 64 + 64)


def entropy_bound(v):
    return (2 + math.log2(v)) * rel_s(v) + 8 * U * (math.log2(v) + 1)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(53, 600), (27, 5001)])
def test_scores(n, v, dtype, layout):
    t, dim = place(logits(n, v, v), layout, dtype)
    x = stored(t, layout)
    p, logp, h, lse = formula(x)
    targets = p.argmax(axis=1)
    targets[::4] = np.array([np.flatnonzero(q > 0)[-1] for q in p])[::4]
    got = darb.darb_token_logprobs(t, torch.from_numpy(targets).cuda(), 3, dim=dim)
    want = np.take_along_axis(logp, targets[:, None], axis=1)[:, 0]
    size = rel_s(v) + 8 * U * (np.abs(want) + math.log2(v) + 1)
    same(got.logprob.cpu(), want, size)
    same(got.entropy.cpu(), h, entropy_bound(v))
    same(got.lse.cpu(), lse, rel_s(v) + 2 * U * np.abs(lse))
    order = np.argsort(-x, axis=1, kind="stable")[:, :3]
    np.testing.assert_array_equal(got.top_index.cpu().numpy(), order)


def check_grad(n, v, layout, dtype, pad=0, offset=0, out_pad=None, out_offset=0):
    """out_pad None: in place; else a gradient with a leading dimension and a start of its own."""
    x = logits(n, v, n * 7 + v)
    t, dim = place(x, layout, dtype, pad, offset)
    x = stored(t, layout)
    p, logp, h, _ = formula(x)
    g = np.random.default_rng(n)
    targets = p.argmax(axis=1)
    targets[1::3] = g.integers(0, v, n)[1::3]
    targets[5::7] = -1
    a, b = g.standard_normal(n).astype(np.float32), g.standard_normal(n).astype(np.float32)
    tg = torch.from_numpy(targets).cuda()
    fwd = darb.darb_token_logprobs(t, tg, dim=dim)
    out = t if out_pad is None else place(np.zeros_like(x, np.float32), layout, dtype, out_pad, out_offset)[0]
    darb.darb_token_logprobs_grad(t, tg, fwd.lse, torch.from_numpy(a).cuda(), fwd.entropy, torch.from_numpy(b).cuda(), dim=dim, out=out)
    a = np.where(targets < 0, 0.0, a.astype(np.float64))
    want = -p * (a[:, None] + b[:, None] * (logp + h[:, None]))
    given = np.flatnonzero(targets >= 0)
    want[given, targets[given]] += a[given]
    aa, bb = np.abs(a)[:, None], np.abs(b.astype(np.float64))[:, None]
    size = rel_s(v) + 2.0 ** -16 + 8 * U * (np.abs(logp) + math.log2(v) + 1)
    bound = p * ((aa + bb * np.abs(logp + h[:, None])) * size + bb * (size + entropy_bound(v))) + 8 * U * (np.abs(want) + p * (aa + bb * (np.abs(logp) + h[:, None])))
    bound += 2.0 ** -120 + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0.0)
    got = stored(out, layout)
    same(got, want, bound)
    # neither part changes when every logit of a token moves alike
    assert np.all(np.abs(got.sum(axis=1)) <= bound.sum(axis=1))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(1, 700), (26, 700), (53, 130), (64, 700), (30, 5001), (131, 65), (27, 20011)])
def test_gradients(n, v, dtype, layout):
    check_grad(n, v, layout, dtype)                                   # in place
    check_grad(n, v, layout, dtype, pad=n % 2 if layout == "columns" else 3, out_pad=n % 2 if layout == "columns" else 3)
    check_grad(n, v, layout, dtype, pad=2, offset=1, out_pad=5, out_offset=2)   # rows that start differently
