"""Offsets of the policy loss that fall or lie outside of the tokens: results are not defined, but no buffer's
neighbours are written and calls that follow with the same buffers are right."""
import itertools

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
FORMS = list(itertools.product((darb.PER_TOKEN, darb.PER_SEQUENCE), (darb.PER_TOKEN, darb.PER_SEQUENCE)))
FAR = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def guarded(n, dtype):
    """A buffer of n values between 64 others, and the whole of it."""
    whole = torch.full((n + 128,), 77, dtype=dtype, device="cuda")
    return whole[64:64 + n], whole


def offsets_of(kind, n):
    g = np.random.default_rng(n)
    if kind == "falls once":      # the search of the second chunk ends at a sequence that starts behind it
        return [0, n, 100, n]
    if kind == "falls to a start":
        return [0, n - 1, 100, 100, 2048, n]
    if kind == "any order":
        return list(g.integers(0, n + 1, 600))
    if kind == "backwards":
        return sorted((int(v) for v in g.integers(0, n + 1, 40)), reverse=True)
    if kind == "far behind":
        return [0, FAR, 100, n]
    if kind == "far first":
        return [FAR, 0, 4 * n]
    return [-FAR, 30, -1, 2 ** 63 - 1, -2 ** 63, n // 2, n + 1]


@pytest.mark.parametrize("kind", ["falls once", "falls to a start", "any order", "backwards", "far behind", "far first", "far on both sides"])
@pytest.mark.parametrize("n", [700, 4096, 5000, 30011])
def test_offsets_that_fall(n, kind):
    gen = torch.Generator(device="cuda").manual_seed(n)
    offsets = torch.tensor(offsets_of(kind, n), dtype=torch.int64, device="cuda")
    sequences = offsets.numel() - 1
    lp, old, ref, ent = (torch.randn(n, generator=gen, device="cuda") * 0.1 for _ in range(4))
    mask = torch.rand(n, generator=gen, device="cuda") < 0.9
    adv = torch.randn(sequences, generator=gen, device="cuda")
    good = torch.linspace(0, n, sequences + 1, dtype=torch.float64).long().cuda()
    for ratio, mean in FORMS:
        kw = dict(ref_logprob=ref, entropy=ent, mask=mask, kl_coef=0.1, entropy_coef=0.1, ratio=ratio, mean=mean)
        want = darb.darb_policy_loss(lp, old, adv, good, **kw)
        need = darb.darb_policy_loss_work(n)
        (stats, all_stats), (d_lp, all_lp), (d_ent, all_ent) = guarded(5, torch.float32), guarded(n, torch.float32), guarded(n, torch.float32)
        work, all_work = guarded(need, torch.uint8)
        out = darb.PolicyLoss(stats, d_lp, d_ent, work if need else None)
        darb.darb_policy_loss(lp, old, adv, offsets, out=out, **kw)
        for part, whole in ((stats, all_stats), (d_lp, all_lp), (d_ent, all_ent), (work, all_work)):
            assert bool((whole[:64] == 77).all()) and bool((whole[64 + part.numel():] == 77).all())
        d_lp.zero_(), d_ent.zero_()
        darb.darb_policy_loss(lp, old, adv, good, out=out, **kw)
        assert all(torch.equal(a, b) for a, b in zip(out[:3], want[:3]))
