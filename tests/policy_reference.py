"""The clipped policy loss and its gradients in 64 bits, with bounds for fp32 arithmetic.

With u = 2^-24: a weight carries two roundings, e^d two units (4 u) and the rounding of d (|d| u), e^x - 1 two
units and e^x |x| u, e^x - 1 - x at most 16 u and 2 |x| u (where it is taken as a difference, |x| >= 1, its terms
are at most 2.4 times as large as it), every product one; the coefficients are rounded to fp32.  Sums go
through at most 13 roundings in 32 bits (8 tokens of a thread, 5 of a warp), then are held in 64.
"""
import numpy as np

U = 2.0 ** -24
TOKEN, SEQUENCE = 0, 1


def sequence_of(n, offsets):
    ids = np.full(n, -1)
    for s in range(len(offsets) - 1):
        ids[offsets[s]:offsets[s + 1]] = s
    return ids


def policy(lp, old, advantage, offsets, ref=None, ent=None, mask=None, low=0.2, high=0.2, kl=0.0, bonus=0.0, ratio=TOKEN, mean=TOKEN):
    """((stats, d_logprob, d_entropy), their bounds, the sequences)."""
    n, count_s = len(lp), len(offsets) - 1
    ids = sequence_of(n, offsets)
    on = (ids >= 0) & (np.ones(n, bool) if mask is None else mask)
    ids0 = np.maximum(ids, 0)
    zero = lambda a: np.where(on, 0.0 if a is None else np.where(on, a, 0.0).astype(np.float64), 0.0)  # noqa: E731
    d = zero(lp) - zero(old)
    count = np.bincount(ids0[on], minlength=max(count_s, 1)).astype(np.float64)
    if ratio == SEQUENCE:
        d = (np.bincount(ids0[on], weights=d[on], minlength=max(count_s, 1)) / np.maximum(count, 1))[ids0]
    if mean == TOKEN:
        w = on / max(count.sum(), 1)
    else:
        w = on / (np.maximum(count, 1) * max((count > 0).sum(), 1))[ids0]
    A = advantage.astype(np.float64)[ids0] if count_s else np.zeros(n)
    with np.errstate(over="ignore", divide="ignore"):
        r = np.exp(d)
        cut = on & np.where(A >= 0, d > np.log1p(high), d < np.log1p(-low))
    used = np.where(cut, np.where(A >= 0, 1 + high, 1 - low), r)
    slope = np.where(cut, 0.0, -A * r)
    x = zero(ref) - zero(lp) if ref is not None else np.zeros(n)
    em1 = np.expm1(x)
    excess = np.where(np.abs(x) < 1e-3, x * x / 2 * (1 + x / 3 * (1 + x / 4 * (1 + x / 5))), em1 - x)
    H = zero(ent)
    terms = [w * -A * used, w * excess, w * H, w * cut]
    sums = [t.sum() for t in terms]
    stats = np.array([sums[0] + kl * sums[1] - bonus * sums[2], *sums])
    d_lp = w * (slope - kl * em1)
    d_ent = np.where(on, -bonus * w, 0.0)
    errs = [np.abs(terms[0]) * (10 + np.abs(d)), np.abs(terms[1]) * (22 + 2 * np.abs(x)), np.abs(terms[2]) * 6, np.abs(terms[3]) * 4]
    e = [U * (t.sum() + 13 * np.abs(v).sum()) for t, v in zip(errs, terms)]
    e_stats = np.array([e[0] + abs(kl) * (e[1] + 2 * U * sums[1]) + abs(bonus) * (e[2] + 2 * U * np.abs(terms[2]).sum()), *e])
    e_stats += 2 * U * np.abs(stats)
    e_lp = U * w * (np.abs(slope) * (12 + np.abs(d)) + abs(kl) * (12 * np.abs(em1) + np.exp(x) * np.abs(x)))
    return (stats, d_lp, d_ent), (e_stats, e_lp, 6 * U * np.abs(d_ent)), ids
