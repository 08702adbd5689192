"""Log probabilities of given tokens, entropy and best alternatives, and their gradient, on the GPU.

The reference computes in 64 bits from the stored logits (fp32 or bf16).  Bounds, with u = 2^-24:
the kernels form e_v = 2^(x_v log2 e - r) with one rounding of the exponent (relative error of e_v
at most ln 2 * u * |d_v|, and e_v |d_v| sums to at most log2(vocab) s) and an instruction of relative
error 2^-22, and add at most vocab / 256 + 64 of them in a chain, so
  rel(s) <= 2^-22 + u (log2 vocab + vocab / 256 + 64),
log2 s and the final sums round once each at the size of their operands.
"""
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def rel_s(v):
    return 2.0 ** -22 + U * (math.log2(v) + v / 256 + 64)


def place(x, layout, dtype, pad=0, offset=0):
    """A (tokens, vocab) array on the GPU in a layout, with a leading dimension larger by `pad`, starting
    `offset` elements into its allocation; returns (tensor, dim)."""
    n, v = x.shape
    a = x if layout == "rows" else x.T
    r, c = a.shape
    flat = torch.full((offset + r * (c + pad),), float("nan"), dtype=DTYPES[dtype], device="cuda")
    t = flat[offset:].view(r, c + pad)[:, :c]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return t, (-1 if layout == "rows" else 0)


def stored(t, layout):
    """The stored logits as (tokens, vocab) in 64 bits."""
    a = t.float().cpu().numpy().astype(np.float64)
    return a if layout == "rows" else a.T


def reference(x, targets, k):
    """(logprob, entropy, lse, top_logprob, top_index) in 64 bits of finite or masked (-inf) logits."""
    n, v = x.shape
    m = x.max(axis=1)
    empty = m == -np.inf
    m0 = np.where(empty, 0.0, m)[:, None]
    e = np.exp(x - m0)
    s = e.sum(axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = m0[:, 0] + np.log(s)
        ent = np.where(empty, 0.0, np.log(s) - np.where(e > 0, e * np.where(e > 0, x - m0, 0.0), 0.0).sum(axis=1) / s)
        logp = np.where(empty[:, None], -np.inf, x - lse[:, None])
    lp = np.array([0.0 if t < 0 else np.nan if t >= v else logp[i, t] for i, t in enumerate(targets)])
    order = np.argsort(-x, axis=1, kind="stable")[:, :k]
    return lp, ent, lse, np.take_along_axis(logp, order, axis=1), order


def same(got, want, bound):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.where(fine, 0.0, got), np.where(fine, 0.0, want))
    err = np.abs(got[fine] - want[fine])
    bound = np.broadcast_to(bound, want.shape)[fine]
    assert np.all(err <= bound), f"error {err.max()} above {bound[np.argmax(err - bound)]}"


def check(x, layout, dtype, targets, k, pad=0, offset=0):
    t, dim = place(x, layout, dtype, pad, offset)
    xs = stored(t, layout)
    n, v = xs.shape
    tg = torch.tensor(targets, dtype=torch.int64, device="cuda")
    got = darb.darb_token_logprobs(t, tg, k, dim=dim)
    lp, ent, lse, top, idx = reference(xs, targets, k)
    big = np.abs(np.where(np.isfinite(xs), xs, 0.0)).max(axis=1)
    size = rel_s(v) + 4 * U * (1.45 * big + math.log2(v) + 1)
    same(got.lse.cpu(), lse, size)
    same(got.logprob.cpu(), lp, size)
    same(got.entropy.cpu(), ent, (2 + math.log2(v)) * rel_s(v) + 4 * U * (math.log2(v) + 1))
    if k:
        np.testing.assert_array_equal(got.top_index.cpu().numpy(), idx)
        # a wider spread of logits below the maximum: relative to the value as well
        fine = np.where(np.isfinite(top), np.abs(top), 0.0)
        same(got.top_logprob.cpu(), top, size[:, None] + 4 * U * fine)
    return t, tg, got


LAYOUTS = ("rows", "columns")
SIZES = [(1, 1), (1, 7), (3, 31), (2, 33), (5, 1000), (33, 257), (20, 10000), (1, 32000), (9, 4099), (2, 131072), (70, 513),
         (300, 129)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", SIZES)
def test_scores_match_the_reference(n, v, dtype, layout):
    g = np.random.default_rng(n * 1000 + v)
    x = 3.0 * g.standard_normal((n, v)).astype(np.float32)
    targets = g.integers(0, v, n)
    targets[g.random(n) < 0.2] = -1
    for k in sorted({0, 1, min(5, v), min(32, v)}):
        check(x, layout, dtype, targets, k)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (5, 3), (8, 8)])
def test_strides_and_alignments(pad, offset, dtype, layout):
    g = np.random.default_rng(pad * 10 + offset)
    x = g.standard_normal((13, 1037)).astype(np.float32)
    check(x, layout, dtype, g.integers(0, 1037, 13), 7, pad, offset)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", [50, 5000, 40000])
def test_masks(v, dtype, layout):
    g = np.random.default_rng(v)
    x = 2.0 * g.standard_normal((9, v)).astype(np.float32)
    x[0] = -np.inf                                       # nothing left
    x[1, g.random(v) < 0.95] = -np.inf                   # most masked
    x[2] = -np.inf
    x[2, [3, v - 1]] = [0.5, 0.25]                       # fewer entries than alternatives
    x[3, : v // 2] = -1e9                                # a large negative mask before the entries
    x[4, v // 2:] = float(np.finfo(np.float32).min)      # (-inf in bf16)
    x[5] = -1e9                                          # all entries masked so: uniform
    x[5, 1] = -1e9
    x[6] = -3.0e38                                       # near the type's lowest
    x[7] = -10000.0
    x[8, 1:] = -np.inf                                   # one entry
    targets = np.array([1, 0, 3, v - 1, 0, 2, 4, 5, 0])
    for k in (0, 3, 20):
        check(x, layout, dtype, targets, k)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("scale", [1e4, 3e4, 1e6, 1e30, 2e38])
def test_large_logits(scale, layout):
    """Far past what the fast path's reference holds: sums of plain differences."""
    g = np.random.default_rng(3)
    x = (scale * (1 + 1e-6 * g.standard_normal((4, 600)))).astype(np.float32)
    x[1] = -x[1]
    x[2, ::2] = -x[2, ::2]
    t, dim = place(x, layout, "f32")
    got = darb.darb_token_logprobs(t, torch.zeros(4, dtype=torch.int64, device="cuda"), 5, dim=dim)
    d = x.astype(np.float64) - x.max(axis=1, keepdims=True)
    s = np.exp(d).sum(axis=1)
    # differences are exact, or rounded once; the fast path (up to 2^14) rounds at the size of the logits
    size = rel_s(600) + 4 * U * (np.abs(d).max() if scale > 2 ** 14 else 1.45 * scale + np.abs(d).max())
    size = np.minimum(size, 1e300)
    with np.errstate(over="ignore"):   # a log probability past the range of fp32 is -inf
        want = (d[:, 0] - np.log(s)).astype(np.float32)
    same(got.logprob.cpu(), want, size)
    same(got.lse.cpu(), x.max(axis=1).astype(np.float64) + np.log(s), size + 8 * U * scale)
    np.testing.assert_array_equal(got.top_index.cpu().numpy(), np.argsort(-x, axis=1, kind="stable")[:, :5])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("v", [40, 9000])
def test_nan_and_infinity_stay_in_their_token(v, layout):
    g = np.random.default_rng(5)
    x = g.standard_normal((6, v)).astype(np.float32)
    x[1, 17] = np.nan
    x[3, 5] = np.inf
    x[4, 9] = -np.inf
    t, dim = place(x, layout, "f32")
    got = darb.darb_token_logprobs(t, torch.full((6,), 3, dtype=torch.int64, device="cuda"), 2, dim=dim)
    for o in (got.logprob, got.entropy, got.lse):
        np.testing.assert_array_equal(np.isnan(o.cpu().numpy()), [False, True, False, True, False, False])
    top = got.top_index.cpu().numpy()
    assert top[1, 0] == 17 and top[3, 0] == 5   # NaN counts as the largest
    rest = np.where(np.isnan(x[1]), -np.inf, x[1])
    assert top[1, 1] == rest.argmax()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_go_to_the_lowest_index(dtype, layout):
    v = 20000
    g = np.random.default_rng(6)
    x = np.zeros((6, v), np.float32)                             # all equal
    x[1] = g.integers(0, 3, v)                                    # three values
    x[2] = np.where(g.random(v) < 0.5, 0.0, -0.0)                 # the two zeros tie
    x[3] = np.sort(g.standard_normal(v))                          # ascending, descending: the largest lie together
    x[4] = x[3][::-1]
    x[5, :600] = 1.0
    check(x, layout, dtype, np.zeros(6, np.int64), 32)
    check(x, layout, dtype, np.full(6, v - 1), 1)


def test_targets_outside_and_outputs_left_out():
    x = torch.randn(4, 100, device="cuda")
    tg = torch.tensor([-1, -5, 100, 1 << 40], device="cuda")
    got = darb.darb_token_logprobs(x, tg)
    assert got.logprob[:2].eq(0).all() and got.logprob[2:].isnan().all()
    none = darb.darb_token_logprobs(x)                            # no targets: no log probability
    assert none.logprob is None and torch.equal(none.entropy, got.entropy)
    only = darb.TokenLogprobs(None, None, torch.empty(4, device="cuda"), None, None)
    assert torch.equal(darb.darb_token_logprobs(x, out=only).lse, got.lse)
    zero = darb.darb_token_logprobs(x[:0], tg[:0], 3)
    assert zero.logprob.shape == (0,) and zero.top_index.shape == (0, 3)


def test_views_of_either_axis_and_one_column():
    x = torch.randn(50, 333, device="cuda")
    tg = torch.randint(0, 333, (50,), device="cuda")
    want = darb.darb_token_logprobs(x, tg, 4)
    y = x.t().contiguous()                                        # vocab x tokens
    for got in (darb.darb_token_logprobs(y, tg, 4, dim=0), darb.darb_token_logprobs(y.t(), tg, 4)):
        assert torch.equal(got.top_index, want.top_index)
        assert torch.allclose(got.logprob, want.logprob, rtol=0, atol=1e-5)
    col = darb.darb_token_logprobs(y[:, 7:8], tg[7:8], 4, dim=0)  # features a leading dimension apart
    assert torch.equal(col.top_index, want.top_index[7:8])


def test_calls_repeat_bit_for_bit_on_any_stream():
    x = torch.randn(64, 50001, device="cuda").bfloat16()
    tg = torch.randint(0, 50001, (64,), device="cuda")
    a = darb.darb_token_logprobs(x, tg, 10)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = darb.darb_token_logprobs(x, tg, 10)
    c = darb.darb_token_logprobs(x, tg, 10, stream=s)
    d = darb.darb_token_logprobs(x, tg, 10, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for o in (b, c, d):
        assert all(torch.equal(p, q) for p, q in zip(a, o))


# ---- the gradient ----

def grad_reference(x, targets, a, b):
    """In 64 bits."""
    n, v = x.shape
    m = x.max(axis=1, keepdims=True)
    empty = m[:, 0] == -np.inf
    e = np.exp(x - np.where(m == -np.inf, 0.0, m))
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(empty[:, None], 0.0, e / e.sum(axis=1, keepdims=True))
        logp = np.where(p > 0, np.log(np.where(p > 0, p, 1.0)), 0.0)
    h = -(p * logp).sum(axis=1)
    g = -(np.where(targets < 0, 0.0, a) * ~empty)[:, None] * p - b[:, None] * p * (logp + h[:, None])
    for i, t in enumerate(targets):
        if t >= 0 and not empty[i]:
            g[i, t] += a[i]
    return g, p, logp, h


def grad_check(x, layout, dtype, targets, a, b, pad=0, offset=0, in_place=False):
    t, dim = place(x, layout, dtype, pad, offset)
    xs = stored(t, layout)
    n, v = xs.shape
    tg = torch.tensor(targets, dtype=torch.int64, device="cuda")
    fwd = darb.darb_token_logprobs(t, tg, dim=dim)
    da = torch.tensor(a, dtype=torch.float32, device="cuda")
    db = torch.tensor(b, dtype=torch.float32, device="cuda")
    got = darb.darb_token_logprobs_grad(t, tg, fwd.lse, da, fwd.entropy, db, dim=dim, out=t if in_place else None)
    assert (got.data_ptr() == t.data_ptr()) == in_place
    want, p, logp, h = grad_reference(xs, targets, da.double().cpu().numpy(), db.double().cpu().numpy())
    # p has the error of lse and of x - lse, at most `size`, and that of the exponential
    big = np.abs(np.where(np.isfinite(xs), xs, 0.0)).max(axis=1)[:, None]
    size = 2 * rel_s(v) + 8 * U * (1.45 * big + math.log2(v) + np.abs(logp))
    aa, bb = np.abs(a)[:, None], np.abs(b)[:, None]
    bound = (aa + bb * (np.abs(logp) + h[:, None])) * p * size + bb * p * (2 + math.log2(v)) * size + 4 * U * (aa * (p > 0) + np.abs(want))
    # below the smallest normal number there is nothing left of a gradient
    bound = bound + 2.0 ** -120 + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0.0)
    same(stored(got, layout), want, bound)
    return got


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(1, 1), (2, 9), (33, 64), (20, 10000), (7, 4099), (1, 40001), (130, 65)])
def test_gradients_match_the_formula(n, v, dtype, layout):
    g = np.random.default_rng(n + v)
    x = 2.0 * g.standard_normal((n, v)).astype(np.float32)
    targets = g.integers(0, v, n)
    targets[g.random(n) < 0.2] = -1
    a, b = g.standard_normal(n).astype(np.float32), g.standard_normal(n).astype(np.float32)
    grad_check(x, layout, dtype, targets, a, b)
    grad_check(x, layout, dtype, targets, a, 0 * b, in_place=True)
    grad_check(x, layout, dtype, targets, 0 * a, b, pad=3, offset=1)
    grad_check(x, layout, dtype, targets, a, b, pad=8, offset=5, in_place=True)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_gradients_of_masked_tokens(layout):
    g = np.random.default_rng(8)
    x = g.standard_normal((5, 700)).astype(np.float32)
    x[0] = -np.inf                       # no gradient at all
    x[1, 3:] = -np.inf
    x[2, ::2] = -1e9
    x[3] = -1e9
    targets = np.array([4, 1, 5, 6, -1])
    got = grad_check(x, layout, "f32", targets, np.ones(5, np.float32), np.full(5, 0.3, np.float32))
    assert stored(got, layout)[0].any() == False  # noqa: E712


def test_gradients_agree_with_differences():
    g = np.random.default_rng(9)
    n, v = 6, 400
    x = g.standard_normal((n, v)).astype(np.float32)
    targets = g.integers(0, v, n)
    a, b = g.standard_normal(n), g.standard_normal(n)
    f = lambda y: (lambda r: float(a @ r[0] + b @ r[1]))(reference(y, targets, 0))
    t = torch.from_numpy(x).cuda()
    tg = torch.from_numpy(targets).cuda()
    fwd = darb.darb_token_logprobs(t, tg)
    grad = darb.darb_token_logprobs_grad(t, tg, fwd.lse, torch.tensor(a, dtype=torch.float32, device="cuda"), fwd.entropy,
                                         torch.tensor(b, dtype=torch.float32, device="cuda")).double().cpu().numpy()
    x64, h = x.astype(np.float64), 1e-4
    for trial in range(5):
        step = g.standard_normal((n, v))
        step[trial, targets[trial]] += 10.0
        diff = (f(x64 + h * step) - f(x64 - h * step)) / (2 * h)
        # third derivatives are O(1): differences are off by h^2, the gradient by fp32 rounding
        assert abs(diff - (grad * step).sum()) <= 1e-5 * (1 + np.abs(grad * step).sum())


def test_gradients_of_absent_parts():
    x = torch.randn(3, 50, device="cuda")
    tg = torch.tensor([1, -1, 50], device="cuda")
    fwd = darb.darb_token_logprobs(x, tg)
    d = torch.ones(3, device="cuda")
    g = darb.darb_token_logprobs_grad(x, tg, fwd.lse, d)
    assert g[0].isfinite().all() and g[1].eq(0).all() and g[2].isnan().all()
    e = darb.darb_token_logprobs_grad(x, None, fwd.lse, None, fwd.entropy, d)
    # the entropy does not change when every logit moves alike
    assert e.isfinite().all() and torch.all(e.sum(dim=1).abs() < 1e-5)
    z = darb.darb_token_logprobs_grad(x[:0], tg[:0], fwd.lse[:0], d[:0])
    assert z.shape == (0, 50)


def test_the_binding_refuses():
    x = torch.randn(4, 60, device="cuda")
    tg = torch.zeros(4, dtype=torch.int64, device="cuda")
    fwd = darb.darb_token_logprobs(x, tg)
    call = darb.darb_token_logprobs
    bad = [lambda: call(x.cpu(), tg), lambda: call(x.half(), tg), lambda: call(x, tg.int()), lambda: call(x, tg[:3]),
           lambda: call(x, tg, 33), lambda: call(x, tg, -1), lambda: call(x[:, ::2], tg, 0, 0), lambda: call(x.view(2, 2, 60), tg),
           lambda: call(x, tg, dim=2), lambda: call(x[:, :5], tg, 6), lambda: call(x[:, :1].expand(4, 60), tg),
           lambda: call(x, tg, out=fwd._replace(lse=fwd.entropy)),
           lambda: call(x, tg, out=fwd._replace(lse=x.view(-1)[:4])),
           lambda: darb.darb_token_logprobs_grad(x, None, fwd.lse, fwd.lse),
           lambda: darb.darb_token_logprobs_grad(x, tg, fwd.lse, fwd.entropy, None, fwd.entropy),
           lambda: darb.darb_token_logprobs_grad(x, tg, None, fwd.entropy),
           lambda: darb.darb_token_logprobs_grad(x, tg, fwd.lse, fwd.entropy, out=x[:, :59]),
           lambda: darb.darb_token_logprobs_grad(x, tg, fwd.lse, fwd.entropy, out=x.view(-1)[:240].view(60, 4).t()),
           lambda: darb.darb_token_logprobs_grad(x[:3], tg[:3], fwd.lse[:3], fwd.entropy[:3], out=x[1:])]
    for i, f in enumerate(bad):
        with pytest.raises(darb.DarbError) as e:
            f()
        assert e.value.status == darb.ERR_INVALID_ARG, i


@pytest.mark.parametrize("layout", LAYOUTS)
def test_logits_further_apart_than_32_bits_count(layout):
    """Rows (or entries) whose offsets in elements and in bytes pass 2^32."""
    n, v = (3, 1000) if layout == "rows" else (40, 70)
    ld = (1 << 31) + 24 if layout == "rows" else (1 << 26) + 3
    lines, width = (n, v) if layout == "rows" else (v, n)
    flat = torch.empty((lines - 1) * ld + width, dtype=torch.bfloat16, device="cuda")
    t = flat.as_strided((lines, width), (ld, 1))
    x = torch.from_numpy(np.random.default_rng(1).standard_normal((n, v)).astype(np.float32)).cuda().bfloat16()
    t.copy_(x if layout == "rows" else x.t())
    dim = -1 if layout == "rows" else 0
    tg = torch.arange(n, device="cuda")
    want, got = darb.darb_token_logprobs(x, tg, 5), darb.darb_token_logprobs(t, tg, 5, dim=dim)
    assert torch.equal(got.top_index, want.top_index)
    assert torch.allclose(got.logprob, want.logprob, rtol=0, atol=1e-5) and torch.allclose(got.entropy, want.entropy, rtol=0, atol=1e-4)
    d = torch.ones(n, device="cuda")
    a = darb.darb_token_logprobs_grad(x, tg, want.lse, d)
    b = darb.darb_token_logprobs_grad(t, tg, want.lse, d, dim=dim, out=t)
    assert torch.allclose(a.float(), (b if layout == "rows" else b.t()).float(), rtol=2.0 ** -7, atol=1e-7)


@pytest.mark.parametrize("strides", [(1, 1), (1, 4), (3, 1), (5, 2)])
def test_one_column_of_wider_matrices(strides):
    """One token: dense features here, features a leading dimension apart there."""
    v = 300
    a, b = (torch.zeros(v, s, device="cuda")[:, :1] for s in strides)
    a.copy_(torch.randn(v, 1, device="cuda"))
    tg, d = torch.tensor([7], device="cuda"), torch.ones(1, device="cuda")
    row = a.t().contiguous()
    fwd = darb.darb_token_logprobs(a, tg, 3, dim=0)
    want = darb.darb_token_logprobs(row, tg, 3)
    assert torch.equal(fwd.top_index, want.top_index) and torch.allclose(fwd.logprob, want.logprob, rtol=0, atol=1e-5)
    got = darb.darb_token_logprobs_grad(a, tg, want.lse, d, dim=0, out=b)
    assert got.data_ptr() == b.data_ptr()
    assert torch.allclose(got.t(), darb.darb_token_logprobs_grad(row, tg, want.lse, d), rtol=1e-5, atol=1e-7)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,v", [(400, 1001), (160, 2100), (1300, 4200), (2500, 600), (320, 13000), (620, 7001), (4, 120001),
                                 (155, 60000)])
def test_scores_of_every_split(n, v, dtype, layout):
    """Few and many threads a token, one CTA and several."""
    g = np.random.default_rng(n + v)
    x = 3.0 * g.standard_normal((n, v)).astype(np.float32)
    x[g.random((n, v)) < 0.1] = -np.inf
    targets = g.integers(0, v, n)
    for k in (0, 6):
        check(x, layout, dtype, targets, k)
