"""Layer norm and its backward pass on the GPU, against the formulas in 64 bits.

Bounds, with u = 2^-24 and N features: a sum of N terms in fp32 adds at most C = N / 32 + 64 in a
chain (the kernels use at least 32 threads a token), so the mean is off by at most C u max|x|, a
centred value by twice that, rstd relative to itself by (C + 8) u and twice the error of a centred value
over the standard deviation.
"""
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


def place(x, layout, dtype, pad=0, offset=0):
    """A (steps, tokens, features) array on the GPU: rows (steps must be 1), columns (features x tokens)
    or steps (steps x features x tokens); returns (tensor, dim)."""
    s, n, f = x.shape
    a = x[0] if layout == "rows" else x[0].T if layout == "columns" else x.transpose(0, 2, 1)
    lead = a.shape[:-1]
    width = a.shape[-1] + pad
    flat = torch.full((offset + int(np.prod(lead)) * width,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    t = flat[offset:].view(*lead, width)[..., :a.shape[-1]]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return t, {"rows": -1, "columns": 0, "steps": 1}[layout]


def tokens_of(t, layout):
    """(all tokens, features) in 64 bits."""
    a = t.float().cpu().numpy().astype(np.float64)
    return a if layout == "rows" else a.T if layout == "columns" else a.transpose(0, 2, 1).reshape(-1, a.shape[1])


def close(got, want, bound, what=""):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    err = np.abs(got - want)
    assert np.isfinite(got).all() and np.all(err <= bound), f"{what}: error {err.max()}, {np.max(err / np.maximum(bound, 1e-300))} of the bound"


def vec(a):
    return None if a is None else torch.tensor(np.asarray(a, np.float32), device="cuda")


def run_case(s, n, f, layout, dtype, pad=0, offset=0, shift=0.0, gamma=True, in_place=False, eps=1e-5):
    g = np.random.default_rng(s * 7 + n * 13 + f)
    x = (g.standard_normal((s, n, f)) * (0.5 + g.random((s, n, 1))) + shift).astype(np.float32)
    ga = (1 + 0.3 * g.standard_normal(f)).astype(np.float32) if gamma else None
    be = g.standard_normal(f).astype(np.float32) if gamma else None
    t, dim = place(x, layout, dtype, pad, offset)
    xs = tokens_of(t, layout)
    keep = t.clone() if not in_place else t.contiguous().clone()
    y, mean, rstd = darb.darb_layer_norm(t, vec(ga), vec(be), eps, dim=dim, y=t if in_place else None)
    mu, var = xs.mean(axis=1), xs.var(axis=1)
    rs = 1 / np.sqrt(var + eps)
    G, B = (1.0, 0.0) if ga is None else (ga.astype(np.float64), be.astype(np.float64))
    xh = (xs - mu[:, None]) * rs[:, None]
    chain = f / 32 + 64
    top = np.abs(xs).max(axis=1)
    e_mean = chain * U * top
    close(mean.cpu().numpy().reshape(-1), mu, e_mean, "mean")
    rel = (chain + 8) * U + 2 * (e_mean + 2 * U * top) * rs
    close(rstd.cpu().numpy().reshape(-1), rs, rs * rel, "rstd")
    want = xh * G + B
    bound = (np.abs(xh) * (rel[:, None] + 4 * U) + ((e_mean + 2 * U * top) * rs)[:, None]) * np.abs(G) + 4 * U * (np.abs(want) + np.abs(B))
    bf = 2.0 ** -8 if dtype == "bf16" else 0.0
    close(tokens_of(y, layout), want, bound + bf * (np.abs(want) + bound), "y")
    if not in_place:
        assert torch.equal(t, keep)

    # backward, with what the forward pass wrote
    t.copy_(keep) if in_place else None
    dyv = g.standard_normal((s, n, f)).astype(np.float32)
    d, _ = place(dyv, layout, dtype, pad, offset)
    ds = tokens_of(d, layout)
    dx, dg, db = darb.darb_layer_norm_grad(d, t, vec(ga), mean, rstd, dim=dim, dx=d if in_place else None)
    gg = ds * G
    c0, c1 = gg.mean(axis=1, keepdims=True), (gg * xh).mean(axis=1, keepdims=True)
    want = rs[:, None] * (gg - c0 - xh * c1)
    e_xh = np.abs(xh) * (rel[:, None] + 2 * U) + ((e_mean + 2 * U * top) * rs)[:, None]      # error of xh
    a0, a1 = np.abs(gg).mean(axis=1, keepdims=True), (np.abs(gg) * np.abs(xh)).mean(axis=1, keepdims=True)
    e1 = (np.abs(gg) * e_xh).mean(axis=1, keepdims=True) + (chain + 4) * U * a1
    bound = rs[:, None] * ((chain + 4) * U * a0 + e_xh * np.abs(c1) + (np.abs(xh) + e_xh) * e1
                           + 4 * U * (np.abs(gg) + np.abs(c0) + np.abs(xh * c1))) + np.abs(want) * (rel[:, None] + 4 * U)
    close(tokens_of(dx, layout), want, bound + bf * (np.abs(want) + bound), "dx")
    m = xs.shape[0]
    chain_m = m + 64
    close(dg.cpu(), (ds * xh).sum(axis=0), (np.abs(ds) * e_xh).sum(axis=0) + chain_m * U * (np.abs(ds) * (np.abs(xh) + e_xh)).sum(axis=0) + 1e-30, "dgamma")
    close(db.cpu(), ds.sum(axis=0), chain_m * U * np.abs(ds).sum(axis=0) + 1e-30, "dbeta")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,f", [(1, 1), (1, 2), (3, 7), (5, 64), (17, 100), (9, 255), (40, 513), (8, 1500), (3, 2049), (25, 4096),
                                 (2, 8195), (3, 12288), (1, 20001), (2000, 33), (5000, 4), (700, 1024)])
def test_token_rows(n, f, dtype):
    run_case(1, n, f, "rows", dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("s,n,f", [(1, 1, 1), (1, 20, 1500), (1, 31, 7), (1, 33, 300), (35, 20, 150), (3, 1, 64), (2, 64, 1024), (7, 5, 2),
                                   (1, 300, 40), (64, 3, 33)])
def test_token_columns(s, n, f, dtype):
    if s == 1:
        run_case(s, n, f, "columns", dtype)
    run_case(s, n, f, "steps", dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["rows", "columns", "steps"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (5, 2), (8, 8)])
def test_strides_and_alignments(pad, offset, layout, dtype):
    run_case(3 if layout == "steps" else 1, 21, 203, layout, dtype, pad, offset)


@pytest.mark.parametrize("layout", ["rows", "columns", "steps"])
def test_in_place_without_gain_and_far_from_zero(layout):
    s = 2 if layout == "steps" else 1
    run_case(s, 19, 300, layout, "f32", in_place=True)
    run_case(s, 19, 300, layout, "bf16", in_place=True)
    run_case(s, 19, 300, layout, "f32", gamma=False)
    run_case(s, 19, 300, layout, "f32", shift=100.0)      # the mean is far larger than the spread
    run_case(s, 19, 300, layout, "f32", eps=1.0)


def test_buffers_that_start_differently():
    """Input, output and gradients with alignments of their own."""
    n, f = 11, 130
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(n, f, device="cuda").to(dtype)
        dy = torch.randn(n, f, device="cuda").to(dtype)
        ga = torch.randn(f, device="cuda")
        y0, mean, rstd = darb.darb_layer_norm(x, ga)
        want = darb.darb_layer_norm_grad(dy, x, ga, mean, rstd)
        def moved(t, o, pad):
            b = torch.zeros(o + n * (f + pad), dtype=dtype, device="cuda")[o:].view(n, f + pad)[:, :f]
            return b.copy_(t)
        y = moved(y0 * 0, 3, 5)
        darb.darb_layer_norm(moved(x, 1, 2), ga, y=y)
        tol = 1e-5 if dtype == torch.float32 else 4e-2
        assert torch.allclose(y.float(), y0.float(), rtol=tol, atol=tol)
        got = darb.darb_layer_norm_grad(moved(dy, 2, 1), moved(x, 1, 6), ga, mean, rstd, dx=moved(x, 5, 3))
        for a, b in zip(got, want):
            assert torch.allclose(a.float(), b.float(), rtol=tol, atol=10 * tol)


@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_constant_and_non_finite_tokens(layout):
    x = np.random.default_rng(0).standard_normal((1, 6, 40)).astype(np.float32)
    x[0, 1] = 3.0
    x[0, 2, 5] = np.nan
    x[0, 4, 7] = np.inf
    t, dim = place(x, layout, "f32")
    y, mean, rstd = darb.darb_layer_norm(t, dim=dim)
    got = tokens_of(y, layout)
    assert np.all(got[1] == 0) and np.isnan(got[[2, 4]]).all() and np.isfinite(got[[0, 1, 3, 5]]).all()
    assert abs(float(rstd[1]) - 1e-5 ** -0.5) < 1e-3


@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_gradients_agree_with_differences(layout):
    g = np.random.default_rng(4)
    n, f = 7, 45
    x, ga, be = g.standard_normal((1, n, f)).astype(np.float32), g.standard_normal(f).astype(np.float32), g.standard_normal(f).astype(np.float32)
    w = g.standard_normal((1, n, f)).astype(np.float32)

    def loss(x, ga, be):
        mu, var = x.mean(axis=-1, keepdims=True), x.var(axis=-1, keepdims=True)
        return float((w * ((x - mu) / np.sqrt(var + 1e-5) * ga + be)).sum())

    t, dim = place(x, layout, "f32")
    d, _ = place(w, layout, "f32")
    _, mean, rstd = darb.darb_layer_norm(t, vec(ga), vec(be), dim=dim)
    dx, dg, db = darb.darb_layer_norm_grad(d, t, vec(ga), mean, rstd, dim=dim)
    grads = [tokens_of(dx, layout)[None], dg.double().cpu().numpy(), db.double().cpu().numpy()]
    args, h = [a.astype(np.float64) for a in (x, ga, be)], 1e-4
    for i in range(3):
        step = g.standard_normal(args[i].shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * step, args[i] - h * step
        diff = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(diff - (grads[i] * step).sum()) <= 1e-4 * (1 + np.abs(grads[i] * step).sum())


def test_no_tokens_no_weights_and_repeats():
    f = 37
    x = torch.randn(0, f, device="cuda")
    y, mean, rstd = darb.darb_layer_norm(x)
    assert y.shape == (0, f) and mean.shape == (0,)
    dg, db = torch.ones(f, device="cuda"), torch.ones(f, device="cuda")
    darb.darb_layer_norm_grad(x, x, None, mean, rstd, dgamma=dg, dbeta=db)
    assert dg.eq(0).all() and db.eq(0).all()                       # the sum over no tokens
    x, dy = torch.randn(999, 777, device="cuda"), torch.randn(999, 777, device="cuda")
    y, mean, rstd = darb.darb_layer_norm(x)
    torch.cuda.synchronize()
    a = darb.darb_layer_norm_grad(dy, x, None, mean, rstd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = darb.darb_layer_norm_grad(dy, x, None, mean, rstd, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    need = darb.darb_layer_norm_grad_work(darb.TOKEN_ROWS, 1, 999, 777)
    own = darb.darb_layer_norm_grad(dy, x, None, mean, rstd, work=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(a, own))          # scratch of the caller's, or of the pool
    c = darb.darb_layer_norm_grad(dy, x, None, mean, rstd, weights=False)
    assert torch.equal(c[0], a[0]) and c[1] is None and c[2] is None


def test_the_binding_refuses():
    x = torch.randn(4, 60, device="cuda")
    v = torch.ones(60, device="cuda")
    y, mean, rstd = darb.darb_layer_norm(x, v, v)
    norm, back = darb.darb_layer_norm, darb.darb_layer_norm_grad
    bad = [lambda: norm(x.cpu()), lambda: norm(x.double()), lambda: norm(x, v[:59]), lambda: norm(x, v.bfloat16()),
           lambda: norm(x, eps=-1.0), lambda: norm(x, eps=float("nan")), lambda: norm(x, y=y[:3]), lambda: norm(x[:, ::2]),
           lambda: norm(x[:3], y=x[1:]), lambda: norm(x, mean=x.view(-1)[:4]), lambda: norm(x.view(4, 6, 10), dim=-1),
           lambda: norm(x, y=torch.empty(60, 4, device="cuda").t()), lambda: norm(x, v, y=x.bfloat16()),
           lambda: back(y, x, v, mean, rstd[:3]), lambda: back(y, x, v, None, rstd), lambda: back(y.bfloat16(), x, v, mean, rstd),
           lambda: back(y, x, v, mean, rstd, work=torch.empty(16, dtype=torch.uint8, device="cuda")),
           lambda: back(y, x, v, mean, rstd, dx=x), lambda: back(y, x, v, mean, rstd, dgamma=v)]
    for i, f in enumerate(bad):
        with pytest.raises(darb.DarbError) as e:
            f()
        assert e.value.status == darb.ERR_INVALID_ARG, i


@pytest.mark.parametrize("layout", ["rows", "columns"])
def test_tokens_further_apart_than_32_bits_count(layout):
    n, f = (3, 800) if layout == "rows" else (40, 70)
    ld = (1 << 31) + 24 if layout == "rows" else (1 << 26) + 3
    lines, width = (n, f) if layout == "rows" else (f, n)
    flat = torch.empty((lines - 1) * ld + width, dtype=torch.bfloat16, device="cuda")
    t = flat.as_strided((lines, width), (ld, 1))
    dim = -1 if layout == "rows" else 0
    x = torch.randn(n, f, device="cuda").bfloat16()
    put = x if layout == "rows" else x.t().contiguous()
    ga = torch.randn(f, device="cuda")
    y, mean, rstd = darb.darb_layer_norm(put, ga, dim=dim)
    t.copy_(put)
    _, mean2, rstd2 = darb.darb_layer_norm(t, ga, dim=dim, y=t)
    assert torch.allclose(mean, mean2, rtol=0, atol=1e-6) and torch.allclose(rstd, rstd2, rtol=1e-5)
    assert torch.allclose(t.float(), y.float(), rtol=2.0 ** -7, atol=1e-6)
    dy = torch.randn(lines, width, device="cuda").bfloat16()
    want = darb.darb_layer_norm_grad(dy, put, ga, mean, rstd, dim=dim)
    t.copy_(dy)
    got = darb.darb_layer_norm_grad(t, put, ga, mean, rstd, dim=dim, dx=t)
    for a, b in zip(got, want):
        assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-4)


def test_a_pool_without_room_is_reported(monkeypatch):
    x = torch.randn(64, 256, device="cuda")
    y, mean, rstd = darb.darb_layer_norm(x)
    monkeypatch.setenv("DARB_TEST_POOL_LIMIT", "1000")
    with pytest.raises(darb.DarbError) as e:
        darb.darb_layer_norm_grad(y, x, None, mean, rstd)
    assert e.value.status == darb.ERR_OOM
    darb.darb_layer_norm_grad(y, x, None, mean, rstd, weights=False)   # needs none
    torch.cuda.synchronize()


def test_captured_in_a_graph():
    x, dy = torch.randn(3, 70, 20, device="cuda"), torch.randn(3, 70, 20, device="cuda")
    ga = torch.randn(70, device="cuda")
    want = darb.darb_layer_norm(x, ga, dim=1)
    back = darb.darb_layer_norm_grad(dy, x, ga, want[1], want[2], dim=1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = darb.darb_layer_norm(x, ga, dim=1)
        got_back = darb.darb_layer_norm_grad(dy, x, ga, got[1], got[2], dim=1)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + back, got + got_back))


@pytest.mark.parametrize("strides", [(1, 1, 1), (1, 4, 1), (3, 1, 2), (1, 1, 5), (2, 3, 4)])
def test_one_column_of_wider_matrices(strides):
    f = 150
    a, b, c = (torch.zeros(f, s, device="cuda")[:, :1] for s in strides)
    a.copy_(torch.randn(f, 1, device="cuda"))
    ga = torch.randn(f, device="cuda")
    row = a.t().contiguous()
    y, mean, rstd = darb.darb_layer_norm(row, ga)
    got = darb.darb_layer_norm(a, ga, dim=0, y=b)
    assert torch.allclose(got[0].t(), y, rtol=1e-5, atol=1e-6)
    want = darb.darb_layer_norm_grad(y, row, ga, mean, rstd)
    back = darb.darb_layer_norm_grad(b, a, ga, mean, rstd, dim=0, dx=c)
    assert torch.allclose(back[0].t(), want[0], rtol=1e-4, atol=1e-5)
    assert torch.allclose(back[1], want[1], rtol=1e-4, atol=1e-5) and torch.allclose(back[2], want[2], rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,f,pad", [(3000, 300, 0), (2600, 210, 3), (2500, 515, 1), (1300, 1030, 0)])
def test_many_partial_results(n, f, pad, dtype):
    run_case(1, n, f, "rows", dtype, pad=pad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("s,n,f", [(40, 33, 600), (64, 99, 70), (10, 100, 700), (20, 37, 520), (9, 25, 1100)])
def test_column_tiles_of_every_split(s, n, f, dtype):
    run_case(s, n, f, "steps", dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,f,pad", [(200, 12288, 0), (170, 9001, 0), (330, 8500, 3), (9, 14500, 1), (40, 16000, 0)])
def test_long_rows(n, f, pad, dtype):
    run_case(1, n, f, "rows", dtype, pad=pad)
