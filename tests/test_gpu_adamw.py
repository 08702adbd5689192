"""AdamW steps over many tensors on the GPU, states in fp32 and in 8 bits.

With fp32 states every operation is one IEEE fp32 operation, so numpy in fp32 has to give the same bits;
the formula in 64 bits bounds the result: seven roundings reach a moment or a parameter's update, so
(8 u) of the sum of the magnitudes of its terms, u = 2^-24.  In 8 bits the update is the same from the
decoded moments, and codes are checked bit for bit against the rounding rule in numpy.
"""
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F = np.float32
SIZES = [1, 0, 255, 256, 257, 4096, 4097, 70001, 8, 33 * 300, 1 << 17]
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def numbers(sizes, seed, offset=0):
    """Parameters, gradients, moments and roots of tensors (numpy), one list each."""
    g = np.random.default_rng(seed)
    got = [[], [], [], []]
    for n in sizes:
        scale = 1e-3 * np.exp(0.7 * g.standard_normal(n))
        for out, a in zip(got, (0.05 * g.standard_normal(n), scale * g.standard_normal(n), 0.3 * scale * g.standard_normal(n),
                                scale * np.exp(0.3 * g.standard_normal(n)))):
            out.append(a.astype(F))
    return got


def put(a, dtype=torch.float32, offset=0):
    """On the GPU, `offset` elements into an allocation."""
    t = torch.zeros(len(a) + offset, dtype=dtype, device="cuda")[offset:]
    t.copy_(torch.from_numpy(np.asarray(a, F)))
    return t


def step32(p, g, m, v, scale, t, lr, beta1, beta2, eps, weight_decay):
    """One step in fp32, operation by operation; returns (p, m, v, root)."""
    with np.errstate(all="ignore"):
        g = g * F(scale)
        m = m * F(beta1) + g * F(1 - beta1)
        v = v * F(beta2) + (g * g) * F(1 - beta2)
        r = np.sqrt(v)
        d = r * F(1 / math.sqrt(1 - beta2 ** t)) + F(eps)
        return p * F(1 - lr * weight_decay) - (m * F(lr / (1 - beta1 ** t))) / d, m, v, r


def noise(first, n, seed):
    z = (np.arange(first, first + n, dtype=np.uint64) * np.uint64(0x9E3779B1) + np.uint64((seed * 0x9E3779B97F4A7C15 & 2 ** 64 - 1) >> 32))
    z = z.astype(np.uint32)
    z = (z ^ z >> np.uint32(15)) * np.uint32(0x6A09E667)
    z = (z ^ z >> np.uint32(13)) * np.uint32(0xBB67AE85)
    z = z ^ z >> np.uint32(16)
    return z >> np.uint32(16), z & np.uint32(0xFFFF)


def quantised(a, z, root):
    """(values of the codes, scales) of one tensor in blocks of 256: the rule in fp32."""
    n = len(a)
    pad = -n % 256
    b = np.pad(a, (0, pad)).reshape(-1, 256)
    with np.errstate(all="ignore"):
        top = np.abs(b).max(axis=1)                       # (NaN if there is one)
        scale = top * F(1 / 448)
        inv = np.where(scale >= np.finfo(F).tiny, F(1) / scale, F(0)).astype(F)
        x = (b * inv[:, None]).reshape(-1)[:n]
        mag = np.abs(x)
        shift = np.where(mag < F(2.0 ** -6), F(2.0 ** -6), F(0))
        bits = ((mag + shift).view(np.uint32) + (z << np.uint32(4)) + np.uint32(8)) & np.uint32(0xFFF00000)
        code = np.minimum(bits.view(F) - shift, F(448))
        code = np.where(np.isnan(mag), mag, code)
        if root:
            code = np.where((a > 0) & (code == 0), F(2.0 ** -9), code)
        return np.copysign(code, x).astype(F), scale.astype(F)


def expand(scale, n):
    return np.repeat(scale, 256)[:n]


@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("copies", [False, True])
def test_fp32_states(copies, offset, grads):
    p, g, m, r = numbers(SIZES, 1)
    gd = torch.float32 if grads == "f32" else torch.bfloat16
    P, G, M, V = [put(a, offset=offset) for a in p], [put(a, gd, offset) for a in g], [put(a, offset=offset) for a in m], [put(a * a, offset=offset) for a in r]
    C = [put(a, torch.bfloat16, offset) for a in p] if copies else None
    scale = torch.tensor(0.25, device="cuda")
    with darb.darb_adamw_create(P, M, V, copies=C, grad_dtype=gd) as plan:
        for t in (1, 7):
            before = [[x.cpu().numpy() for x in xs] for xs in (P, M, V)]
            darb.darb_adamw_step(plan, G, t, grad_scale=scale, **HYPER)
            for i in range(len(SIZES)):
                gi = G[i].float().cpu().numpy()
                want = step32(before[0][i], gi, before[1][i], before[2][i], 0.25, t, **HYPER)
                for got, w in zip((P[i], M[i], V[i]), want):
                    np.testing.assert_array_equal(got.cpu().numpy().view(np.uint32), w.view(np.uint32))
                # and against the formula in 64 bits
                p64, g64, m64, v64 = (a.astype(np.float64) for a in (before[0][i], gi * F(0.25), before[1][i], before[2][i]))
                m1, v1 = 0.9 * m64 + 0.1 * g64, 0.999 * v64 + 0.001 * g64 * g64
                upd = 1e-3 / (1 - 0.9 ** t) * m1 / (np.sqrt(v1 / (1 - 0.999 ** t)) + 1e-8)
                am = 0.9 * np.abs(m64) + 0.1 * np.abs(g64)
                assert np.all(np.abs(M[i].cpu().numpy() - m1) <= 8 * U * am)
                assert np.all(np.abs(V[i].cpu().numpy() - v1) <= 8 * U * v1)
                bound = 8 * U * (np.abs(p64) + np.abs(upd) + np.abs(upd) * am / np.maximum(np.abs(m1), 1e-300))
                assert np.all(np.abs(P[i].cpu().numpy() - (p64 * (1 - 1e-5) - upd)) <= bound)
                if copies:
                    assert torch.equal(C[i], P[i].bfloat16())


@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 5])
def test_states_in_8_bits(offset, grads):
    p, g, m, r = numbers(SIZES, 2)
    r[5][:256] = 0.0          # a block that never had a gradient
    m[5][:256] = 0.0
    g[5][:256] = 0.0
    r[7][300:310] *= 1e-7     # roots far below their block's largest
    g[7][300:310] *= 1e-7
    gd = torch.float32 if grads == "f32" else torch.bfloat16
    E = torch.float8_e4m3fn
    P, G = [put(a, offset=offset) for a in p], [put(a, gd, offset) for a in g]
    M, V, MS, VS = [], [], [], []
    first, starts = 0, []
    for i, n in enumerate(SIZES):
        z = noise(first, n, 5)
        starts.append(first)
        first += -(-n // 256) * 256
        for a, zz, root, codes, scales in ((m[i], z[0], False, M, MS), (r[i], z[1], True, V, VS)):
            c, s = quantised(a, zz, root)
            t = torch.zeros(n + offset, dtype=E, device="cuda")[offset:]
            codes.append(t.copy_(torch.from_numpy(c).to(E)))
            scales.append(put(s, offset=offset))
    C = [put(a, torch.bfloat16) for a in p]
    with darb.darb_adamw_create(P, M, V, MS, VS, copies=C, grad_dtype=gd) as plan:
        for t, seed in ((1, 99), (2, 1 << 63)):
            old = [[x.float().cpu().numpy() for x in xs] for xs in (P, M, V, MS, VS)]
            darb.darb_adamw_step(plan, G, t, seed=seed, **HYPER)
            for i, n in enumerate(SIZES):
                gi = G[i].float().cpu().numpy()
                mi, ri = old[1][i] * expand(old[3][i], n), old[2][i] * expand(old[4][i], n)
                want = step32(old[0][i], gi, mi, ri * ri, 1.0, t, **HYPER)
                np.testing.assert_array_equal(P[i].cpu().numpy(), want[0])
                assert torch.equal(C[i], P[i].bfloat16())
                z = noise(starts[i], n, seed)
                for got, scale, a, zz, root in ((M[i], MS[i], want[1], z[0], False), (V[i], VS[i], want[3], z[1], True)):
                    c, s = quantised(a, zz, root)
                    np.testing.assert_array_equal(scale.cpu().numpy(), s)
                    np.testing.assert_array_equal(got.float().cpu().numpy(), c)
                    # every element is within one code of its value: 2^-3 of it, or 2^-9 of the scale's unit
                    if n and not root:
                        err = np.abs(c.astype(np.float64) * expand(s, n) - a)
                        assert np.all(err <= np.abs(a) * 2.0 ** -3 + expand(s, n) * 2.0 ** -9)
                assert not np.any((want[3] > 0) & (V[i].float().cpu().numpy() == 0))
        darb.darb_adamw_sync_status(plan)   # no wait gave up


def test_rounding_keeps_the_mean():
    """Moments that decay by a thousandth a step: codes follow, which rounding to the nearest would not."""
    n, steps = 1 << 16, 300
    g = np.random.default_rng(3)
    r0 = np.exp(0.5 * g.standard_normal(n)).astype(F)
    E = torch.float8_e4m3fn
    c, s = quantised(r0, noise(0, n, 1)[1], True)
    P, M, V = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda").to(E), torch.from_numpy(c).to(E).cuda()
    MS, VS = torch.zeros(n // 256, device="cuda"), put(s)
    start = (V.float().cpu().numpy() * expand(s, n)).astype(np.float64)
    with darb.darb_adamw_create([P], [M], [V], [MS], [VS]) as plan:
        zero = torch.zeros(n, device="cuda")
        for t in range(1, steps + 1):
            darb.darb_adamw_step(plan, [zero], t, **HYPER)
    now = (V.float().cpu().numpy().astype(np.float64) * expand(VS.cpu().numpy(), n))
    want = start * 0.999 ** (steps / 2)
    # The mean of r is kept by every rounding.  A step's rounding has at most half a code (2^-4 of r) of
    # deviation but moves a code with probability below 1/16 only; over 300 steps and 65536 elements the mean
    # ratio deviates by less than 0.0002 (one sigma); 0.005 is far outside, and far inside the 0.14 of a root that stays.
    assert abs((now / want).mean() - 1) < 0.005
    assert P.eq(0).all() and M.float().eq(0).all()


@pytest.mark.parametrize("codes", [False, True])
def test_gradients_left_out_and_non_finite(codes):
    n = 1000
    E = torch.float8_e4m3fn
    def state():
        P = [torch.ones(n, device="cuda") for _ in range(3)]
        if not codes:
            return P, [torch.zeros(n, device="cuda") for _ in P], [torch.zeros(n, device="cuda") for _ in P], None, None
        return (P, [torch.zeros(n, device="cuda").to(E) for _ in P], [torch.zeros(n, device="cuda").to(E) for _ in P],
                [torch.zeros(4, device="cuda") for _ in P], [torch.zeros(4, device="cuda") for _ in P])
    P, M, V, MS, VS = state()
    g = torch.full((n,), 0.5, device="cuda")
    bad = g.clone()
    bad[300] = float("nan")
    bad[700] = float("inf")
    with darb.darb_adamw_create(P, M, V, MS, VS) as plan:
        darb.darb_adamw_step(plan, [None, bad, g], 1, **HYPER)
        assert P[0].eq(1).all() and M[0].float().eq(0).all()
        hit = torch.zeros(n, dtype=torch.bool, device="cuda")
        hit[[300, 700]] = True
        assert torch.equal(P[1].isfinite(), ~hit)
        assert torch.allclose(P[2], torch.tensor(1 - 1e-5 - 1e-3, device="cuda"), rtol=0, atol=1e-6)
        if codes:   # a block's states share its scale
            assert not MS[1][[1, 2]].isfinite().any() and MS[1][[0, 3]].isfinite().all()


def test_more_tensors_than_one_launch_takes_and_graphs():
    k = 1000
    sizes = [(i * 37) % 700 for i in range(k)]
    p, g, m, r = numbers(sizes, 8)
    P, G, M, V = [put(a) for a in p], [put(a) for a in g], [put(a) for a in m], [put(a * a) for a in r]
    with darb.darb_adamw_create(P, M, V) as plan:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            darb.darb_adamw_step(plan, G, 3, **HYPER)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i in (0, 1, 447, 448, 449, 895, 896, 999):
            want = step32(p[i], g[i], m[i], r[i] * r[i], 1.0, 3, **HYPER)
            np.testing.assert_array_equal(P[i].cpu().numpy(), want[0])
            np.testing.assert_array_equal(V[i].cpu().numpy(), want[2])


def test_the_binding_refuses():
    n = 600
    f = lambda k=n, d=torch.float32: torch.zeros(k, device="cuda").to(d)
    E = torch.float8_e4m3fn
    P, M, V = [f()], [f()], [f()]
    create = darb.darb_adamw_create
    bad = [lambda: create([], [], []), lambda: create(P, M, []), lambda: create([f(d=torch.bfloat16)], M, V), lambda: create(P, [f(599)], V),
           lambda: create(P, M, V, [f(3)]), lambda: create(P, M, V, [f(3)], [f(3)]), lambda: create(P, [f(d=E)], [f(d=E)], [f(2)], [f(3)]),
           lambda: create(P, P, V), lambda: create(P, M, M), lambda: create([f().cpu()], M, V), lambda: create([f(1200)[::2]], M, V),
           lambda: create(P, M, V, copies=[f()]), lambda: create(P, M, V, copies=[P[0].view(torch.bfloat16)[:n]]),
           lambda: create(P, M, V, grad_dtype=torch.float16)]
    plan = create(P, M, V)
    step = lambda g, t=1, **kw: darb.darb_adamw_step(plan, g, t, **dict(HYPER, **kw))
    G = [f()]
    bad += [lambda: step([]), lambda: step([f(599)]), lambda: step([f(d=torch.bfloat16)]), lambda: step(P), lambda: step(M), lambda: step(G, 0),
            lambda: step(G, lr=-1.0), lambda: step(G, lr=float("nan")), lambda: step(G, beta1=1.0), lambda: step(G, beta2=-0.1),
            lambda: step(G, eps=float("inf")), lambda: step(G, weight_decay=-0.1), lambda: step(G, grad_scale=torch.ones(2, device="cuda"))]
    for i, fn in enumerate(bad):
        with pytest.raises(darb.DarbError) as e:
            fn()
        assert e.value.status == darb.ERR_INVALID_ARG, i
    assert P[0].eq(0).all()
    darb.darb_adamw_destroy(plan)
    darb.darb_adamw_destroy(plan)   # nothing left to do
    with pytest.raises(darb.DarbError):
        step(G)


@pytest.mark.parametrize("codes", [False, True])
def test_a_tensor_of_more_elements_than_32_bits_count(codes):
    n = (1 << 31) + 5000
    tail = 1000
    E = torch.float8_e4m3fn
    P = torch.zeros(n, device="cuda")
    G = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    G[-tail:] = torch.randn(tail, device="cuda").bfloat16()
    new = (lambda: torch.zeros(n, dtype=torch.uint8, device="cuda").view(E)) if codes else (lambda: torch.zeros(n, device="cuda"))
    scales = [[torch.zeros(-(-n // 256), device="cuda")] for _ in range(2)] if codes else []
    with darb.darb_adamw_create([P], [new()], [new()], *scales, grad_dtype=torch.bfloat16) as plan:
        darb.darb_adamw_step(plan, [G], 1, **HYPER)
        torch.cuda.synchronize()
        g, z = G[-tail:].float().cpu().numpy(), np.zeros(tail, F)
        np.testing.assert_array_equal(P[-tail:].cpu().numpy(), step32(z, g, z, z, 1.0, 1, **HYPER)[0])
        assert P[:-tail].count_nonzero() == 0
