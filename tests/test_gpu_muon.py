"""Updates with orthogonalised momentum on the GPU, against the formulas in 64 bits.

What is tested tightly: the momentum (three roundings in fp32: 4 u of its terms, u = 2^-24) and the update's
form.  X goes through 15 products whose errors the iteration passes on; its bounds are of its norm:

* one fp16 number an operand.  X, A' and B' are off by 2^-12 relative to themselves (half a step of 11 bits), of
  random sign, in norm.  With X of singular values s <= 1.2, a step X' = a X + b S X + c S^2 X (S = X X^T): A' off by
  2^-12 |A'|, in B' by (|b| + 2 |c| |A'|) 2^-12 |A'|, and so on.  By the derivative of the iteration, an error e in X
  comes out as at most |a + 3 b s^2 + 5 c s^4| e <= 3.45 e in the directions where s is small and as less than
  2.3 e where it is near 1; five iterations without any cancelling could make 2^-12 * 3.45^4 = 3.5 % of an error of the
  first, but X itself grows by the same 3.45 a step there, so that relative to X an error stays what it was.  Errors of
  five steps, of three products each, of 2^-12 times at most |b| + 2 |c| = 8.8 for the largest of them: 15 * 8.8 *
  2^-12 = 3.2e-2 if all had one sign; of random sign, with sqrt(15) for 15, 8.3e-3.  That is the bound.
* two fp16 numbers an operand: 2^-22 each, and sums of up to N terms in fp32, which are off by at most sqrt(N) 2^-23
  relative to the norms of their terms for random signs: 8.8 sqrt(15) (2^-22 + sqrt(N) 2^-23).
"""
import math

import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.muon_reference import step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def limit(dtype, rows, cols):
    return 8.8 * math.sqrt(15) * (2.0 ** -12 if dtype == "bf16" else 2.0 ** -22 + math.sqrt(max(rows, cols)) * 2.0 ** -23)


def matrices(shapes, dtype, seed=0, shift=0, scale=1e-3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def rand(r, c, t=torch.float32, s=1.0):
        flat = torch.zeros(r * c + shift, dtype=t, device="cuda")
        flat[shift:] = (s * torch.randn(r * c, generator=gen, device="cuda")).to(t)
        return flat[shift:].view(r, c)
    p = [rand(r, c, s=0.1) for r, c in shapes]
    m = [rand(r, c, s=scale) for r, c in shapes]
    g = [rand(r, c, DTYPES[dtype], scale) for r, c in shapes]
    for t in g:   # a few directions that stand out
        if min(t.shape) > 8:
            low = scale * torch.randn(t.shape[0], 4, generator=gen, device="cuda") @ torch.randn(4, t.shape[1], generator=gen, device="cuda")
            t.copy_(t.float() + low)
    return p, m, g


def check(shapes, dtype, lr=0.05, beta=0.95, decay=0.1, nesterov=True, grad_scale=None, shift=0, scale=1e-3, steps=1):
    p, m, g = matrices(shapes, dtype, len(shapes), shift, scale)
    copies = [torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") if i % 2 == 0 else None for i, s in enumerate(shapes)]
    with darb.darb_muon_create(p, m, copies, DTYPES[dtype]) as plan:
        for _ in range(steps):
            before = [[t.double().cpu().numpy() for t in ts] for ts in (p, m, g)]
            gs = None if grad_scale is None else torch.tensor(grad_scale, device="cuda")
            darb.darb_muon_step(plan, g, lr, beta, decay, nesterov=nesterov, grad_scale=gs)
            darb.darb_muon_sync_status(plan)
            for i, (r, c) in enumerate(shapes):
                p0, m0, g0 = (b[i] for b in before)
                s = 1.0 if grad_scale is None else float(np.float32(grad_scale))
                want_p, want_m, x = step(p0, m0, g0, lr, beta, decay, nesterov=nesterov, scale=s)
                err_m = np.abs(m[i].double().cpu().numpy() - want_m)
                assert (err_m <= 5 * U * (beta * np.abs(m0) + (1 - beta) * np.abs(g0 * s)) + 2.0 ** -140).all(), (r, c)
                size = lr * 0.2 * math.sqrt(max(r, c))
                got_x = (p0 * (1 - lr * decay) - p[i].double().cpu().numpy()) / size
                rounding = 4 * U * np.linalg.norm(p0) / size   # of the parameter, in units of X
                off = np.linalg.norm(got_x - x)
                assert off <= limit(dtype, r, c) * np.linalg.norm(x) + rounding, (r, c, off / np.linalg.norm(x), limit(dtype, r, c))
                if copies[i] is not None:
                    assert torch.equal(copies[i], p[i].bfloat16())


SHAPES = [(1, 1), (1, 9), (9, 1), (5, 7), (64, 64), (65, 63), (63, 65), (128, 128), (129, 257), (257, 129), (31, 500), (500, 31), (300, 301),
          (512, 512), (600, 1111), (1111, 600)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, dtype):
    check([(rows, cols)], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_matrices(dtype):
    check([(40, 300), (300, 40), (1, 5), (700, 700), (130, 64), (2, 2), (260, 1000)], dtype, steps=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(64, 6000)], [(5999, 65)], [(1, 30000)], [(200, 4000), (33, 2500), (3000, 130), (7, 7)], [(513, 513)]])
def test_long_products_of_few_tiles(shapes, dtype):
    """Whose depth several CTAs share; twice, as the second step finds what the first one left."""
    check(shapes, dtype, steps=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_enough_for_every_tile_width(dtype):
    check([(2100, 4300), (1700, 1500)], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(beta=0.0), dict(decay=0.0), dict(grad_scale=0.25), dict(shift=1), dict(shift=2),
                                dict(scale=1e-12), dict(scale=1e-30), dict(scale=1e12), dict(scale=1e22), dict(lr=0.0)])
def test_forms(kw, dtype):
    if kw.get("lr") == 0.0:
        p, m, g = matrices([(70, 90)], dtype)
        keep = p[0].clone()
        with darb.darb_muon_create(p, m, grad_dtype=DTYPES[dtype]) as plan:
            darb.darb_muon_step(plan, g, 0.0)
        assert torch.equal(p[0], keep)
        return
    if kw.get("scale") == 1e-30:   # below eps: X is u / (|u| + eps), next to nothing
        p, m, g = matrices([(70, 90)], dtype, scale=1e-30)
        keep = p[0].double()
        with darb.darb_muon_create(p, m, grad_dtype=DTYPES[dtype]) as plan:
            darb.darb_muon_step(plan, g, 0.05, weight_decay=0.0)
        assert bool(((p[0].double() - keep).abs() <= U * keep.abs()).all())
        return
    check([(70, 90), (130, 75)], dtype, **kw)


def test_a_matrix_without_a_gradient_and_zeros():
    p, m, g = matrices([(80, 200), (50, 50), (90, 30)], "f32")
    g[2].zero_(), m[2].zero_()
    keep = [t.clone() for t in (*p, *m)]
    with darb.darb_muon_create(p, m) as plan:
        darb.darb_muon_step(plan, [g[0], None, g[2]], 0.1, weight_decay=0.5)
        darb.darb_muon_step(plan, [None, None, None], 0.1)
        darb.darb_muon_sync_status(plan)
    assert torch.equal(p[1], keep[1]) and torch.equal(m[1], keep[4]) and not torch.equal(p[0], keep[0])
    assert not m[2].any() and bool(((p[2] - keep[2] * 0.95).abs() <= 2 * U * keep[2].abs()).all())   # X = 0: the decay alone


def test_a_nan_stays_in_its_matrix():
    p, m, g = matrices([(80, 200), (50, 60)], "bf16")
    keep = p[0].clone()
    g[0][3, 5] = float("nan")
    with darb.darb_muon_create(p, m, grad_dtype=torch.bfloat16) as plan:
        darb.darb_muon_step(plan, g, 0.1)
        darb.darb_muon_sync_status(plan)
        assert bool(p[0].isnan().all()) and bool(p[1].isfinite().all()) and m[0].isnan().sum() == 1
        # and the plan is not spoilt for gradients to come
        p[0].copy_(keep), m[0].zero_(), g[0].nan_to_num_(0.0)
        darb.darb_muon_step(plan, g, 0.1)
    assert bool(p[0].isfinite().all()) and not torch.equal(p[0], keep)


def test_graphs_streams_and_repeats():
    """The same bits from eager steps, from a captured one that is replayed, and on another stream; two plans at once."""
    shapes = [(300, 520), (520, 200)]
    results = []
    for how in ("eager", "graph", "stream", "two"):
        p, m, g = matrices(shapes, "f32", 3)
        with darb.darb_muon_create(p, m) as plan:
            if how == "graph":
                gr = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(gr):
                    darb.darb_muon_step(plan, g, 0.05)
                for _ in range(3):
                    gr.replay()
                torch.cuda.synchronize()
            elif how == "two":
                p2, m2, g2 = matrices(shapes, "f32", 4)
                other = torch.cuda.Stream()
                torch.cuda.synchronize()
                with darb.darb_muon_create(p2, m2) as second:
                    for _ in range(3):
                        darb.darb_muon_step(plan, g, 0.05)
                        darb.darb_muon_step(second, g2, 0.05, stream=other)
                    torch.cuda.synchronize()
            else:
                st = torch.cuda.Stream() if how == "stream" else torch.cuda.current_stream()
                torch.cuda.synchronize()
                for _ in range(3):
                    darb.darb_muon_step(plan, g, 0.05, stream=st)
                torch.cuda.synchronize()
            darb.darb_muon_sync_status(plan)
        results.append((*p, *m))
    assert all(torch.equal(a, b) for r in results[1:] for a, b in zip(r, results[0]))


def test_refusals():
    p, m, g = matrices([(8, 6), (5, 5)], "f32")
    for bad in (dict(params=p, m=m[:1]), dict(params=p, m=[m[0], m[1].bfloat16()]), dict(params=p, m=[m[0].t(), m[1]]), dict(params=p, m=p),
                dict(params=[t.view(-1) for t in p], m=[t.view(-1) for t in m]), dict(params=p, m=m, copies=[None]),
                dict(params=p, m=m, copies=[p[0], None]), dict(params=p, m=m, grad_dtype=torch.float16), dict(params=[], m=[])):
        with pytest.raises(darb.DarbError):
            darb.darb_muon_create(**bad)
    with darb.darb_muon_create(p, m) as plan:
        for grads in ([g[0]], [g[0], g[1].bfloat16()], [g[0].t(), g[1]], [p[0], g[1]], [g[0], m[0].view(-1)[:25].view(5, 5)]):
            with pytest.raises(darb.DarbError):
                darb.darb_muon_step(plan, grads, 0.1)
        with pytest.raises(darb.DarbError):
            darb.darb_muon_step(plan, g, -0.1)
        with pytest.raises(darb.DarbError):
            darb.darb_muon_step(plan, g, 0.1, grad_scale=p[0].view(-1)[:1])
