"""How near X of an orthogonalised update comes, and plans of more matrices than a launch takes gradients.

The bounds are of the scheme itself (muon_scheme.py, all of its sums in 64 bits).  One fp16 number an operand: the kernel's
roundings are the scheme's but where a sum in fp32 falls on the other side of one, so that its error has the same
size; 1.4 times as much is allowed.  Without the diagonals in fp32, or without the rest of X that they multiply, it is
1.7 times as much at least.  Two numbers an operand: what is left is the sums' rounding in fp32, of which only an order of
magnitude is known beforehand; half of the least error that any operand's lost second number makes is allowed."""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests import muon_reference, muon_scheme
from tests.test_gpu_muon import U, limit
from tests.test_muon_scheme import direction

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(64, 6000), (6000, 64), (128, 128), (300, 301), (512, 512)])
def test_nothing_of_an_operand_is_lost(rows, cols, dtype):
    g = torch.from_numpy(direction(rows, cols)).to(dtype).cuda()
    p, m = [torch.zeros(rows, cols, device="cuda")], [torch.zeros(rows, cols, device="cuda")]
    size = 0.2 * max(rows, cols) ** 0.5
    with darb.darb_muon_create(p, m, grad_dtype=dtype) as plan:
        darb.darb_muon_step(plan, [g], 1.0 / size, beta=0.0, weight_decay=0.0)
        darb.darb_muon_sync_status(plan)
    u = g.double().cpu().numpy()
    x = muon_reference.orthogonalise(u)
    error = lambda got: np.linalg.norm(got - x) / np.linalg.norm(x)  # noqa: E731
    numbers = 1 if dtype == torch.bfloat16 else 2
    of = lambda lost: error(muon_scheme.orthogonalise(u, numbers, lost))  # noqa: E731
    worse = min(of(lost) for lost in (muon_scheme.ONE if numbers == 1 else muon_scheme.TWO))
    bound = 1.4 * of(None) if numbers == 1 else worse / 2
    assert worse > 1.2 * bound
    off = error(-p[0].double().cpu().numpy())
    print("error", off, "bound", bound)
    assert off <= bound + 4 * U, (off, bound)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("filled", [1.0, 0.1])
def test_more_matrices_than_a_launch_takes_gradients(filled, dtype):
    """460, some without a gradient, some without elements.  Where most have none, so few tiles are left that several CTAs
    share the depth of the long ones."""
    r = np.random.default_rng(3)
    shapes = [tuple(int(v) for v in r.integers(0, 34, 2) * (r.random() < filled)) for _ in range(456)] + [(64, 6000), (5, 5), (4000, 130), (1, 9000)]
    gen = torch.Generator(device="cuda").manual_seed(9)
    p, m, g = ([torch.randn(s, generator=gen, device="cuda") * scale for s in shapes] for scale in (0.1, 1e-3, 1e-3))
    g = [t.to(dtype) for t in g]
    lr, beta, decay = 0.05, 0.95, 0.1
    kind = "bf16" if dtype == torch.bfloat16 else "f32"
    with darb.darb_muon_create(p, m, grad_dtype=dtype) as plan:
        for turn in range(3):
            none = [i % 7 == turn or (turn == 2 and i >= 440) for i in range(len(shapes))]
            before = [[t.double().cpu().numpy() for t in ts] for ts in (p, m, g)]
            darb.darb_muon_step(plan, [None if skip else t for t, skip in zip(g, none)], lr, beta, decay)
            darb.darb_muon_sync_status(plan)
            for i, (rows, cols) in enumerate(shapes):
                p0, m0, g0 = (b[i] for b in before)
                got_p, got_m = p[i].double().cpu().numpy(), m[i].double().cpu().numpy()
                if none[i] or rows * cols == 0:
                    assert (got_p == p0).all() and (got_m == m0).all(), i
                    continue
                _, want_m, x = muon_reference.step(p0, m0, g0, lr, beta, decay)
                assert (np.abs(got_m - want_m) <= 5 * U * (beta * np.abs(m0) + (1 - beta) * np.abs(g0)) + 2.0 ** -140).all(), i
                size = lr * 0.2 * max(rows, cols) ** 0.5
                off = np.linalg.norm((p0 * (1 - lr * decay) - got_p) / size - x)
                assert off <= limit(kind, rows, cols) * np.linalg.norm(x) + 4 * U * np.linalg.norm(p0) / size, (i, rows, cols)
