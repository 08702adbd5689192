"""Gradients and gradient scales that lie in a buffer which the step writes are refused."""
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
E = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def carve(sizes):
    """One allocation of bytes in pieces at multiples of 16, so that what reaches past a piece stays in it."""
    total = sum(-(-s // 16) * 16 for s in sizes) + 65536
    flat, at, got = torch.zeros(total, dtype=torch.uint8, device="cuda"), 0, []
    for s in sizes:
        got.append((at, s))
        at += -(-s // 16) * 16
    return flat, got


@pytest.mark.parametrize("codes", [False, True])
def test_refusals(codes):
    n = (600, 5000, 40)
    per = lambda f: [f(k) for k in n]
    state, blocks = (1 if codes else 4), (lambda k: -(-k // 256) * 4)
    sizes = per(lambda k: 4 * k) + per(lambda k: state * k) * 2 + (per(blocks) * 2 if codes else []) + per(lambda k: 2 * k)
    flat, at = carve(sizes)
    view = lambda i, dtype: flat[at[i][0]:at[i][0] + at[i][1]].view(dtype)
    kind = E if codes else torch.float32
    P, M, V = ([view(3 * j + i, torch.float32 if j == 0 else kind) for i in range(3)] for j in range(3))
    scales = [[view(3 * j + i, torch.float32) for i in range(3)] for j in (3, 4)] if codes else []
    last = 5 if codes else 3
    C = [view(3 * last + i, torch.bfloat16) for i in range(3)]
    G = [torch.ones(k, device="cuda") for k in n]
    with darb.darb_adamw_create(P, M, V, *scales, copies=C) as plan:
        def step(grads=None, **kw):
            darb.darb_adamw_step(plan, G if grads is None else grads, 1, 1e-3, **kw)

        def refused(*a, **kw):
            with pytest.raises(darb.DarbError) as e:
                step(*a, **kw)
            assert e.value.status == darb.ERR_INVALID_ARG
        for start, size in at:
            # gradients of tensor 2 (160 bytes) and of tensor 1, over the first, a middle and the last word of every buffer
            for word in {start // 4, (start + size // 2) // 4, (start + size - 1) // 4}:
                inside = flat[4 * word:].view(torch.uint8)[:160].view(torch.float32)
                refused([G[0], G[1], inside])
                refused([None, None, inside])
                refused(grad_scale=flat[4 * word:4 * word + 4].view(torch.float32))
        refused([G[0], flat[:20000].view(torch.float32), G[2]])
        assert flat.eq(0).all()
        step(grad_scale=G[0][:1])            # (in a gradient: both are only read)
        step([None, None, G[2]])
        darb.darb_adamw_sync_status(plan)
        torch.cuda.synchronize()
        assert all(bool(p.ne(0).all()) for p in P)
