"""Layer norm's gradients of gain and offset over very many tokens whose rows start differently, on the GPU.

The library adds short blocks of tokens first.  With u = 2^-24, blocks of at most 128 tokens, at most N / 4096 /
64 of them after one another in an accumulator and 512 + 64 accumulators after one another in the second
kernel, a sum is off by at most u (N / 2^18 + 704) of the sum of magnitudes.  (One term after the other, N / 64
of them an accumulator, is above that from some 100 000 tokens on.)
"""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,f", [(1 << 20, 5), (3_000_017, 3), (40_000, 300)])
def test_rows_that_start_differently(n, f, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, f, generator=gen, device="cuda").to(dtype)
    # a gradient with a mean: the sums grow, and every addition rounds the same way for long
    dy = torch.full((n, f + 1), 0.7, device="cuda").to(dtype)[:, :f]
    _, mean, rstd = darb.darb_layer_norm(x)
    dx = torch.empty(n, f + 2, dtype=dtype, device="cuda")[:, :f]
    _, dg, db = darb.darb_layer_norm_grad(dy, x, None, mean, rstd, dx=dx)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    d = dy.double()
    bound = U * (n / 2 ** 18 + 704)
    for got, terms in ((db, d), (dg, d * xh)):
        err = (got.double() - terms.sum(0)).abs()
        # (a term of dgamma is rounded three times itself)
        assert bool((err <= (bound + 4 * U) * terms.abs().sum(0)).all()), (err / terms.abs().sum(0) / U).max()
