"""Products with one vector, which is copied at once but for its last three elements at most: every remainder, addresses that
are not aligned, and vectors that do not lie together.  Every weight is kept (blocks of one), so that the product is the
dense one; sums of n terms in fp32 are off by at most n 2^-24 of the terms' sizes, and each product by 2^-24."""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 6, 7, 8, 511, 1025, 1026, 1027, 1028])
def test_every_remainder(cols, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 70
    W = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    handle = darb.darb_encode(W, np.ones(rows, np.int32))
    try:
        for shift in range(4):
            for stride in (1, 2):
                x = torch.full((cols * stride + shift + 4,), float("nan"), device="cuda")[shift:shift + cols * stride:stride]
                x.copy_(torch.randn(cols, generator=gen, device="cuda"))
                got = darb.darb_spmm(handle, torch.as_strided(x, (cols, 1), (stride, 1))).double()
                want, size = W.double() @ x.double()[:, None], W.double().abs() @ x.double().abs()[:, None]
                assert bool(((got - want).abs() <= (cols + 1) * U * size).all()), (shift, stride)
    finally:
        darb.darb_destroy(handle)
