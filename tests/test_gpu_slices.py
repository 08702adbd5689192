"""Inputs and outputs that are slices of one wider buffer: they share no element, and the calls take them."""
import pytest
import torch

from paper_1911_08020_gb300 import darb

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def halves(n, f, count, dtype, gap=0):
    """`count` tensors n x f side by side in one buffer (gap: elements between them), random."""
    b = torch.randn(n, count * (f + gap), device="cuda").to(DTYPES[dtype])
    return b, [b[:, i * (f + gap):i * (f + gap) + f] for i in range(count)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [-1, 0])
@pytest.mark.parametrize("n,f,gap", [(33, 512, 0), (40, 203, 0), (9, 60, 5), (1, 77, 0), (300, 8, 0), (5, 3000, 1)])
def test_side_by_side(n, f, gap, dim, dtype):
    close = dict(rtol=1e-5, atol=1e-5) if dtype == "f32" else dict(rtol=2.0 ** -7, atol=2.0 ** -9)
    buffer, (x, dy, y, dx) = halves(n, f, 4, dtype, gap)
    kept, tokens, features = buffer.clone(), x.shape[1 + dim if dim else 1], x.shape[dim]
    gamma = torch.randn(features, device="cuda")
    want = darb.darb_layer_norm(x.contiguous(), gamma, dim=dim)
    back = darb.darb_layer_norm_grad(dy.contiguous(), x.contiguous(), gamma, want[1], want[2], dim=dim)
    got = darb.darb_layer_norm(x, gamma, dim=dim, y=y)
    got_back = darb.darb_layer_norm_grad(dy, x, gamma, got[1], got[2], dim=dim, dx=dx)
    for a, b in zip(got + got_back, want + back):
        assert torch.allclose(a.float(), b.float(), **close)
    targets = torch.arange(tokens, device="cuda") % features
    scores = darb.darb_token_logprobs(x, targets, dim=dim)
    d = torch.ones(tokens, device="cuda")
    plain = darb.darb_token_logprobs_grad(x.contiguous(), targets, scores.lse, d, dim=dim)
    assert torch.allclose(darb.darb_token_logprobs_grad(x, targets, scores.lse, d, dim=dim, out=y).float(), plain.float(), **close)
    # the inputs and what lies between the slices are as they were
    assert torch.equal(x, kept[:, :f]) and torch.equal(dy, kept[:, f + gap:2 * f + gap])
    if gap:
        assert all(torch.equal(buffer[:, i * (f + gap) + f:(i + 1) * (f + gap)], kept[:, i * (f + gap) + f:(i + 1) * (f + gap)]) for i in range(4))


def test_steps_side_by_side():
    s, f, n = 3, 50, 20
    b = torch.randn(s, f, 2 * n, device="cuda")
    x, y = b[:, :, :n], b[:, :, n:]
    want = darb.darb_layer_norm(x.contiguous(), dim=1)
    got = darb.darb_layer_norm(x, dim=1, y=y)
    assert all(torch.allclose(p, q, rtol=1e-5, atol=1e-5) for p, q in zip(got, want))


def test_slices_that_share_elements_are_refused():
    b = torch.randn(16, 400, device="cuda")
    x = b[:, :200]
    _, mean, rstd = darb.darb_layer_norm(x.contiguous())
    targets = torch.zeros(16, dtype=torch.int64, device="cuda")
    lse = darb.darb_token_logprobs(x, targets).lse
    flat = b.view(-1)
    wraps = flat[399 + 1 - 100:][:14 * 400 + 200].as_strided((15, 200), (400, 1))   # past a row's end into the next one's start
    other = flat.as_strided((16, 200), (399, 1), 200)                               # another leading dimension
    for shared, like in ((b[:, 199:399], x), (b[:, 100:300], x), (b[1:, :200], x[:15]), (wraps, x[:15]), (other, x)):
        k = like.shape[0]
        for call in (lambda: darb.darb_layer_norm(like, y=shared),
                     lambda: darb.darb_layer_norm_grad(like, b[:k, 200:], None, mean[:k], rstd[:k], dx=shared, weights=False),
                     lambda: darb.darb_token_logprobs_grad(like, targets[:k], lse[:k], lse[:k].clone(), out=shared)):
            with pytest.raises(darb.DarbError) as e:
                call()
            assert e.value.status == darb.ERR_INVALID_ARG
    with pytest.raises(darb.DarbError):
        darb.darb_layer_norm(x, mean=b[0, 190:206])   # a vector that starts among a row's features
    mean2 = b[3, 220:236]                              # one between them
    darb.darb_layer_norm(x, mean=mean2)
    assert torch.allclose(mean2, mean, rtol=0, atol=1e-6)
