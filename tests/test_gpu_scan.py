"""The gated recurrence and its backward pass on the GPU, against the recurrence in 64 bits (bounds: scan_reference.py).

A result in bf16 is off by half a step more, 2^-8 relative to itself.
"""
import numpy as np
import pytest
import torch

from paper_1911_08020_gb300 import darb
from tests.scan_reference import back, forward

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FLOOR = 2.0 ** -118   # what the base-2 exponential flushes to 0, times the tests' largest values


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


class Layout:
    """Values (steps, channels) as a tensor of one of the layouts, and back; channels = outer * inner."""

    def __init__(self, kind, steps, outer, inner, dtype):
        self.kind, self.steps, self.outer, self.inner, self.dtype = kind, steps, outer, inner, DTYPES[dtype]
        self.dim = 0 if kind in ("steps", "slices") else 1

    def place(self, a, pad=0, offset=0):
        t, o, i = self.steps, self.outer, self.inner
        lead = (t, o) if self.dim == 0 else (o, t)
        flat = torch.full((offset + lead[0] * lead[1] * (i + pad),), float("nan"), dtype=self.dtype, device="cuda")
        view = flat[offset:].view(*lead, i + pad)[..., :i]
        if a is not None:
            b = torch.from_numpy(np.ascontiguousarray(a)).view(t, o, i)
            view.copy_(b if self.dim == 0 else b.transpose(0, 1))
        view.flat = flat
        return view

    def read(self, v):
        a = v.float().cpu().numpy().astype(np.float64)
        return (a if self.dim == 0 else a.transpose(1, 0, 2)).reshape(self.steps, -1)

    def state(self, a):
        return torch.tensor(a, dtype=torch.float32, device="cuda").view(self.outer, self.inner)


def inputs(lay, logits, seed=0, pads=(0, 0), offsets=(0, 0)):
    g = np.random.default_rng(seed + lay.steps * 7 + lay.outer * 3 + lay.inner)
    shape = (lay.steps, lay.outer * lay.inner)
    gate = (1.5 * g.standard_normal(shape) + g.uniform(-1, 6, shape[1])).clip(-12, 12)
    if not logits:
        gate = 1 / (1 + np.exp(-gate)) * np.where(g.random(shape) < 0.1, -1, 1)
    return lay.place(gate, pads[0], offsets[0]), lay.place(g.standard_normal(shape), pads[1], offsets[1]), g


def within(got, want, bound, dtype, what):
    bound = bound + FLOOR + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}, {np.max(np.abs(got - want) / bound)} of the bound"


def untouched(view):
    """What lies between and before the elements of a view is what it was."""
    mask = torch.ones_like(view.flat, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool(view.flat[mask].isnan().all())


def both_ways(kind, steps, outer, inner, dtype, logits=True, coupled=True, start=True, pads=(0, 0, 0), offsets=(0, 0, 0), in_place=False):
    lay = Layout(kind, steps, outer, inner, dtype)
    gate, x, g = inputs(lay, logits, 0, pads[:2], offsets[:2])
    channels = outer * inner
    h0 = g.standard_normal(channels).astype(np.float32)
    gates = darb.GATES_LOGITS if logits else darb.GATES_VALUES
    gv, xv = lay.read(gate), lay.read(x)
    first = h0.astype(np.float64) if start else np.zeros(channels)
    want, bound = forward(gv, xv, first, logits, coupled)
    h = x if in_place else lay.place(None, pads[2], offsets[2])
    h0_t = lay.state(h0) if start else None
    last = h0_t if start and in_place else None
    x_keep = x.clone()
    got, h_last = darb.darb_gated_scan(gate, x, h0_t, dim=lay.dim, gates=gates, coupled=coupled, h=h, h_last=last)
    assert got is h and (not start or last is None or h_last is h0_t)
    hv = lay.read(h)
    within(hv, want, bound, lay.dtype, "h")
    within(h_last.cpu().numpy().astype(np.float64).reshape(-1), want[-1], bound[-1], torch.float32, "h_last")
    untouched(h)
    assert in_place or torch.equal(x, x_keep)

    dh_v, d_last_v = g.standard_normal(gv.shape), g.standard_normal(channels).astype(np.float32)
    dh = lay.place(dh_v, pads[0], offsets[2])
    if in_place:
        x = lay.place(xv, pads[1], offsets[1])
        h = lay.place(hv)
    d_last = lay.state(d_last_v)
    wants = back(lay.read(dh), gv, xv, lay.read(h), first, d_last_v.astype(np.float64), logits, coupled)
    d_gate = gate if in_place else lay.place(None, pads[2], offsets[0])
    d_x = x if in_place else lay.place(None, pads[2], offsets[1])
    d_h0 = d_last if in_place else torch.empty_like(d_last)
    darb.darb_gated_scan_grad(dh, gate, x, h, lay.state(h0) if start else None, d_last, dim=lay.dim, gates=gates, coupled=coupled,
                              d_gate=d_gate, d_x=d_x, d_h0=d_h0)
    within(lay.read(d_gate), wants[0], wants[3], lay.dtype, "d_gate")
    within(lay.read(d_x), wants[1], wants[4], lay.dtype, "d_x")
    within(d_h0.cpu().numpy().astype(np.float64).reshape(-1), wants[2], wants[5], torch.float32, "d_h0")
    untouched(d_gate)
    untouched(d_x)


SHAPES = [   # kind, steps, outer, inner
    ("steps", 1, 1, 1), ("steps", 1, 5, 4), ("steps", 2, 3, 20), ("steps", 35, 150, 20), ("steps", 300, 1, 77), ("steps", 4097, 1, 12),
    ("product", 1, 3, 1), ("product", 2, 40, 1), ("product", 127, 33, 1), ("product", 129, 31, 1), ("product", 3000, 17, 1),
    ("product", 500, 21, 2), ("product", 260, 11, 3), ("product", 1029, 9, 5), ("product", 77, 5, 6), ("product", 640, 13, 7),
    ("product", 200, 10, 4), ("product", 200, 4, 8), ("product", 150, 3, 9), ("product", 2500, 5, 33),
    ("rows", 1000, 2, 300), ("rows", 33, 7, 129), ("rows", 600, 1, 4), ("rows", 9, 200, 64),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,steps,outer,inner", SHAPES)
def test_shapes(kind, steps, outer, inner, dtype):
    both_ways(kind, steps, outer, inner, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("logits,coupled,start", [(True, False, True), (False, True, False), (False, False, True), (True, True, False)])
@pytest.mark.parametrize("kind,steps,outer,inner", [("rows", 140, 3, 72), ("product", 300, 6, 3), ("steps", 513, 1, 13)])
def test_forms(kind, steps, outer, inner, dtype, logits, coupled, start):
    both_ways(kind, steps, outer, inner, dtype, logits, coupled, start)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pads,offsets", [((4, 8, 12), (0, 4, 8)), ((3, 0, 1), (1, 2, 3)), ((40, 40, 0), (4, 8, 4))])
@pytest.mark.parametrize("kind,steps,outer,inner", [("rows", 200, 3, 40), ("slices", 60, 5, 24), ("product", 150, 7, 2), ("product", 40, 5, 1)])
def test_strides(kind, steps, outer, inner, dtype, pads, offsets):
    both_ways(kind, steps, outer, inner, dtype, pads=pads, offsets=offsets)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,steps,outer,inner", [("rows", 700, 2, 128), ("product", 900, 5, 1), ("product", 300, 4, 6), ("steps", 35, 40, 20)])
def test_in_place(kind, steps, outer, inner, dtype):
    both_ways(kind, steps, outer, inner, dtype, in_place=True)


@pytest.mark.parametrize("layout", ["rows", "product"])
def test_gates_that_close_and_keep(layout):
    """+-inf are exact gates; a NaN stays in its channel, from its step on."""
    lay = Layout(layout, 400, 8, 1 if layout == "product" else 32, "f32")
    gate, x, g = inputs(lay, True)
    gv = lay.read(gate)
    gv[100, 0], gv[200:, 1], gv[:, 2], gv[150, 3] = -np.inf, np.inf, np.inf, np.nan
    gate.copy_(lay.place(gv))
    h0 = g.standard_normal(gv.shape[1]).astype(np.float32)
    h, last = darb.darb_gated_scan(gate, x, lay.state(h0), dim=lay.dim)
    hv, xv = lay.read(h), lay.read(x)
    assert hv[100, 0] == xv[100, 0]                       # starts anew
    assert (hv[:, 2] == h0[2]).all()
    # From step 199 on the state stays.  Steps are put together in another order for every step, so that its values
    # need not have the same last place; each stands for the same state in 64 bits and is off by at most its bound,
    # so that two of them differ by at most the sum of theirs.
    finite = np.where(np.isinf(gv[:, 1:2]), 40.0, gv[:, 1:2])   # a = 1 in 64 bits as well
    want, bound = forward(finite, xv[:, 1:2], h0[1:2].astype(np.float64), True, True)
    assert np.ptp(want[199:]) < 1e-13 and (np.abs(hv[200:, 1] - hv[199, 1]) <= (bound[200:] + bound[199])[:, 0]).all()
    assert np.isfinite(hv[:150, 3]).all() and np.isnan(hv[150:, 3]).all()
    others = np.delete(hv, 3, axis=1)
    assert np.isfinite(others).all() and np.isfinite(np.delete(last.cpu().numpy().reshape(-1), 3)).all()


def test_no_steps_and_no_channels():
    h0 = torch.randn(6, 5, device="cuda")
    empty = torch.empty(0, 6, 5, device="cuda")
    h, last = darb.darb_gated_scan(empty, empty, h0)
    assert h.shape == empty.shape and torch.equal(last, h0)
    assert not darb.darb_gated_scan(empty, empty)[1].any()
    assert torch.equal(darb.darb_gated_scan_grad(empty, empty, empty, empty, h0, h0.flip(0))[2], h0.flip(0))
    none = torch.empty(9, 0, device="cuda")
    assert darb.darb_gated_scan(none, none)[1].shape == (0,)


@pytest.mark.parametrize("kind,outer,inner", [("rows", 3, 96), ("product", 5, 1), ("steps", 2, 50)])
def test_stretches_are_one_sequence(kind, outer, inner):
    """A sequence cut anywhere, its state carried over in place, is the whole one within the bound of both."""
    steps = 500
    lay = Layout(kind, steps, outer, inner, "f32")
    gate, x, g = inputs(lay, True)
    whole, last = darb.darb_gated_scan(gate, x, None, dim=lay.dim)
    state = torch.zeros(outer, inner, device="cuda")
    parts = []
    for a, b in ((0, 1), (1, 2), (2, 131), (131, 131), (131, 500)):
        cut = [t.narrow(lay.dim, a, b - a) for t in (gate, x)]
        parts.append(darb.darb_gated_scan(*cut, state, dim=lay.dim, h_last=state)[0])
    _, bound = forward(lay.read(gate), lay.read(x), np.zeros(outer * inner), True, True)
    assert (np.abs(lay.read(torch.cat(parts, lay.dim)) - lay.read(whole)) <= 2 * bound).all()
    assert (np.abs((state - last).double().cpu().numpy().reshape(-1)) <= 2 * bound[-1]).all()


def test_on_streams_and_in_graphs():
    """Two captured graphs replayed next to each other, and calls on another stream, give the same bits."""
    lay = Layout("rows", 900, 2, 256, "bf16")
    gate, x, g = inputs(lay, True)
    dh = lay.place(g.standard_normal((900, 512)))
    want = darb.darb_gated_scan(gate, x, dim=1)
    wants = darb.darb_gated_scan_grad(dh, gate, x, want[0], dim=1)
    outs, graphs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for st in streams:
        h, h_last = torch.empty_like(want[0]), torch.empty_like(want[1])
        d = [torch.empty_like(w) for w in wants[:2]]
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr, stream=st):
            darb.darb_gated_scan(gate, x, dim=1, h=h, h_last=h_last)
            darb.darb_gated_scan_grad(dh, gate, x, h, dim=1, d_gate=d[0], d_x=d[1])
        outs.append((h, h_last, *d))
        graphs.append(gr)
    for _ in range(3):
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    for h, h_last, *d in outs:
        assert torch.equal(h, want[0]) and torch.equal(h_last, want[1]) and all(torch.equal(a, b) for a, b in zip(d, wants))
    with torch.cuda.stream(streams[0]):
        h, _ = darb.darb_gated_scan(gate, x, dim=1)
    streams[0].synchronize()
    assert torch.equal(h, want[0])


def test_gates_of_a_pruned_product():
    """The gates and candidates of all steps from one product, and the layer's gradients back through it."""
    F, I, T, B = 48, 64, 130, 3
    gen = torch.Generator(device="cuda").manual_seed(5)
    W = torch.randn(2 * F, I, generator=gen, device="cuda") / 8
    handle = darb.darb_encode(W, np.full(2 * F, 4, np.int32))
    try:
        X = torch.randn(I, T * B, generator=gen, device="cuda")
        Y = darb.darb_spmm(handle, X)
        gate, x = Y.view(2, F, T, B)
        h, _ = darb.darb_gated_scan(gate, x, dim=1)
        arrays = [t.double().cpu().numpy().transpose(1, 0, 2).reshape(T, F * B) for t in (gate, x)]
        want, bound = forward(*arrays, np.zeros(F * B), True, True)
        got = h.double().cpu().numpy().transpose(1, 0, 2).reshape(T, F * B)
        within(got, want, bound, torch.float32, "h")
        dh = torch.randn(h.shape, generator=gen, device="cuda")
        dY = torch.empty_like(Y)
        darb.darb_gated_scan_grad(dh, gate, x, h, dim=1, d_gate=dY.view(2, F, T, B)[0], d_x=dY.view(2, F, T, B)[1])
        wants = back(dh.double().cpu().numpy().transpose(1, 0, 2).reshape(T, F * B), *arrays, got, np.zeros(F * B), np.zeros(F * B), True, True)
        for k in range(2):
            within(dY.view(2, F, T, B)[k].double().cpu().numpy().transpose(1, 0, 2).reshape(T, F * B), wants[k], wants[3 + k], torch.float32, "dY")
    finally:
        darb.darb_destroy(handle)


def test_refusals():
    gate = x = torch.zeros(4, 3, 8, device="cuda")
    bad = [dict(gate=gate[:3]), dict(gate=gate.bfloat16()), dict(h0=torch.zeros(3, 7, device="cuda")), dict(h=torch.empty(4, 3, 9, device="cuda")),
           dict(dim=3), dict(h_last=torch.empty(24, device="cuda", dtype=torch.bfloat16)), dict(gates=2), dict(x=x[None], gate=gate[None], dim=0),
           dict(gate=gate.cpu()), dict(h=gate, gate=gate, x=torch.ones_like(x)), dict(gate=gate[:, :1].expand(4, 3, 8), h0=None)]
    for kw in bad:
        args = dict(dict(gate=gate, x=x), **kw)
        with pytest.raises(darb.DarbError):
            darb.darb_gated_scan(args.pop("gate"), args.pop("x"), args.pop("h0", None), **args)
    with pytest.raises(darb.DarbError):
        darb.darb_gated_scan(torch.zeros(4, 1, 8, device="cuda").expand(4, 3, 8), x.clone())
    with pytest.raises(darb.DarbError):
        darb.darb_gated_scan_grad(x, x, x, x, d_gate=x.clone()[..., :4], d_x=None)
    with pytest.raises(darb.DarbError):
        darb.darb_gated_scan_grad(x, gate, x, x.clone(), d_gate=(d := torch.empty_like(x)), d_x=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,cols", [(0, slice(0, 64)), (0, slice(3, 40)), (1, slice(0, 100)), (1, slice(0, 100, 2))])
def test_offsets_past_32_bits(dim, cols, dtype):
    """Slices of a buffer whose rows lie 2^29 elements apart."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough device memory")
    buf = torch.empty(6, 1 << 29, dtype=DTYPES[dtype], device="cuda")
    parts = [buf[:, 1024 * k:1024 * (k + 1)][:, cols] for k in range(6)]
    gen = torch.Generator(device="cuda").manual_seed(7)
    for t in parts:
        t.copy_(2 * torch.randn(t.shape, generator=gen, device="cuda"))
    gate, x, dh, h, d_gate, d_x = parts
    small = [t.clone() for t in (gate, x, dh)]   # dense, and so by another kernel
    darb.darb_gated_scan(gate, x, dim=dim, h=h)
    darb.darb_gated_scan_grad(dh, gate, x, h, dim=dim, d_gate=d_gate, d_x=d_x)
    a = [t.double().cpu().numpy() if dim == 0 else t.double().cpu().numpy().T for t in (small[0], small[1], small[2], h, d_gate, d_x)]
    zero = np.zeros(a[0].shape[1])
    want, bound = forward(a[0], a[1], zero, True, True)
    within(a[3], want, bound, DTYPES[dtype], "h")
    wants = back(a[2], a[0], a[1], a[3], zero, zero, True, True)
    within(a[4], wants[0], wants[3], DTYPES[dtype], "d_gate")
    within(a[5], wants[1], wants[4], DTYPES[dtype], "d_x")
    assert torch.equal(gate, small[0]) and torch.equal(x, small[1])
    del buf, parts, gate, x, dh, h, d_gate, d_x, t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_one_buffer(dtype):
    """Halves of rows, neighbouring columns, and steps that take turns: no byte is shared, and all are taken."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    fresh = lambda *s: (2 * torch.randn(*s, generator=gen, device="cuda")).to(DTYPES[dtype])  # noqa: E731
    rows, turns, columns = fresh(3, 50, 6 * 8), fresh(5, 90 * 3), fresh(70, 4, 3 * 16)
    for parts, dim in ((rows.split(8, dim=2), 1), ([turns[:, k::3] for k in range(3)], 1), (columns.split(16, dim=2), 0)):
        gate, x, h = parts[:3]
        want = darb.darb_gated_scan(gate.clone(), x.clone(), dim=dim)[0]
        keep = [t.clone() for t in parts]
        darb.darb_gated_scan(gate, x, dim=dim, h=h)
        a = [t.double().cpu().numpy().swapaxes(0, dim).reshape(t.shape[dim], -1) for t in (keep[0], keep[1], h, want)]
        zero = np.zeros(a[0].shape[1])
        ref, bound = forward(a[0], a[1], zero, True, True)
        within(a[2], ref, bound, DTYPES[dtype], "h")
        within(a[3], ref, bound, DTYPES[dtype], "dense h")
        assert all(torch.equal(t, k) for t, k in zip((*parts[:2], *parts[3:]), (*keep[:2], *keep[3:])))


def test_deterministic():
    lay = Layout("product", 5000, 64, 1, "f32")
    gate, x, _ = inputs(lay, True)
    runs = [darb.darb_gated_scan(gate, x, dim=1) for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs for a, b in zip(r, runs[0]))
