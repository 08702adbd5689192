"""A recurrent layer, a policy loss and an orthogonalised update around pruned layers, as measurable cases.

What a model whose layers are pruned and trained again needs beside ``perf/operators.py``: a recurrence
over whole sequences whose gates are one product of all steps, and its backward pass; the loss of answers
that the model drew itself, with the gradients that ``darb_token_logprobs_grad`` takes; and the update of
weight matrices whose momentum is orthogonalised.  Four kinds of pass:

* ``scan``    a gated linear recurrence over steps (``darb_gated_scan``);
* ``back``    its backward pass (``darb_gated_scan_grad``);
* ``policy``  the clipped policy loss with a KL term, and its gradients (``darb_policy_loss``);
* ``muon``    one step over all matrices of a model (``darb_muon_step``).

Activations lie as the sequence calls write them (``steps``: steps x features x batch), as one product over
all steps leaves them (``product``: features x (steps x batch), gates and candidates below each other), or
as token rows (``rows``: batch x steps x features, gates and candidates side by side).
"""
import math

import torch

own = False

LR, BETA, DECAY, NS_EPS = 2e-4, 0.95, 0.01, 1e-7   # a rate for training that starts from trained weights
NS = (3.4445, -4.7750, 2.0315)   # the coefficients of an iteration, five iterations
CLIP_LOW, CLIP_HIGH, KL, BONUS = 0.2, 0.28, 0.05, 0.01


def listed():
    return [
        # One step of the language model's layer at batch 20: serving, the state goes in and comes out.
        {"name": "scan_step", "kind": "scan", "layout": "steps", "dtype": "f32", "steps": 1, "features": 1500, "batch": 20, "gates": "logits", "coupled": True, "start": True},
        # 35 steps of it, one stretch of training text.
        {"name": "scan_lm", "kind": "scan", "layout": "steps", "dtype": "f32", "steps": 35, "features": 1500, "batch": 20, "gates": "logits", "coupled": True, "start": True},
        # One long stream, the gates of all steps from one product: time is the contiguous axis, and odd.
        {"name": "scan_stream", "kind": "scan", "layout": "product", "dtype": "f32", "steps": 20011, "features": 1024, "batch": 1, "gates": "logits", "coupled": True, "start": False},
        # Long documents as token rows, few of them: time has to be split to fill the GPU.
        {"name": "scan_documents", "kind": "scan", "layout": "rows", "dtype": "bf16", "steps": 16384, "features": 2048, "batch": 4, "gates": "logits", "coupled": True, "start": False},
        # Backward through the stretch of the language model.
        {"name": "back_lm", "kind": "back", "layout": "steps", "dtype": "f32", "steps": 35, "features": 1500, "batch": 20, "gates": "logits", "coupled": True, "start": True},
        # Backward through the documents.
        {"name": "back_documents", "kind": "back", "layout": "rows", "dtype": "bf16", "steps": 16384, "features": 2048, "batch": 4, "gates": "logits", "coupled": True, "start": False},
        # A handful of short answers: latency is all there is.
        {"name": "policy_few", "kind": "policy", "tokens": 300, "sequences": 8, "ratio": "tokens", "mean": "tokens", "kl": True, "bonus": True},
        # A batch of long answers of ragged lengths, each answer counting the same.
        {"name": "policy_batch", "kind": "policy", "tokens": 1500000, "sequences": 1000, "ratio": "tokens", "mean": "sequences", "kl": True, "bonus": True},
        # The same with one ratio for each answer.
        {"name": "policy_answers", "kind": "policy", "tokens": 400000, "sequences": 512, "ratio": "sequences", "mean": "sequences", "kl": True, "bonus": False},
        # The gates of a few small recurrent layers, tall and odd.
        {"name": "muon_small", "kind": "muon", "grads": "f32", "layers": 3, "rows": 600, "cols": 301, "more_rows": 128, "more_cols": 500},
        # Two fully-connected layers, bf16 gradients, and the bf16 weights that are encoded next.
        {"name": "muon_fc", "kind": "muon", "grads": "bf16", "layers": 1, "rows": 4096, "cols": 9216, "more_rows": 4096, "more_cols": 4096},
        # The gate matrices of the language model's two layers and a projection, fp32 gradients.
        {"name": "muon_lm", "kind": "muon", "grads": "f32", "layers": 2, "rows": 6000, "cols": 3000, "more_rows": 1500, "more_cols": 1500},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("scan", "scan", "scan", "back", "back", "policy", "policy", "muon", "muon"))
    if kind == "muon":
        case = {"kind": kind, "grads": rng.choice(("f32", "bf16")), "layers": rng.randint(1, 3),
                "rows": _spread(rng, 64, 6000), "cols": _spread(rng, 64, 6000),
                "more_rows": _spread(rng, 64, 4096), "more_cols": _spread(rng, 64, 4096)}
        while _products(case) > 2.5e12:
            case["rows"], case["cols"] = case["rows"] * 4 // 5, case["cols"] * 4 // 5
        return case
    if kind == "policy":
        tokens = _spread(rng, 100, 1500000)
        return {"kind": kind, "tokens": tokens, "sequences": _spread(rng, 1, min(tokens, 4000)),
                "ratio": rng.choice(("tokens", "tokens", "sequences")), "mean": rng.choice(("tokens", "sequences")),
                "kl": rng.random() < 0.7, "bonus": rng.random() < 0.5}
    case = {"kind": kind, "layout": rng.choice(("steps", "product", "rows")), "dtype": rng.choice(("f32", "bf16")),
            "steps": _spread(rng, 1, 32768), "features": _spread(rng, 16, 4096)}
    case["batch"] = _spread(rng, 1, max(1, min(256, 120_000_000 // (case["steps"] * case["features"]))))
    while case["steps"] * case["features"] * case["batch"] > 120_000_000:
        case["steps"] //= 2
    case["gates"] = rng.choice(("logits", "logits", "values"))
    case["coupled"] = rng.random() < 0.7
    case["start"] = rng.random() < 0.5
    return case


def _products(case):
    """Multiply-adds twice over, of five iterations: X X^T and its square are symmetric, half of each is enough."""
    total = 0
    for rows, cols in _sizes(case):
        n, m = min(rows, cols), max(rows, cols)
        total += 5 * (n * n * m + n ** 3 + 2 * n * n * m)
    return total


def _sizes(case):
    return [(case["rows"], case["cols"])] * case["layers"] + [(case["more_rows"], case["more_cols"])]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _dim(case):
    """The axis of the steps."""
    return 0 if case["layout"] == "steps" else 1


def _activations(case, gen, count):
    """`count` tensors of N(0, 1) in the case's layout, the parts of one product's result where it is a product's."""
    t, f, b = case["steps"], case["features"], case["batch"]
    dtype = _dtype(case["dtype"])
    if case["layout"] == "steps":
        return [torch.randn(t, f, b, generator=gen, device="cuda").to(dtype) for _ in range(count)]
    if case["layout"] == "product":
        return list(torch.randn(count * f, t * b, generator=gen, device="cuda").to(dtype).view(count, f, t, b))
    return list(torch.randn(b, t, count * f, generator=gen, device="cuda").to(dtype).split(f, dim=2))


def _state_shape(case):
    return {"steps": (case["features"], case["batch"]), "product": (case["features"], case["batch"]),
            "rows": (case["batch"], case["features"])}[case["layout"]]


class _State:
    """What a program has in hand before a call."""

    def __init__(self, case, seed):
        self.case = case
        getattr(self, "_" + case["kind"])(case, _generator(seed))

    def _scan(self, case, gen):
        self.gate, self.x = _activations(case, gen, 2)
        f = case["features"]
        # biases of the gates: features that forget at once beside features that remember for a thousand steps
        bias = torch.rand(f, generator=gen, device="cuda") * 7.0 - 1.0
        bias = bias.view({"steps": (1, f, 1), "product": (f, 1, 1), "rows": (1, 1, f)}[case["layout"]])
        self.gate.copy_(self.gate.float() + bias)
        if case["gates"] == "values":
            self.gate.copy_(torch.sigmoid(self.gate.float()))
        self.h0 = torch.randn(_state_shape(case), generator=gen, device="cuda") if case["start"] else None
        # buffers that a program keeps from step to step
        self.h = torch.empty(self.x.shape, dtype=self.x.dtype, device="cuda")
        self.h_last = torch.empty(_state_shape(case), device="cuda")

    def _back(self, case, gen):
        self._scan(case, gen)
        h = _plain_scan(self)[0]   # the forward pass has left its states
        self.h.copy_(h)
        self.dh = _activations(case, gen, 1)[0]
        self.d_last = torch.randn(_state_shape(case), generator=gen, device="cuda")
        self.d_h0 = torch.empty(_state_shape(case), device="cuda") if case["start"] else None
        # the parts of one buffer, as the backward pass of the product takes them
        self.d_gate, self.d_x = _activations(case, gen, 2)

    def _policy(self, case, gen):
        n, s = case["tokens"], case["sequences"]
        # answers of ragged lengths, a few of them empty, with some padding behind the last
        cut = torch.rand(s, generator=gen, device="cuda").square() + 0.02
        cut[torch.rand(s, generator=gen, device="cuda") < 0.02] = 0.0
        ends = (torch.cumsum(cut.double(), 0) / cut.double().sum().clamp(min=1e-9) * (n - n // 50)).long()
        self.offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), ends])
        self.logprob = -torch.rand(n, generator=gen, device="cuda").log().square() * 0.7
        self.old = self.logprob + 0.12 * torch.randn(n, generator=gen, device="cuda")
        self.ref = self.logprob + 0.2 * torch.randn(n, generator=gen, device="cuda") if case["kl"] else None
        self.entropy = 2.0 * torch.rand(n, generator=gen, device="cuda") if case["bonus"] else None
        self.advantage = torch.randn(s, generator=gen, device="cuda")
        self.mask = torch.rand(n, generator=gen, device="cuda") < 0.93   # tool output, truncated answers
        self.out = None
        if own:
            from paper_1911_08020_gb300 import darb
            self.out = darb.PolicyLoss.empty(n, "cuda", entropy=case["bonus"])
            # tokens behind the last sequence are left as they were
            self.out.d_logprob.zero_()
            if case["bonus"]:
                self.out.d_entropy.zero_()

    def _muon(self, case, gen):
        self.p, self.m, self.g, self.copies = [], [], [], []
        for rows, cols in _sizes(case):
            # gradients have rows and columns of different sizes, and a few directions that stand out
            size = torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device="cuda")) * torch.exp(0.5 * torch.randn(1, cols, generator=gen, device="cuda"))
            some = torch.randn(rows, 8, generator=gen, device="cuda") @ torch.randn(8, cols, generator=gen, device="cuda")
            self.p.append(0.05 * torch.randn(rows, cols, generator=gen, device="cuda"))
            self.g.append((1e-3 * (size * torch.randn(rows, cols, generator=gen, device="cuda") + 0.3 * some)).to(_dtype(case["grads"])))
            self.m.append(2e-4 * (size * torch.randn(rows, cols, generator=gen, device="cuda") + some))
            self.copies.append(self.p[-1].to(torch.bfloat16))
        self.grad_scale = torch.full((), 0.5, device="cuda")   # what clipping by the gradients' norm gives
        if own:
            from paper_1911_08020_gb300 import darb
            self.plan = darb.darb_muon_create(self.p, self.m, copies=self.copies, grad_dtype=_dtype(case["grads"]))


def prepare(case, seed):
    return _State(case, seed)


def _gates(s, gate, x):
    """(a, 1 - a, a's derivative, what enters the state) in the precision of the arguments."""
    if s.case["gates"] == "logits":
        a, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
        slope = a * rest
    else:
        a, rest, slope = gate, 1.0 - gate, torch.ones_like(gate)
    return a, rest, slope, rest * x if s.case["coupled"] else x


def _doubling(a, u):
    """Along the first axis, h_t = a_t h_(t-1) + u_t with nothing before: after k rounds an element stands for 2^k steps."""
    a, h, shift = a.clone(), u, 1
    while shift < h.shape[0]:
        h = torch.cat([h[:shift], torch.addcmul(h[shift:], a[shift:], h[:-shift])])
        a[shift:] = a[shift:] * a[:-shift]
        shift *= 2
    return h


def _plain_scan(s):
    dim = _dim(s.case)
    a, _, _, u = _gates(s, s.gate.float().movedim(dim, 0), s.x.float().movedim(dim, 0))
    if s.h0 is not None:
        u = torch.cat([u[:1] + a[:1] * s.h0, u[1:]])
    h = _doubling(a, u)
    return h.movedim(0, dim).to(s.x.dtype), h[-1].clone()


def _plain_back(s):
    dim = _dim(s.case)
    gate, x, h, dh = (t.float().movedim(dim, 0) for t in (s.gate, s.x, s.h, s.dh))
    a, rest, slope, _ = _gates(s, gate, x)
    start = torch.zeros_like(h[0]) if s.h0 is None else s.h0
    before = torch.cat([start.unsqueeze(0), h[:-1]])
    # what flows to a step from the next one: from the last step backwards
    dh = torch.cat([dh[:-1], dh[-1:] + s.d_last])
    last_first = torch.cat([a[1:], torch.zeros_like(a[:1])]).flip(0)
    g = _doubling(last_first, dh.flip(0)).flip(0)
    d_gate = g * slope * (before - x if s.case["coupled"] else before)
    d_x = g * rest if s.case["coupled"] else g
    got = {"d_gate": d_gate.movedim(0, dim).to(s.x.dtype), "d_x": d_x.movedim(0, dim).to(s.x.dtype)}
    if s.h0 is not None:
        got["d_h0"] = a[0] * g[0]
    return got


def _sums(t, ids, parts):
    """Sums of a token vector over its sequences, in 64 bits."""
    return torch.zeros(parts, dtype=torch.float64, device=t.device).index_add_(0, ids, t.double())


def _plain_policy(s):
    case, n, parts = s.case, s.case["tokens"], s.case["sequences"]
    at = torch.arange(n, device="cuda")
    ids = torch.searchsorted(s.offsets, at, right=True) - 1     # of empty sequences with one start, the last
    inside = at < s.offsets[-1]
    ids = ids.clamp(0, parts - 1)
    on = s.mask & inside
    count = _sums(on, ids, parts)
    delta = torch.where(on, s.logprob.double() - s.old.double(), 0.0)   # 64 bits: next to a border they decide
    if case["ratio"] == "sequences":
        delta = (_sums(delta, ids, parts) / count.clamp(min=1))[ids]
    if case["mean"] == "tokens":
        weight = torch.where(on, 1.0 / count.sum().clamp(min=1), 0.0)
    else:
        weight = torch.where(on, 1.0 / ((count > 0).sum().clamp(min=1) * count.clamp(min=1))[ids], 0.0)
    weight = weight.float()
    a = s.advantage[ids]
    ratio = torch.exp(delta.float())
    low, high = math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)
    cut = torch.where(a >= 0, delta > high, delta < low)
    used = torch.where(cut, torch.where(a >= 0, 1.0 + CLIP_HIGH, 1.0 - CLIP_LOW), ratio)
    # a token moves its answer's ratio by one part in the answer's tokens, and all of them have that ratio: the sum is one token's
    d = torch.where(cut, 0.0, -a * ratio)
    kl = torch.zeros(n, device="cuda")
    if s.ref is not None:
        away = torch.where(on, s.ref.double() - s.logprob.double(), 0.0)   # 64 bits: small differences of numbers near one
        kl = (torch.expm1(away) - away).float()
        d = d - KL * torch.expm1(away).float()
    policy = (weight.double() * torch.where(on, -a * used, 0.0)).sum()
    kl_mean = (weight.double() * kl).sum()
    clipped = (weight.double() * (cut & on)).sum()
    entropy = torch.zeros_like(policy)
    if s.entropy is not None:
        entropy = (weight.double() * torch.where(on, s.entropy, 0.0)).sum()
    got = {"stats": torch.stack([policy + KL * kl_mean - BONUS * entropy, policy, kl_mean, entropy, clipped]).float(),
           "d_logprob": torch.where(on, weight * d, 0.0)}
    if s.entropy is not None:
        got["d_entropy"] = torch.where(on, -BONUS * weight, 0.0)
    return got


def _plain_muon(s):
    a, b, c = NS
    for p, m, g, copy in zip(s.p, s.m, s.g, s.copies):
        g = g.float() * s.grad_scale
        m.copy_(m * BETA + g * (1.0 - BETA))
        u = g * (1.0 - BETA) + m * BETA
        tall = u.shape[0] > u.shape[1]
        x = (u.t() if tall else u) / (torch.sqrt((u.double() * u.double()).sum()).float() + NS_EPS)
        for _ in range(5):
            gram = x @ x.t()
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        x = x.t() if tall else x
        p.copy_(p * (1.0 - LR * DECAY) - (LR * 0.2 * math.sqrt(max(p.shape))) * x)
        copy.copy_(p)


def run(state):
    s, case = state, state.case
    kind = case["kind"]
    if own:
        from paper_1911_08020_gb300 import darb
        if kind in ("scan", "back"):
            gates = darb.GATES_LOGITS if case["gates"] == "logits" else darb.GATES_VALUES
    if kind == "scan":
        if not own:
            h, h_last = _plain_scan(s)
        else:
            h, h_last = darb.darb_gated_scan(s.gate, s.x, s.h0, dim=_dim(case), gates=gates, coupled=case["coupled"], h=s.h, h_last=s.h_last)
        return {"h": h, "h_last": h_last}
    if kind == "back":
        if not own:
            return _plain_back(s)
        darb.darb_gated_scan_grad(s.dh, s.gate, s.x, s.h, s.h0, s.d_last, dim=_dim(case), gates=gates, coupled=case["coupled"],
                                  d_gate=s.d_gate, d_x=s.d_x, d_h0=s.d_h0)
        return {"d_gate": s.d_gate, "d_x": s.d_x, **({"d_h0": s.d_h0} if case["start"] else {})}
    if kind == "policy":
        if not own:
            return _plain_policy(s)
        o = darb.darb_policy_loss(s.logprob, s.old, s.advantage, s.offsets, ref_logprob=s.ref, entropy=s.entropy, mask=s.mask,
                                  clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL if case["kl"] else 0.0,
                                  entropy_coef=BONUS if case["bonus"] else 0.0,
                                  ratio=darb.PER_TOKEN if case["ratio"] == "tokens" else darb.PER_SEQUENCE,
                                  mean=darb.PER_TOKEN if case["mean"] == "tokens" else darb.PER_SEQUENCE, out=s.out)
        return {"stats": o.stats, "d_logprob": o.d_logprob, **({"d_entropy": o.d_entropy} if case["bonus"] else {})}
    if own:
        darb.darb_muon_step(s.plan, s.g, LR, BETA, DECAY, grad_scale=s.grad_scale)
    else:
        _plain_muon(s)
    return {"p": s.p, "copy": s.copies, "m": s.m}


def work(case):
    kind = case["kind"]
    if kind == "muon":
        n = sum(rows * cols for rows, cols in _sizes(case))
        # parameter and momentum in and out, the gradient in, the bf16 weight out
        return {"bytes": n * (16 + (4 if case["grads"] == "f32" else 2) + 2), "flops": _products(case)}
    if kind == "policy":
        n = case["tokens"]
        per = 8 + 1 + 4 + (4 if case["kl"] else 0) + (8 if case["bonus"] else 0)
        return {"bytes": n * per + case["sequences"] * 12, "flops": 20 * n}
    n = case["steps"] * case["features"] * case["batch"]
    width = 4 if case["dtype"] == "f32" else 2
    states = 4 * case["features"] * case["batch"] * (2 if case["start"] else 1)
    if kind == "scan":
        return {"bytes": 3 * n * width + states, "flops": 8 * n}
    return {"bytes": 6 * n * width + 2 * states, "flops": 14 * n}


def _exact_gates(case, gate):
    if case["gates"] == "logits":
        e = torch.exp(-gate.abs())
        near, far = 1.0 / (1.0 + e), e / (1.0 + e)
        return torch.where(gate >= 0, near, far), torch.where(gate >= 0, far, near)
    return gate, 1.0 - gate


def _exact_scan(case, seed):
    s = prepare(case, seed)
    dim = _dim(case)
    a, rest = _exact_gates(case, s.gate.double().movedim(dim, 0))
    u = s.x.double().movedim(dim, 0)
    u = rest * u if case["coupled"] else u
    h = torch.zeros(_state_shape(case), dtype=torch.float64, device="cuda") if s.h0 is None else s.h0.double()
    out = torch.empty_like(u)
    for t in range(case["steps"]):
        h = torch.addcmul(u[t], a[t], h)
        out[t] = h
    return {"h": out.movedim(0, dim), "h_last": h}


def _exact_back(case, seed):
    s = prepare(case, seed)
    dim = _dim(case)
    gate, x, h, dh = (t.double().movedim(dim, 0) for t in (s.gate, s.x, s.h, s.dh))
    a, rest = _exact_gates(case, gate)
    g = s.d_last.double()
    d_gate, d_x = torch.empty_like(a), torch.empty_like(a)
    for t in range(case["steps"] - 1, -1, -1):
        g = g + dh[t]
        if t:
            before = h[t - 1]
        else:
            before = torch.zeros_like(g) if s.h0 is None else s.h0.double()
        d_a = g * before
        d_x[t] = g
        if case["coupled"]:
            d_a = d_a - g * x[t]
            d_x[t] *= rest[t]
        d_gate[t] = d_a * a[t] * rest[t] if case["gates"] == "logits" else d_a
        g = g * a[t]
    got = {"d_gate": d_gate.movedim(0, dim), "d_x": d_x.movedim(0, dim)}
    if case["start"]:
        got["d_h0"] = g
    return got


def _exact_policy(case, seed):
    """In 64 bits, the gradients by automatic differentiation of the loss."""
    s = prepare(case, seed)
    offsets = s.offsets.tolist()
    lp = s.logprob.double().requires_grad_()
    ent = s.entropy.double().requires_grad_() if case["bonus"] else None
    lengths = s.offsets.diff()
    n_in = offsets[-1]
    ids = torch.repeat_interleave(torch.arange(case["sequences"], device="cuda"), lengths)
    on = s.mask[:n_in].double()
    zeros = torch.zeros(case["sequences"], dtype=torch.float64, device="cuda")
    count = zeros.index_add(0, ids, on)
    if case["mean"] == "tokens":
        weight = on / count.sum()
    else:
        weight = on / (count[ids].clamp(min=1) * (count > 0).sum())
    logr = lp[:n_in] - s.old[:n_in].double()
    if case["ratio"] == "sequences":
        logr = (zeros.index_add(0, ids, logr * on) / count.clamp(min=1))[ids]
    a = s.advantage.double()[ids]
    r = logr.exp()
    gain = torch.minimum(r * a, r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * a)
    policy = -(weight * gain).sum()
    zero = torch.zeros_like(policy)
    kl, entropy = zero, zero
    if case["kl"]:
        d = s.ref[:n_in].double() - lp[:n_in]
        kl = (weight * (d.exp() - 1.0 - d)).sum()
    if case["bonus"]:
        entropy = (weight * ent[:n_in]).sum()
    loss = policy + (KL * kl if case["kl"] else 0.0) - (BONUS * entropy if case["bonus"] else 0.0)
    loss.backward()
    outside = (a > 0) & (r > 1.0 + CLIP_HIGH) | (a < 0) & (r < 1.0 - CLIP_LOW)
    got = {"stats": torch.stack([loss, policy, kl, entropy, (weight * outside).sum()]).detach(), "d_logprob": lp.grad}
    if case["bonus"]:
        got["d_entropy"] = ent.grad
    return got


def _exact_muon(case, seed):
    s = prepare(case, seed)
    a, b, c = NS
    got = {"p": [], "copy": [], "m": []}
    for p, m, g in zip(s.p, s.m, s.g):
        g = g.double() * s.grad_scale.double()
        m = torch.lerp(m.double(), g, 1.0 - BETA)
        u = torch.lerp(g, m, BETA)
        x = u / (torch.linalg.matrix_norm(u) + NS_EPS)
        for _ in range(5):
            if x.shape[0] <= x.shape[1]:
                gram = x @ x.mT
                x = a * x + torch.addmm(b * gram, gram, gram, alpha=c) @ x
            else:
                gram = x.mT @ x
                x = a * x + x @ torch.addmm(b * gram, gram, gram, alpha=c)
        p = p.double() - LR * DECAY * p.double() - LR * 0.2 * max(p.shape) ** 0.5 * x
        got["p"].append(p)
        got["copy"].append(p)
        got["m"].append(m)
    return got


def exact(case, seed):
    return {"scan": _exact_scan, "back": _exact_back, "policy": _exact_policy, "muon": _exact_muon}[case["kind"]](case, seed)
