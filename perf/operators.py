"""Scoring and training around a pruned layer, as measurable cases.

The prune-retrain loop scores the tokens that a model was given, takes the gradient of that score, goes
back through the normalisation between the layers, updates the dense weights and encodes them again.
Five kinds of pass:

* ``score``    the log probability of given tokens, the entropy and the k best alternatives (``darb_token_logprobs``);
* ``loss``     the gradient of log probability and entropy with respect to the logits (``darb_token_logprobs_grad``);
* ``norm``     layer norm (``darb_layer_norm``);
* ``back``     its backward pass, with the gradients of gain and offset (``darb_layer_norm_grad``);
* ``adamw``    one AdamW step over all tensors of a model (``darb_adamw_step``).

Activations lie either as token rows (tokens x features) or as token columns (features x tokens, the
layout that ``darb_spmm`` and the sequence calls read and write).
"""
import math

import torch

own = False

BLOCK = 256        # elements that share a scale where a state is held in 8 bits
CODE_MAX = 448.0   # the largest value of an e4m3 code
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # One token of one stream: the word just chosen, with the alternatives shown beside it.  Latency is all there is.
        {"name": "score_one", "kind": "score", "layout": "rows", "dtype": "bf16", "tokens": 1, "vocab": 32000, "k": 8, "masked": 0.0},
        # One step of a language model with 10000 words at batch 20, the logits as darb_spmm leaves them.
        {"name": "score_lm_step", "kind": "score", "layout": "columns", "dtype": "f32", "tokens": 20, "vocab": 10000, "k": 5, "masked": 0.0},
        # A long prompt scored at once.
        {"name": "score_prompt", "kind": "score", "layout": "rows", "dtype": "bf16", "tokens": 4096, "vocab": 32000, "k": 5, "masked": 0.0},
        # Answers drawn under a grammar: most words are masked at every position, a ragged count of both.
        {"name": "score_masked", "kind": "score", "layout": "rows", "dtype": "f32", "tokens": 1023, "vocab": 128001, "k": 20, "masked": 0.9},
        # The loss of the language model's training step: 35 steps of 20 streams, one product's logits.
        {"name": "loss_lm", "kind": "loss", "layout": "columns", "dtype": "f32", "tokens": 700, "vocab": 10000, "masked": 0.0, "entropy": False},
        # The loss of a prompt with an entropy bonus.
        {"name": "loss_prompt", "kind": "loss", "layout": "rows", "dtype": "bf16", "tokens": 4096, "vocab": 32000, "masked": 0.0, "entropy": True},
        # The hidden state between two layers of the language model, one step.
        {"name": "norm_lm_step", "kind": "norm", "layout": "columns", "dtype": "f32", "steps": 1, "tokens": 20, "features": 1500},
        # The activations of a wide layer over a large batch, an odd number of tokens.
        {"name": "norm_rows", "kind": "norm", "layout": "rows", "dtype": "bf16", "steps": 1, "tokens": 8191, "features": 4096},
        # Backward through a whole sequence of hidden states (steps x features x batch).
        {"name": "back_lm", "kind": "back", "layout": "columns", "dtype": "f32", "steps": 35, "tokens": 20, "features": 1500},
        # Backward through the wide layer.
        {"name": "back_rows", "kind": "back", "layout": "rows", "dtype": "bf16", "steps": 1, "tokens": 8192, "features": 4096},
        # Every tensor of the language model: two layers of gates, embedding and output table, biases.
        {"name": "adamw_lm", "kind": "adamw", "states": "f32", "grads": "f32", "layers": 2, "rows": 6000, "cols": 3000, "tables": 2, "words": 10000, "width": 1500},
        # Two fully-connected layers with states in 8 bits, bf16 gradients, and the bf16 weights that are encoded next.
        {"name": "adamw_fc_8bit", "kind": "adamw", "states": "e4m3", "grads": "bf16", "layers": 1, "rows": 4096, "cols": 9216, "tables": 1, "words": 4096, "width": 4096},
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("score", "score", "score", "loss", "loss", "norm", "back", "back", "adamw", "adamw"))
    if kind == "adamw":
        layers, tables = rng.randint(1, 6), rng.randint(0, 2)
        rows, cols = _spread(rng, 16, 6000), _spread(rng, 16, 9216)
        words, width = _spread(rng, 100, 10000), _spread(rng, 16, 4096)
        most = 60_000_000
        while layers * rows * cols + tables * words * width > most:
            rows, words = max(1, rows * 2 // 3), max(1, words * 2 // 3)
        return {"kind": kind, "states": rng.choice(("f32", "e4m3")), "grads": rng.choice(("f32", "bf16")),
                "layers": layers, "rows": rows, "cols": cols, "tables": tables, "words": words, "width": width}
    case = {"kind": kind, "layout": rng.choice(("rows", "rows", "columns")), "dtype": rng.choice(("f32", "bf16"))}
    if kind in ("score", "loss"):
        case["vocab"] = _spread(rng, 1000, 131072)
        case["tokens"] = _spread(rng, 1, max(1, min(8192, 65_000_000 // case["vocab"])))
        case["masked"] = rng.choice((0.0, 0.0, 0.9))
        if kind == "score":
            case["k"] = rng.choice((0, 1, 5, 20))
        else:
            case["entropy"] = rng.random() < 0.5
        return case
    case["features"] = _spread(rng, 64, 12288)
    case["steps"] = _spread(rng, 1, 64) if case["layout"] == "columns" else 1
    most = max(1, min(16384, 33_000_000 // (case["features"] * case["steps"])))
    case["tokens"] = _spread(rng, 1, min(most, 256) if case["layout"] == "columns" else most)
    return case


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _dim(case):
    """The axis of the features (or of the vocabulary)."""
    return -1 if case["layout"] == "rows" else -2


def _layout(case, t):
    """Token rows (N x F) in the layout of the case."""
    return t if case["layout"] == "rows" else t.transpose(-1, -2).contiguous()


def _sizes(case):
    """Elements of every tensor of the model: a matrix and two biases a layer, and the tables."""
    got = []
    for _ in range(case["layers"]):
        got += [case["rows"] * case["cols"], case["rows"], case["rows"]]
    return got + [case["words"] * case["width"]] * case["tables"]


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _logits(case, seed):
    """Logits with the spread that a language model's have, the tokens that were given, and the masked entries."""
    gen = _generator(seed)
    n, v = case["tokens"], case["vocab"]
    x = 2.5 * torch.randn(n, v, generator=gen, device="cuda")
    x -= 1.5 * torch.log1p(torch.arange(v, device="cuda", dtype=torch.float32))   # frequent words first
    targets = (torch.rand(n, generator=gen, device="cuda") ** 4 * v).long().clamp(max=v - 1)
    x[torch.arange(n, device="cuda"), targets] += 4.0
    if case["masked"]:
        hide = torch.rand(n, v, generator=gen, device="cuda") < case["masked"]
        hide[torch.arange(n, device="cuda"), targets] = False
        x.masked_fill_(hide, -math.inf)
    # positions that are padding have no token
    targets[torch.rand(n, generator=gen, device="cuda") < 0.05] = -1
    return _layout(case, x.to(_dtype(case["dtype"]))), targets, gen


def _activations(case, gen):
    """N(0, 1) activations with a scale and an offset for each token, in the layout of the case."""
    n = case["tokens"]
    lead = (case["steps"],) if case["layout"] == "columns" else ()
    x = torch.randn(*lead, n, case["features"], generator=gen, device="cuda")
    x = x * (0.5 + torch.rand(*lead, n, 1, generator=gen, device="cuda")) + 0.3 * torch.randn(*lead, n, 1, generator=gen, device="cuda")
    return _layout(case, x.to(_dtype(case["dtype"])))


def _noise(n, seed):
    """For elements 0 to n - 1 two random numbers each, of 16 bits, from the step's seed: the input of the states' rounding."""
    z = torch.arange(n, device="cuda") * 0x9E3779B1 + ((seed * 0x9E3779B97F4A7C15 & (1 << 64) - 1) >> 32) & 0xFFFFFFFF
    z = (z ^ z >> 15) * 0x6A09E667 & 0xFFFFFFFF
    z = (z ^ z >> 13) * 0xBB67AE85 & 0xFFFFFFFF
    z = z ^ z >> 16
    return z >> 16, z & 0xFFFF


def _quantised(t, noise):
    """(codes, scales) of a flat tensor whose length is a whole number of blocks.  A value between two
    codes goes up with the probability that leaves its mean as it is: a moment moves by a thousandth a
    step, which rounding to the nearest code would undo every time."""
    b = t.view(-1, BLOCK)
    scale = b.abs().amax(dim=1, keepdim=True) * (1.0 / CODE_MAX)
    fine = scale >= torch.finfo(torch.float32).tiny
    inverse = torch.where(fine, torch.reciprocal(torch.where(fine, scale, 1.0)), 0.0)
    x = (b * inverse).view(-1)
    # below 2^-6 the codes are 2^-9 apart, as they are from 2^-6 to 2^-5
    a = x.abs()
    shift = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0)
    bits = (a + shift).view(torch.int32) + (noise.int() << 4) + 8 & ~0xFFFFF
    code = torch.where(a.isnan(), a, (bits.view(torch.float32) - shift).clamp(max=CODE_MAX))
    return torch.copysign(code, x), scale.view(-1)


def _moments(case, gen, at):
    """Flat parameters, gradients and moments with the scales that they have some way into training."""
    n = at[-1]
    keep = torch.zeros(n, dtype=torch.bool, device="cuda")
    for size, start in zip(_sizes(case), at):
        keep[start:start + size] = True
    size = 1e-3 * torch.exp(0.7 * torch.randn(n // BLOCK, 1, generator=gen, device="cuda")).expand(-1, BLOCK).reshape(-1)
    p = 0.05 * torch.randn(n, generator=gen, device="cuda")
    g = size * torch.randn(n, generator=gen, device="cuda")
    m = 0.3 * size * torch.randn(n, generator=gen, device="cuda")
    r = size * torch.exp(0.3 * torch.randn(n, generator=gen, device="cuda"))
    return [torch.where(keep, t, 0.0) for t in (p, g, m, r)]


class _State:
    """What a program has in hand before a call."""

    def __init__(self, case, seed):
        self.case, self.plan = case, None
        kind = case["kind"]
        if kind in ("score", "loss"):
            self.x, self.targets, gen = _logits(case, seed)
            if kind == "loss":
                # the forward pass has left its sums; the gradient of a mean over the tokens comes in
                lse = torch.logsumexp(self.x.double(), dim=_dim(case))
                logp = self.x.double() - lse.unsqueeze(_dim(case))
                self.lse = lse.float()
                self.entropy = -torch.where(logp > -math.inf, logp.exp() * logp, 0.0).sum(dim=_dim(case)).float()
                self.d_logprob = -(0.5 + torch.rand(case["tokens"], generator=gen, device="cuda")) / case["tokens"]
                self.d_entropy = 0.01 * self.d_logprob if case["entropy"] else None
                self.grad = torch.empty_like(self.x)
            elif own:
                from paper_1911_08020_gb300 import darb
                self.out = darb.TokenLogprobs.empty(case["tokens"], case["k"], self.x.device)
            return
        gen = _generator(seed)
        if kind in ("norm", "back"):
            self.x = _activations(case, gen)
            f = case["features"]
            self.gamma = 1.0 + 0.2 * torch.randn(f, generator=gen, device="cuda")
            self.beta = 0.1 * torch.randn(f, generator=gen, device="cuda")
            # buffers that a program keeps from step to step
            self.y = torch.empty_like(self.x)
            stat = self.x.double()
            mean, var = stat.mean(dim=_dim(case)), stat.var(dim=_dim(case), unbiased=False)
            self.mean, self.rstd = torch.empty_like(mean, dtype=torch.float32), torch.empty_like(mean, dtype=torch.float32)
            if kind == "back":   # the forward pass has left its statistics
                self.mean.copy_(mean)
                self.rstd.copy_(torch.rsqrt(var + EPS))
                self.dy = _activations(case, gen)
                self.dgamma, self.dbeta = torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
            return
        self.step, self.seed = 100, seed
        at = [0]
        for n in _sizes(case):
            at.append(at[-1] + _padded(n))
        self.at = at
        self.p, g, m, r = _moments(case, gen, at)
        self.g = g.to(_dtype(case["grads"]))
        self.copy = torch.empty(at[-1], dtype=torch.bfloat16, device="cuda").copy_(self.p)
        self.grad_scale = torch.full((), 0.5, device="cuda")   # what clipping by the gradients' norm gives
        self.m_scale = self.v_scale = None
        if case["states"] == "f32":
            self.m, self.v = m, r * r
        else:
            noise = _noise(at[-1], seed)
            (m, self.m_scale), (r, self.v_scale) = _quantised(m, noise[0]), _quantised(r, noise[1])
            self.m, self.v = m.to(torch.float8_e4m3fn), r.to(torch.float8_e4m3fn)
        if own:
            from paper_1911_08020_gb300 import darb

            def parts(t, per=1):
                return None if t is None else [t[a // per:a // per + -(-n // per)] for a, n in zip(at, _sizes(case))]

            self.grads = parts(self.g)
            self.plan = darb.darb_adamw_create(parts(self.p), parts(self.m), parts(self.v), parts(self.m_scale, BLOCK),
                                               parts(self.v_scale, BLOCK), copies=parts(self.copy), grad_dtype=self.g.dtype)


def prepare(case, seed):
    return _State(case, seed)


def _plain_score(x, targets, k, dim):
    x = x.float().movedim(dim, -1)
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    d = x - m
    e = torch.exp(d)
    s = e.sum(dim=-1, keepdim=True)
    log_s = torch.log(s)
    empty = (s == 0).squeeze(-1)
    entropy = (log_s - (e * torch.where(e > 0, d, 0.0)).sum(dim=-1, keepdim=True) / s).squeeze(-1)
    entropy = torch.where(empty, 0.0, entropy)
    logprob = (d.gather(-1, targets.clamp(0, x.shape[-1] - 1).unsqueeze(-1)) - log_s).squeeze(-1)
    logprob = torch.where(empty, -math.inf, logprob)
    logprob = torch.where(targets < 0, 0.0, torch.where(targets >= x.shape[-1], math.nan, logprob))
    got = {"logprob": logprob, "entropy": entropy, "lse": (m + log_s).squeeze(-1)}
    if k:
        # one whole number orders by value, then by the lower index
        bits = (torch.where(x.isnan(), math.nan, x) + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (bits << 32) | (x.shape[-1] - 1 - torch.arange(x.shape[-1], device=x.device))
        top = x.shape[-1] - 1 - (key.topk(k, dim=-1).values & 0xFFFFFFFF)
        got["top_logprob"] = torch.where(empty.unsqueeze(-1), -math.inf, d.gather(-1, top) - log_s)
        got["top_index"] = top.int()
    return got


def _plain_loss(s):
    dim = _dim(s.case)
    x = s.x.float().movedim(dim, -1)
    logp = x - s.lse.unsqueeze(-1)
    p = torch.exp(logp)
    hit = torch.arange(x.shape[-1], device=x.device) == s.targets.unsqueeze(-1)
    a = torch.where(s.targets < 0, 0.0, s.d_logprob).unsqueeze(-1)
    g = a * (hit.float() - p)
    if s.d_entropy is not None:
        g = g - s.d_entropy.unsqueeze(-1) * p * (torch.where(p > 0, logp, 0.0) + s.entropy.unsqueeze(-1))
    return g.movedim(-1, dim).to(s.x.dtype)


def _plain_norm(s):
    dim = _dim(s.case)
    x = s.x.float().movedim(dim, -1)
    mean = x.mean(dim=-1, keepdim=True)
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).mean(dim=-1, keepdim=True) + EPS)
    y = c * rstd * s.gamma + s.beta
    return y.movedim(-1, dim).to(s.x.dtype), mean.squeeze(-1), rstd.squeeze(-1)


def _plain_back(s):
    dim = _dim(s.case)
    x, dy = s.x.float().movedim(dim, -1), s.dy.float().movedim(dim, -1)
    rstd = s.rstd.unsqueeze(-1)
    xh = (x - s.mean.unsqueeze(-1)) * rstd
    g = dy * s.gamma
    dx = rstd * (g - g.mean(dim=-1, keepdim=True) - xh * (g * xh).mean(dim=-1, keepdim=True))
    tokens = tuple(range(x.dim() - 1))
    return dx.movedim(-1, dim).to(s.x.dtype), (dy * xh).sum(dim=tokens), dy.sum(dim=tokens)


def _plain_adamw(s):
    f32 = s.case["states"] == "f32"
    g = s.g.float() * s.grad_scale
    if f32:
        m, v = s.m, s.v
    else:
        m = (s.m.float().view(-1, BLOCK) * s.m_scale.unsqueeze(1)).view(-1)
        r = (s.v.float().view(-1, BLOCK) * s.v_scale.unsqueeze(1)).view(-1)
        v = r * r
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    r = torch.sqrt(v)
    step_size = LR / (1.0 - BETA1 ** s.step)
    denom = r * (1.0 / math.sqrt(1.0 - BETA2 ** s.step)) + ADAM_EPS
    s.p.copy_(s.p * (1.0 - LR * DECAY) - (m * step_size) / denom)
    s.copy.copy_(s.p)
    if f32:
        s.m.copy_(m)
        s.v.copy_(v)
        return
    noise = _noise(m.numel(), s.seed + s.step)
    code, scale = _quantised(m, noise[0])
    s.m.copy_(code.to(torch.float8_e4m3fn))
    s.m_scale.copy_(scale)
    code, scale = _quantised(r, noise[1])
    # a root that is not zero keeps a code that is not zero
    code = torch.where((r > 0) & (code == 0), 2.0 ** -9, code)
    s.v.copy_(code.to(torch.float8_e4m3fn))
    s.v_scale.copy_(scale)


def _moment_values(s):
    """The states as the values that they stand for."""
    if s.case["states"] == "f32":
        return s.m, s.v
    return ((s.m.float().view(-1, BLOCK) * s.m_scale.unsqueeze(1)).view(-1),
            (s.v.float().view(-1, BLOCK) * s.v_scale.unsqueeze(1)).view(-1))


def run(state):
    s, case = state, state.case
    kind = case["kind"]
    if own:
        from paper_1911_08020_gb300 import darb
    if kind == "score":
        if not own:
            return _plain_score(s.x, s.targets, case["k"], _dim(case))
        o = darb.darb_token_logprobs(s.x, s.targets, case["k"], dim=_dim(case), out=s.out)
        got = {"logprob": o.logprob, "entropy": o.entropy, "lse": o.lse}
        return {**got, "top_logprob": o.top_logprob, "top_index": o.top_index} if case["k"] else got
    if kind == "loss":
        if not own:
            return _plain_loss(s)
        return darb.darb_token_logprobs_grad(s.x, s.targets, s.lse, s.d_logprob, s.entropy, s.d_entropy, dim=_dim(case), out=s.grad)
    if kind == "norm":
        if not own:
            return _plain_norm(s)
        return darb.darb_layer_norm(s.x, s.gamma, s.beta, EPS, dim=_dim(case), y=s.y, mean=s.mean, rstd=s.rstd)
    if kind == "back":
        if not own:
            return _plain_back(s)
        return darb.darb_layer_norm_grad(s.dy, s.x, s.gamma, s.mean, s.rstd, dim=_dim(case), dx=s.y, dgamma=s.dgamma, dbeta=s.dbeta)
    if own:
        darb.darb_adamw_step(s.plan, s.grads, s.step, LR, BETA1, BETA2, ADAM_EPS, DECAY, grad_scale=s.grad_scale,
                             seed=s.seed + s.step)
    else:
        _plain_adamw(s)
    s.step += 1
    if case["states"] == "f32":
        return {"p": s.p, "copy": s.copy, "m": s.m, "v": s.v}
    return {"p": s.p, "copy": s.copy, "m": s.m, "m_scale": s.m_scale, "v": s.v, "v_scale": s.v_scale}


def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = sum(_sizes(case))
        grads = 4 if case["grads"] == "f32" else 2
        # the parameter, the moments and (in 8 bits) their scales in and out, the gradient in, the bf16 weight out
        states = 16 if case["states"] == "f32" else 4 + 16 / BLOCK
        return {"bytes": n * (8 + grads + states + 2), "flops": 15 * n}
    width = 4 if case["dtype"] == "f32" else 2
    if kind in ("score", "loss"):
        n, v = case["tokens"], case["vocab"]
        if kind == "score":
            return {"bytes": n * (v * width + 8 + 12 + 8 * case["k"]), "flops": 6 * n * v}
        return {"bytes": n * (2 * v * width + 16), "flops": (8 if case["entropy"] else 4) * n * v}
    n = case["steps"] * case["tokens"]
    f = case["features"]
    if kind == "norm":
        return {"bytes": n * (2 * f * width + 8) + 8 * f, "flops": 8 * n * f}
    return {"bytes": n * (3 * f * width + 8) + 12 * f, "flops": 14 * n * f}


def _exact_score(case, seed):
    x, targets, _ = _logits(case, seed)
    x = x.double() if case["layout"] == "rows" else x.double().t().contiguous()
    logp = torch.log_softmax(x, dim=1)
    lse = torch.logsumexp(x, dim=1)
    rows = torch.arange(x.shape[0], device=x.device)
    logprob = torch.where(targets < 0, 0.0, logp[rows, targets.clamp(min=0)])
    entropy = -torch.xlogy(logp.exp(), logp.exp()).sum(dim=1)
    got = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if case["k"]:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["k"]]
        got["top_logprob"] = logp.gather(1, order)
        got["top_index"] = order.int()
    return got


def _exact_loss(case, seed):
    s = prepare(case, seed)
    x = s.x.double() if case["layout"] == "rows" else s.x.double().t().contiguous()
    p = torch.softmax(x, dim=1)
    a = torch.where(s.targets < 0, 0.0, s.d_logprob.double())
    g = -a[:, None] * p
    given = torch.nonzero(s.targets >= 0).squeeze(1)
    g[given, s.targets[given]] += a[given]
    if s.d_entropy is not None:
        plogp = torch.xlogy(p, p)
        g += s.d_entropy.double()[:, None] * (p * plogp.sum(dim=1, keepdim=True) - plogp)
    return g if case["layout"] == "rows" else g.t().contiguous()


def _rows64(case, t):
    """Activations as token rows in 64 bits."""
    t = t.double()
    return t if case["layout"] == "rows" else t.transpose(1, 2).reshape(-1, case["features"])


def _back64(case, t):
    return t if case["layout"] == "rows" else t.view(case["steps"], case["tokens"], -1).transpose(1, 2).contiguous()


def _exact_norm(case, seed):
    s = prepare(case, seed)
    x = _rows64(case, s.x)
    var, mean = torch.var_mean(x, dim=1, unbiased=False)
    rstd = (var + EPS) ** -0.5
    shape = (case["steps"], case["tokens"]) if case["layout"] == "columns" else (case["tokens"],)
    y = torch.addcmul(s.beta.double(), (x - mean[:, None]) * rstd[:, None], s.gamma.double())
    if case["kind"] == "norm":
        return _back64(case, y), mean.view(shape), rstd.view(shape)
    dy, f = _rows64(case, s.dy), case["features"]
    xh = (x - mean[:, None]) * rstd[:, None]
    gg = dy * s.gamma.double()
    dx = (rstd / f)[:, None] * (f * gg - gg.sum(1, keepdim=True) - xh * torch.einsum("nf,nf->n", gg, xh)[:, None])
    return _back64(case, dx), torch.einsum("nf,nf->f", dy, xh), dy.sum(0)


def _random_code(t, noise):
    """The value of an e4m3 code (three bits of fraction, exponents from -6) next to each of t, below or above as the noise says."""
    exponent = torch.frexp(t.abs().clamp(min=2.0 ** -6)).exponent - 1
    unit = torch.ldexp(torch.ones_like(t), exponent - 3)
    up = torch.floor(t.abs() / unit + (noise.double() + 0.5) / 65536)
    return torch.sign(t) * (up * unit).clamp(max=CODE_MAX)


def _exact_adamw(case, seed):
    s = prepare(case, seed)
    b1, b2 = BETA1, BETA2
    m, v = (t.double() for t in _moment_values(s))
    if case["states"] != "f32":
        v = v.square()
    g = s.g.double() * s.grad_scale.double()
    m += (1 - b1) * (g - m)
    v += (1 - b2) * (g.square() - v)
    mh, vh = m / (1 - b1 ** s.step), v / (1 - b2 ** s.step)
    p = s.p.double()
    p = p - LR * DECAY * p - LR * mh / (vh.sqrt() + ADAM_EPS)
    if case["states"] == "f32":
        return {"p": p, "copy": p, "m": m, "v": v}
    got = {"p": p, "copy": p}
    for name, t, noise in zip("mv", (m, v.sqrt()), _noise(m.numel(), s.seed + s.step)):
        scale = t.view(-1, BLOCK).abs().amax(dim=1) / CODE_MAX
        code = _random_code(torch.where(scale[:, None] > 0, t.view(-1, BLOCK) / scale[:, None], 0.0), noise.view(-1, BLOCK))
        if name == "v":
            code = torch.where((t.view(-1, BLOCK) > 0) & (code == 0), 2.0 ** -9, code)
        got[name], got[name + "_scale"] = code.view(-1), scale
    return got


def exact(case, seed):
    if case["kind"] == "score":
        return _exact_score(case, seed)
    if case["kind"] == "loss":
        return _exact_loss(case, seed)
    if case["kind"] in ("norm", "back"):
        return _exact_norm(case, seed)
    return _exact_adamw(case, seed)
