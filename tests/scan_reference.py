"""The gated recurrence and its backward pass in 64 bits, over the first axis, with bounds for fp32 arithmetic.

With u = 2^-24: exp2 of a product with log2 e is off by at most 4 u (the instruction's two units) and 2 |z| u (the
argument's roundings) relative to itself, a fast division by 4 u, so that sigmoid(z) and sigmoid(-z) are off by at
most K u with K = 14 + 2 max |z|, and a gate that is a value by nothing, its distance from 1 by u.  A term of the
state at step t that came in at step s carries the errors of t - s gates and of as many products and sums:
    |error of h_t| <= u sum_s (t - s) (K + 2) |term| + (K + 40) u sum_s |term|,
the second part for what enters and for the sums in which steps, warps and CTAs are put together.  Both sums
are recurrences of their own.
"""
import numpy as np

U = 2.0 ** -24


def gates_of(gate, logits):
    if not logits:
        return gate, 1.0 - gate, np.ones_like(gate)
    e = np.exp(-np.abs(gate))
    a = np.where(gate >= 0, 1 / (1 + e), e / (1 + e))
    r = np.where(gate >= 0, e / (1 + e), 1 / (1 + e))
    return a, r, a * r


def relative(gate, logits):
    """K of the bound."""
    return 14 + 2 * np.abs(gate).max(initial=0.0) if logits else 2.0


def walk(a, u, first, K):
    """(states, their bounds) of c_t = a_t c_(t-1) + u_t."""
    state, size, late = first, np.abs(first), np.zeros_like(first)
    out, bound = np.empty_like(u), np.empty_like(u)
    for t in range(len(u)):
        late = np.abs(a[t]) * (late + size)
        size = np.abs(a[t]) * size + np.abs(u[t])
        state = a[t] * state + u[t]
        out[t], bound[t] = state, U * ((K + 2) * late + (K + 40) * size)
    return out, bound


def forward(gate, x, h0, logits, coupled):
    """(h, its bound)."""
    a, r, _ = gates_of(gate, logits)
    return walk(a, r * x if coupled else x, h0, relative(gate, logits))


def back(dh, gate, x, h, h0, d_last, logits, coupled):
    """(d_gate, d_x, d_h0, and their bounds), h being what the forward pass left."""
    a, r, slope = gates_of(gate, logits)
    K = relative(gate, logits)
    # g_t = dh_t + a_(t+1) g_(t+1): over the reversed steps
    later = np.concatenate([a[1:], np.ones_like(a[:1])])[::-1]
    g, e = walk(later, dh[::-1], d_last, K)
    g, e = g[::-1], e[::-1]
    before = np.concatenate([h0[None], h[:-1]])
    q = (before - x if coupled else before) * slope
    # the factors: two gates and their product, a difference, the product with g
    e_gate = np.abs(q) * e + (2 * K + 8) * U * np.abs(g) * np.abs(slope) * (np.abs(before) + (np.abs(x) if coupled else 0.0))
    rest = r if coupled else np.ones_like(r)
    return (g * q, g * rest, a[0] * g[0],
            e_gate, np.abs(rest) * e + (K + 4) * U * np.abs(g * rest), np.abs(a[0]) * e[0] + (K + 4) * U * np.abs(a[0] * g[0]))
