"""A layer's matrix products and their gradients in 64 bits, each with a bound on what the bf16 kernels may be off.

A value's bound counts:
  - fp32 sums of K products of bf16 numbers: at most 2^-24 (K + 2) times the sum of the terms' magnitudes (a tensor core
    adds fewer, longer steps and may truncate them: 16 products a step, 2^-23 each);
  - fp32 activations and slopes: 2^-15 relative to the terms they are made of (an exponential whose argument, up to
    about 90, carries 2^-24 relative, and the hardware's few ulps; their second derivatives are below 1.2);
  - a rounding to bf16: half a step, 2^-8 relative.
"""

import math

import torch

ACTS = ("none", "gelu", "gelu_tanh", "silu")
F32, FORM, HALF = 2.0 ** -24, 2.0 ** -15, 2.0 ** -8
STEEP, CURVED = 1.2, 1.2           # the largest |act'| and |act''|
TINY = 2.0 ** -126                 # where fp32 has no more relative precision


def act(x, name):
    if name == "gelu":
        return x * 0.5 * torch.special.erfc(-x / math.sqrt(2))
    if name == "gelu_tanh":
        return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    return x * torch.sigmoid(x) if name == "silu" else x


def slope(x, name):
    if name == "none":
        return torch.ones_like(x)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-x / math.sqrt(2)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    c = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(c * (x + 0.044715 * x ** 3))
    return s + x * s * (1 - s) * c * (1 + 3 * 0.044715 * x * x)


def product(x, w, b=None):
    """x w^T + b in 64 bits, and the bound of its fp32 sum."""
    x, w = x.double(), w.double()
    y, mass = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        y, mass = y + b.double(), mass + b.double().abs()
    return y, F32 * (x.shape[1] + 2) * mass


def _act_bound(p, e, name):
    """Of act(p) when p is e off."""
    return STEEP * e + (0 if name == "none" else FORM * act(p, name).abs() + TINY)


def _slope_bound(p, e, name):
    return 0 if name == "none" else CURVED * e + FORM * (1 + (p * p).clamp(max=8))


def rounded(y, e):
    """The bound of a value that is e off and then rounded to bf16."""
    return e + HALF * (y.abs() + e) + TINY


def linear(x, w, b, name, residual):
    """(y, bound), (p, bound)."""
    p, e = product(x, w, b)
    y, ey = act(p, name), _act_bound(p, e, name)
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2 * F32 * (y.abs() + residual.double().abs())
    return (y, rounded(y, ey)), (p, rounded(p, e))


def gated(x, wg, wu, bg, bu, name):
    (g, eg), (u, eu) = product(x, wg, bg), product(x, wu, bu)
    a, ea = act(g, name), _act_bound(g, eg, name)
    h = a * u
    eh = a.abs() * eu + ea * (u.abs() + eu) + 2 * F32 * h.abs()
    return (h, rounded(h, eh)), (g, rounded(g, eg)), (u, rounded(u, eu))


def linear_delta(dy, x, w, b, pre, name):
    """d and its bound before it is rounded for the products."""
    dy = dy.double()
    if name == "none":
        return dy, torch.zeros_like(dy)
    p, e = (pre.double(), torch.zeros_like(dy)) if pre is not None else product(x, w, b)
    d = dy * slope(p, name)
    return d, dy.abs() * _slope_bound(p, e, name) + 2 * F32 * d.abs() + TINY


def gated_delta(dy, x, wg, wu, bg, bu, gate, up, name):
    dy = dy.double()
    if gate is not None:
        g, u, eg, eu = gate.double(), up.double(), torch.zeros_like(dy), torch.zeros_like(dy)
    else:
        (g, eg), (u, eu) = product(x, wg, bg), product(x, wu, bu)
    s, a = slope(g, name), act(g, name)
    dg, du = dy * u * s, dy * a
    edg = dy.abs() * (s.abs() * eu + _slope_bound(g, eg, name) * (u.abs() + eu)) + 4 * F32 * dg.abs() + TINY
    edu = dy.abs() * _act_bound(g, eg, name) + 2 * F32 * du.abs() + TINY
    return (dg, edg), (du, edu)


def gradients(x, deltas, weights, exact_delta=False):
    """(dx, bound), [(dw, bound)], [(db, bound)] from the deltas (value, bound before rounding to bf16)."""
    x = x.double()
    dx = edx = 0
    dw, db = [], []
    terms = len(weights) * weights[0].shape[0]
    for (d, e), w in zip(deltas, weights):
        w = w.double()
        off = e if exact_delta else rounded(d, e)
        big = d.abs() + off
        dx = dx + d @ w
        edx = edx + off @ w.abs() + F32 * (terms + 2) * (big @ w.abs())
        y = d.T @ x
        dw.append((y, rounded(y, off.T @ x.abs() + F32 * (d.shape[0] + 2) * (big.T @ x.abs()))))
        db.append((d.sum(0), e.sum(0) + F32 * (d.shape[0] + 2) * (d.abs() + e).sum(0) + TINY))
    return (dx, rounded(dx, edx)), dw, db


def check(got, want, what):
    y, bound = want
    off = (got.double() - y).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {float(got[i])}, want "
                             f"{float(y[i])}, bound {float(bound[i]):.3e}")


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

GAP = float("nan")                 # between a row's end and the next row


def rows(n, width, pad, device, fill=GAP):
    """A matrix of which only [:, :width] belongs to it, and the whole buffer with `fill` behind its rows and after it."""
    buffer = torch.full((n + 2, -(-(width + pad) // 8) * 8), fill, dtype=torch.bfloat16, device=device)
    return buffer[:n, :width], buffer


def random_rows(n, width, gain, g, pad=0):
    m, _ = rows(n, width, pad, g.device)
    m.copy_(torch.randn((n, width), generator=g, device=g.device) * gain)
    return m


def untouched(m, buffer):
    """Whether the buffer around m still holds what rows() left there."""
    n, width = m.shape
    return bool(torch.isnan(buffer[n:].float()).all()) and bool(torch.isnan(buffer[:n, width:].float()).all())
