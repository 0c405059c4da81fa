"""What the tests of the feed-forward blocks share: inputs, the operators in 64 bits on the CPU, and how far a result may be off.

Tolerances.  A sum of K products in fp32, in any order, is off by at most (K + 8) 2^-24 of the sum of the terms' sizes S (bf16 products are exact in fp32; 8 for the bias and the
joining of parts), and the framework's gate for fp32 sums is 1e-5 S: the smaller of the two holds.  An activation's or slope's evaluation in fp32 is off by at most 16 steps of 2^-24 (1 + |v|); the slopes
themselves are at most 1.13.  A rounding to type t is off by finfo(t).eps / 2 of the value.  Where rounded values are summed (dz in bf16 before the products) the
roundings are independent and each is at most eps / 2 of its term, so that their sum has a deviation below eps / 2 / sqrt(3) of the root of the terms' squares; five times eps / 2 of that
root is 8.6 deviations."""
import math

import torch

ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(t):
    return torch.finfo(t).eps / 2


def sum_gate(K):
    return min((K + 8) * 2.0 ** -24, 1e-5)


def value(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2))
    return v * torch.sigmoid(v) if act == "silu" else v


def slope(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * torch.special.erfc(-v / math.sqrt(2)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(v)
        return p * (1 + v * (1 - p))
    return torch.ones_like(v)


def evaluation(v):
    return 16 * 2.0 ** -24 * (1 + v.abs())


def whole(gen, shape, most, t=torch.float32):
    """Whole numbers of -most .. most: their sums are exact."""
    return torch.randint(-most, most + 1, shape, generator=gen).to(t)


def normal(gen, shape, std=1.0, t=torch.float32):
    return (torch.randn(shape, generator=gen) * std).to(t)


def places(gen, d_out, ablated):
    """active (or None) of a layer with that share of its neurons ablated, and the stored columns"""
    n = d_out - int(d_out * ablated)
    stored = torch.randperm(d_out, generator=gen)[:n].sort().values
    return (stored.int() if n < d_out else None), stored


def at_offset(t, elements, guard=64):
    """A copy of t on the GPU that begins `elements` elements behind a 512-byte boundary, and the buffer around it, filled with 77."""
    room = torch.full((guard + elements + t.numel() + guard,), 77.0, device="cuda").to(t.dtype)
    flat = room[guard + elements:guard + elements + t.numel()]
    flat.copy_(t.reshape(-1))
    return flat.view(t.shape), room


def untouched(room, elements, n, guard=64):
    return bool((room[:guard + elements] == 77).all()) and bool((room[guard + elements + n:] == 77).all())


def within(got, want, bound, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what
    off = (got - want).abs()
    bad = off > bound
    assert not bad.any(), "%s: off by %.3e where %.3e is allowed, %d of %d, first at %s" % (
        what, off[bad][0], bound.expand_as(off)[bad][0], int(bad.sum()), off.numel(), bad.nonzero()[0].tolist())


def linear(x, W, stored, bias, d_out, act, residual=None):
    """y, z and their bounds before the rounding to the output type"""
    x, W = x.double(), W.double()
    b = torch.zeros(d_out, dtype=torch.float64) if bias is None else bias.double()
    z = x @ W.T + b[stored]
    z_off = sum_gate(x.shape[1]) * (x.abs() @ W.abs().T + b[stored].abs())
    every, off = b.expand(x.shape[0], d_out).clone(), torch.zeros(x.shape[0], d_out, dtype=torch.float64)
    every[:, stored], off[:, stored] = z, z_off
    y = value(every, act)
    off = 1.13 * off + (0 if act in ("none", "relu") else evaluation(every))
    if residual is not None:
        off = off + 2.0 ** -24 * (y.abs() + residual.double().abs())
        y = y + residual.double()
    return y, off, z, z_off


def rounded(y, off, t):
    return off + half_step(t) * (y.abs() + off)


def products_bound(d, off, W, t, terms):
    """Bound of sum_k d(m, k) W(k, n) for d known to `off` in fp32 and rounded to t on its way into the product"""
    d, W = d.abs(), W.double().abs()
    spread = 0 if t == torch.float32 else 5 * half_step(t) * ((d * d) @ (W * W)).sqrt()
    return off @ W + spread + sum_gate(terms) * (1 + half_step(t)) * (d @ W)
