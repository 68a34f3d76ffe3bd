"""Bounds of the gated feed-forward operators in f32 that a lost last part of a
product breaks: what a result's error is expected to be at most, as a root of the
mean square over a matrix.

A sum of n products a_i b_i whose signs are mixed has the size S = (sum (a_i b_i)^2)^1/2,
and so have its partial sums, S (k / n)^1/2 after k.  In chains of f32 on the f32 units
each step rounds by 2^-24 of the partial sum at most.  On the tensor cores runs of 256
are summed 16 at a time and cut off by 2^-23 of the partial sum at most: 2^-23 S
(256 / n)^1/2 times the sum of (j / 16)^1/2 over 16 steps, 11.2, for one run, and the runs'
errors have the signs of their own sums: 22.4 2^-24 S for all.  With what the three parts
of a value leave out (2^-25.6 S) and the runs' sum: 24 2^-24 S.  What is lost without the
third part of one factor is its size, 2^-17.7 of the value as a root of the mean square
(the second part has 8 bits of a rest that is spread evenly over 2^-7): 78 2^-24 S."""
import math

import torch

UNIT = 2.0 ** -24
SUM = 24 * UNIT


def act64(g, act):
    """act(g), its derivative, the sum of the sizes of the derivative's terms, and the share of their values
    by which f32 functions and their arguments' roundings may be off, in units of 2^-24."""
    if act == "silu":
        s, r = torch.sigmoid(g), torch.sigmoid(-g)
        return g * s, s + g * s * r, s + g.abs() * s * r, torch.full_like(g, 12)
    if act == "gelu":
        c, e = 0.5 * torch.erfc(-g / math.sqrt(2.0)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * c, c + g * e, c + g.abs() * e, 12 + 2 * g * g
    if act == "gelu_tanh":  # (1 + tanh y) / 2 = sigmoid(2 y)
        k = 2 * math.sqrt(2 / math.pi)
        y = k * (g + 0.044715 * g ** 3)
        s, r = torch.sigmoid(y), torch.sigmoid(-y)
        by = s * r * k * (1 + 3 * 0.044715 * g * g)
        return g * s, s + g * by, s + g.abs() * by, 16 + 4 * y.abs()
    return g.clamp(min=0), (g > 0).double(), (g > 0).double(), torch.zeros_like(g)


def squares(a, b):
    """(sum (a_i b_i)^2)^1/2 of each element of a b."""
    return ((a * a) @ (b * b)).sqrt()


def expected(x, wg, wu, act, dh):
    """{name: (value, the error expected at most as a root of the mean square)}; not for relu, whose slope jumps."""
    x, wg, wu, d = x.double(), wg.double(), wu.double(), dh.double()
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = SUM * squares(x, wg.t()), SUM * squares(x, wu.t())
    a, slope, size, own = act64(g, act)
    ea = slope.abs() * eg + own * UNIT * a.abs()
    es = 0.8 * eg + own * UNIT * size  # second derivatives are at most 0.8
    r = {"h": (a * u, torch.hypot(ea * u, a * eu) + 2 * UNIT * (a * u).abs())}
    dg, du = d * u * slope, d * a
    edg = d.abs() * torch.hypot(u * es, slope * eu) + 3 * UNIT * dg.abs()
    edu = d.abs() * ea + 2 * UNIT * du.abs()
    through = torch.hypot(squares(edg, wg), squares(edu, wu))
    r["dx"] = (dg @ wg + du @ wu, torch.hypot(through, SUM * torch.hypot(squares(dg, wg), squares(du, wu))))
    for name, q, eq in (("dw_gate", dg, edg), ("dw_up", du, edu)):
        r[name] = (q.t() @ x, torch.hypot(squares(eq.t(), x), SUM * squares(q.t(), x)))
    return r


def share(got, want):
    """The error's root of the mean square by the one expected at most."""
    value, bound = want
    return float(((got.double() - value) ** 2).mean().sqrt() / (bound ** 2).mean().sqrt())
