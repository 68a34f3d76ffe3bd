"""The gated feed-forward operators to the accuracy that each result's type has,
on inputs whose sums are known exactly.

Tails (16 bits).  Each weight's row has one entry, so that g and u are what the
test says.  A value is then rounded once: eps / 2 of it, and the smallest number of
its type.  Before that it is in f32 with the hardware's exponential: 2 + 1.2 |x|
units of 2^-23 for an argument x.  For silu and gelu |x| is at most 72 here, 1.1e-5,
with 5e-6 for gelu's polynomial: within 2^-15 of the value.  For gelu by tanh |x| is at
most 81, 1.2e-5, and the argument's own roundings, four of 2^-24 of it, make 2e-5 more:
within 2^-14.  A slope's terms may cancel: the same share of the sum of their sizes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"bf16": 1e-37, "f16": 2.0 ** -24}
TWO = 2 * math.sqrt(2 / math.pi)


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def act64(g, act):
    """act(g), its derivative and the sum of the sizes of the derivative's terms, in 64 bits without cancellation."""
    if act == "silu":
        s, r = torch.sigmoid(g), torch.sigmoid(-g)
        return g * s, s + g * s * r, s + g.abs() * s * r
    if act == "gelu":
        c, e = 0.5 * torch.erfc(-g / math.sqrt(2.0)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * c, c + g * e, c + g.abs() * e
    if act == "gelu_tanh":  # (1 + tanh y) / 2 = sigmoid(2 y)
        y = TWO * (g + 0.044715 * g ** 3)
        s, r = torch.sigmoid(y), torch.sigmoid(-y)
        by = s * r * TWO * (1 + 3 * 0.044715 * g * g)
        return g * s, s + g * by, s + g.abs() * by
    return g.clamp(min=0), (g > 0).double(), (g > 0).double()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("T", [1, 2, 7, 300])
def test_tails(sf, T, act, dtype):
    H, F, t = 64, 3001, TYPES[dtype]
    half, tiny = torch.finfo(t).eps / 2, TINY[dtype]
    own = 2.0 ** (-14 if act == "gelu_tanh" else -15)
    g = torch.linspace(-9.7 if act == "gelu_tanh" else -12, 3, F, device="cuda").to(t)
    x, dh = torch.zeros((T, H), dtype=t, device="cuda"), torch.zeros((T, F), dtype=t, device="cuda")
    x[:, 0] = x[:, 1] = 1
    dh[0] = 1
    a, slope, size = act64(g.double(), act)
    for u in (1.0, -1024.0):
        wg, wu = torch.zeros((F, H), dtype=t, device="cuda"), torch.zeros((F, H), dtype=t, device="cuda")
        wg[:, 0], wu[:, 1] = g, u
        r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act=act, want=("dw", "h"))
        for got, want, near in ((sf.sf_gated_ffn(x, wg, wu, act=act)[T - 1], a * u, (a * u).abs()), (r.h[T - 1], a * u, (a * u).abs()),
                                (r.dw_up[:, 1], a, a.abs()), (r.dw_gate[:, 0], slope * u, size * abs(u))):
            off = (got.double() - want).abs()
            bound = own * near + half * (want.abs() + own * near) + tiny
            assert bool((off <= bound).all()), (u, float((off / bound).max()), float(g[int((off / bound).argmax())]))
