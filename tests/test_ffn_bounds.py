"""The bounds for f32 products see it when one of the six products of parts is lost:
the products by parts in 64 bits on the CPU, all of them and without each."""
import pytest
import torch
from ffn_bounds import act64, expected, share

ALL = [(0, 0), (0, 2), (2, 0), (1, 1), (0, 1), (1, 0)]


def parts(v):
    """Three bf16 whose sum is v: the upper half, the rest's nearest, its rest's."""
    a = (v.view(torch.int32) & -65536).view(torch.float32)
    b = (v - a).bfloat16().float()
    return a.double(), b.double(), (v - a - b).bfloat16().double()


def product(a, b, which):
    p, q = parts(a.contiguous()), parts(b.contiguous())
    return sum(p[i] @ q[k] for i, k in which)


def operators(x, wg, wu, act, dh, which):
    g, u = product(x, wg.t(), which).float(), product(x, wu.t(), which).float()
    a, slope, _, _ = act64(g.double(), act)
    d = dh.double()
    dg, du = (d * u.double() * slope).float(), (d * a).float()
    return {"h": (a * u.double()).float(), "dx": (product(dg, wg, which) + product(du, wu, which)).float(),
            "dw_gate": product(dg.t(), x, which).float(), "dw_up": product(du.t(), x, which).float()}


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("T,H,F", [(33, 64, 96), (64, 512, 300), (300, 200, 130)])
def test_a_lost_product_is_seen(T, H, F, act):
    gen = torch.Generator().manual_seed(T)
    n = lambda *s, k=1.0: torch.randn(s, generator=gen) * k  # noqa: E731
    x, wg, wu, dh = n(T, H), n(F, H, k=H ** -0.5), n(F, H, k=H ** -0.5), n(T, F, k=0.0625)
    want = expected(x, wg, wu, act, dh)
    fine = operators(x, wg, wu, act, dh, ALL)
    assert all(share(fine[k], want[k]) < 0.5 for k in want)
    for lost in ALL:
        r = operators(x, wg, wu, act, dh, [p for p in ALL if p != lost])
        assert all(share(r[k], want[k]) > 1.5 for k in want), lost
