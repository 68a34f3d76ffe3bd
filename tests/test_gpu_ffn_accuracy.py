"""The gated feed-forward operators to the accuracy that each result's type has,
on inputs whose sums are known exactly.

Tails (16 bits).  Each weight's row has one entry, so that g and u are what the
test says.  A value is then rounded once: eps / 2 of it, and the smallest number of
its type.  Before that it is in f32 with the hardware's exponential: 2 + 1.2 |x|
units of 2^-23 for an argument x.  For silu and gelu |x| is at most 72 here, 1.1e-5,
with 5e-6 for gelu's polynomial: within 2^-15 of the value.  For gelu by tanh |x| is at
most 81, 1.2e-5, and the argument's own roundings, four of 2^-24 of it, make 2e-5 more:
within 2^-14.  A slope's terms may cancel: the same share of the sum of their sizes.

f32.  Errors as roots of the mean square against ffn_bounds, which a lost product of
parts breaks, and inputs whose sums lie in the lower parts alone.  In the tails the
exact functions' errors and their arguments' roundings, in units of 2^-24, with one
each for the products behind them."""
import math

import ffn_bounds
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


def f32_inputs(T, H, F, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, k=1.0: torch.randn(s, generator=gen, device="cuda") * k  # noqa: E731
    return n(T, H), n(F, H, k=H ** -0.5), n(F, H, k=H ** -0.5), n(T, F, k=0.0625)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("T,H,F", [(1, 4096, 300), (3, 2001, 700), (8, 520, 640), (20, 1000, 257), (32, 2048, 1024), (33, 512, 300),
                                   (64, 256, 512), (175, 193, 5239), (300, 1001, 333), (1247, 72, 993), (2305, 2296, 130)])
def test_f32_errors(sf, T, H, F, act):
    x, wg, wu, dh = f32_inputs(T, H, F, T + H)
    want = ffn_bounds.expected(x, wg, wu, act, dh)
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act=act, want=("dx", "dw", "h"))
    off = {n: ffn_bounds.share(getattr(r, n), want[n]) for n in want}
    off["forward"] = ffn_bounds.share(sf.sf_gated_ffn(x, wg, wu, act=act), want["h"])
    assert all(v <= 1 for v in off.values()), off


@pytest.mark.parametrize("T", [1, 8, 20, 33, 300])
def test_f32_sums_of_the_lower_parts(sf, T):
    """h = relu(g) with g a sum whose upper parts cancel: of third parts of x, of third parts of the weights, and
    of products of second parts.  256 terms of size 1 whose sums in f32 are off by 256 2^-24 = 2^-16 at most;
    the sums are 2^-13 (128 2^-20) and 2^-11.1 (64 (2^-8.5)^2, 1.8 2^-9 each)."""
    H, F = 264, 72
    x, wg, wu = torch.zeros((T, H), device="cuda"), torch.zeros((F, H), device="cuda"), torch.zeros((F, H), device="cuda")
    x[:, 256] = 1
    wu[:, 256] = 1
    low, near = 1 + 2.0 ** -8 + 2.0 ** -20, 1 + 2.0 ** -8
    x[:, 0:256:2], x[:, 1:256:2] = low, near
    wg[:, 0:256:2], wg[:, 1:256:2] = 1, -1
    h = sf.sf_gated_ffn(x, wg, wu, act="relu")
    assert bool(((h - 2.0 ** -13).abs() <= 2.0 ** -16).all())
    x[:, 0:256:2], x[:, 1:256:2] = 1, -1
    wg[:, 0:256:2], wg[:, 1:256:2] = low, near
    h = sf.sf_gated_ffn(x, wg, wu, act="relu")
    assert bool(((h - 2.0 ** -13).abs() <= 2.0 ** -16).all())
    a = 1.8 * 2.0 ** -9
    for k, (v, w) in enumerate(((1 + a, 1 + a), (1 + a, -1.0), (1.0, -1 - a), (1.0, 1.0))):
        x[:, k:256:4], wg[:, k:256:4] = v, w
    want = (x[0].double() * wg[0].double()).sum()
    assert float(want) > 2.0 ** -11.2
    h = sf.sf_gated_ffn(x, wg, wu, act="relu")
    assert bool(((h.double() - want).abs() <= 2.0 ** -16).all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("T", [1, 7, 40])
def test_f32_tails(sf, T, act):
    """g and u are single products, exact in every form; values in the normal range of f32."""
    H, F = 64, 3001
    g = torch.linspace(-8 if act == "gelu_tanh" else -12, 3, F, device="cuda")
    x, dh = torch.zeros((T, H), device="cuda"), torch.zeros((T, F), device="cuda")
    x[:, 0] = x[:, 1] = 1
    dh[0] = 1
    wg, wu = torch.zeros((F, H), device="cuda"), torch.zeros((F, H), device="cuda")
    wg[:, 0], wu[:, 1] = g, -3.0
    a, slope, size, own = ffn_bounds.act64(g.double(), act)
    unit = ffn_bounds.UNIT
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act=act, want=("dw", "h"))
    for got, want, near in ((sf.sf_gated_ffn(x, wg, wu, act=act)[T - 1], -3 * a, 3 * a.abs()), (r.h[T - 1], -3 * a, 3 * a.abs()),
                            (r.dw_up[:, 1], a, a.abs()), (r.dw_gate[:, 0], -3 * slope, 3 * size)):
        bound = (own + 2) * unit * near
        off = (got.double() - want).abs()
        assert bool((off <= bound).all()), (float((off / bound).max()), float(g[int((off / bound).nan_to_num().argmax())]))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [601, 20011, 65537])
def test_long_sums_of_one_sign(sf, T, dtype):
    """Weights' gradients in f32 from 16-bit inputs, summed over many tokens: 16 products at a time, each sum cut off
    by 2^-23 of it at most.  du is d itself (relu of 1), exact; the products are exact in f32."""
    H, F, t = 64, 72, TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = (1 + torch.randint(0, 128, (T, H), generator=gen, device="cuda") / 128).to(t)
    x[:, 0] = 1
    dh = (1 + torch.randint(0, 64, (T, F), generator=gen, device="cuda") / 64).to(t)
    wg, wu = torch.zeros((F, H), dtype=t, device="cuda"), torch.zeros((F, H), dtype=t, device="cuda")
    wg[:, 0] = wu[:, 0] = 1
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act="relu", want=("dw",), dw_dtype=torch.float32)
    want = dh.double().t() @ x.double()
    for got in (r.dw_gate, r.dw_up):
        assert bool(((got.double() - want).abs() <= (T / 16 + 2) * 2.0 ** -23 * want).all())


@pytest.mark.parametrize("T,H,F", [(257, 64, 72), (5003, 136, 200), (65537, 64, 72), (65537, 520, 1304), (300007, 72, 520)])
def test_long_f32_sums_do_not_drift(sf, T, H, F):
    """The same in runs of 256 tokens that are added in f32.  A run's partial sums are half of it on the average:
    8 2^-23 of it, one more for its last step; the n runs' additions round by 2^-24 of a partial sum, evenly spread and
    at random, a deviation of 2^-24 n^1/2 / 3: six of them are 2^-23 n^1/2.  Over all elements these cancel."""
    t = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(T + F)
    x = (1 + torch.randint(0, 128, (T, H), generator=gen, device="cuda") / 128).to(t)
    x[:, 0] = 1
    dh = (1 + torch.randint(0, 64, (T, F), generator=gen, device="cuda") / 64).to(t)
    wg, wu = torch.zeros((F, H), dtype=t, device="cuda"), torch.zeros((F, H), dtype=t, device="cuda")
    wg[:, 0] = wu[:, 0] = 1
    was = [torch.randn((F, H), generator=gen, device="cuda") for _ in range(2)]
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act="relu", want=("dw",), dw_dtype=torch.float32)
    more = sf.sf_gated_ffn_grad(x, wg, wu, dh, act="relu", dw_gate=was[0].clone(), dw_up=was[1].clone(), accumulate=True, want=())
    want = sum(dh[a:a + 16384].double().t() @ x[a:a + 16384].double() for a in range(0, T, 16384))
    for got, again, before in ((r.dw_gate, more.dw_gate, was[0]), (r.dw_up, more.dw_up, was[1])):
        off = (got.double() - want) / want
        assert float(off.abs().max()) <= (9 + (T / 256) ** 0.5) * 2.0 ** -23 and abs(float(off.mean())) <= 10 * 2.0 ** -23
        assert torch.equal(again, got + before)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [601, 20011])
def test_f32_weight_gradients_of_many_tokens(sf, T, dtype):
    """Mixed signs, against dg and du rounded once to the type (half a step each, at random) and sums as above,
    whose partial sums grow as the root of their length: 2/3 T / 16 2^-23 of the root of the squares' sum."""
    H, F, t = 96, 136, TYPES[dtype]
    x, wg, wu, dh = (v.to(t) for v in f32_inputs(T, H, F, T))
    want = ffn_bounds.expected(x, wg, wu, "silu", dh)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    a, slope, _ = act64(g, "silu")
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dw",), dw_dtype=torch.float32)
    for name, got, q in (("dw_gate", r.dw_gate, dh.double() * u * slope), ("dw_up", r.dw_up, dh.double() * a)):
        # own: f32 sums before the rounding, the hardware's exponential (2^-18), and what is below the type's numbers
        size = ffn_bounds.squares(q.t(), x.double())
        each = torch.finfo(t).eps / 2 + 2.0 ** -18 + T / 24 * 2.0 ** -23
        least = TINY[dtype] * ffn_bounds.squares(torch.ones_like(q).t(), x.double())
        bound = each * size + want[name][1] + least
        assert ffn_bounds.share(got, (want[name][0], bound)) <= 1


def test_f16_gradients_leave_the_range(sf):
    """dg and du are f16 between the products: above 65504 infinite, below 2^-25 zero, also for weights in f32."""
    T, H, F = 70, 64, 96
    t = torch.float16
    x, wg, wu = torch.zeros((T, H), dtype=t, device="cuda"), torch.zeros((F, H), dtype=t, device="cuda"), torch.zeros((F, H), dtype=t, device="cuda")
    x[:, 0] = x[:, 1] = 1
    wg[:, 0], wu[:, 1] = 2, 1000
    dh = torch.zeros((T, F), dtype=t, device="cuda")
    dh[0, :40], dh[0, 40:] = 100, 2.0 ** -14
    wu[50:, 1] = 2.0 ** -13
    for dt in (t, torch.float32):
        r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dw",), dw_dtype=dt)
        assert bool((r.dw_gate[:40, 0] == float("inf")).all()) and bool(r.dw_up[:40, 0].isfinite().all())
        assert bool((r.dw_gate[40:50, 0] > 0).all()) and bool((r.dw_gate[50:, 0] == 0).all())
        assert bool((r.dw_up[40:, 0] > 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(1, 16), (3, 9)])
def test_many_features_of_few_tokens(sf, T, H, dtype):
    """More features than the form for a few tokens takes: one row for each, its gradients against the formulas."""
    F, t = 65535 * 8 + 9, TYPES[dtype]
    x, wg, wu, dh = (v.to(t) for v in f32_inputs(T, H, F, T))
    st = sf.new_status("cuda")
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dx", "dw", "h"), status=st)
    h = sf.sf_gated_ffn(x, wg, wu, status=st)
    assert int(st.item()) == 0
    want = ffn_bounds.expected(x, wg, wu, "silu", dh)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    a, slope, _ = act64(g, "silu")
    d = dh.double()
    half = 0.0 if dtype == "f32" else torch.finfo(t).eps / 2
    tiny = 0.0 if dtype == "f32" else TINY[dtype]
    dg, du = d * u * slope, d * a
    each = half + (0 if dtype == "f32" else 2.0 ** -18)  # dg and du as they are stored
    through = {"dx": torch.hypot(ffn_bounds.squares(dg, wg.double()), ffn_bounds.squares(du, wu.double())),
               "dw_gate": ffn_bounds.squares(dg.t(), x.double()), "dw_up": ffn_bounds.squares(du.t(), x.double())}
    # sums of all features' products, 16 bits: 2 F / 16 steps of 2^-23 of partial sums that grow as the root of their length
    steps = {"dx": 0.0 if dtype == "f32" else 2 * F / 24 * 2.0 ** -23}
    for name, got in (("h", h), ("h", r.h), ("dx", r.dx), ("dw_gate", r.dw_gate), ("dw_up", r.dw_up)):
        value, bound = want[name]
        bound = bound + half * value.abs() + tiny * (1 + F ** 0.5)
        if name in through:
            bound = bound + (each + steps.get(name, 0.0)) * through[name]
        assert ffn_bounds.share(got, (value, bound)) <= 1, name


@pytest.mark.parametrize("T", [8, 33, 300])
def test_f32_small_values(sf, T):
    """Values of 2^-109 keep all their bits in every form, as tokens, as weights and as gradients."""
    H, F = 64, 136
    gen = torch.Generator(device="cuda").manual_seed(T)
    small = (1 + torch.randint(0, 1 << 23, (T, F), generator=gen, device="cuda") * 2.0 ** -23) * 2.0 ** -109
    x, wg, wu = torch.zeros((T, H), device="cuda"), torch.zeros((F, H), device="cuda"), torch.zeros((F, H), device="cuda")
    x[:, 0], x[:, 1] = small[:, 0], 1
    wg[:, 0], wu[:, 1] = 2.0 ** 100, 1
    want = small[:, :1] * 2.0 ** 100
    assert torch.equal(sf.sf_gated_ffn(x, wg, wu, act="relu"), want.expand(T, F))
    x[:, 0], wg[:, 0] = 2.0 ** 100, small[0, 0]
    assert torch.equal(sf.sf_gated_ffn(x, wg, wu, act="relu"), want[:1].expand(T, F))
    x[:, 0], wg[:, 0] = 1, 1  # du = dh, dg = 0 (u is 0)
    wu[:] = 0
    x[:, 1] = torch.eye(T, device="cuda")[0] * 2.0 ** 100
    r = sf.sf_gated_ffn_grad(x, wg, wu, small, act="relu")
    assert torch.equal(r.dw_up[:, 1], small[0] * 2.0 ** 100)
