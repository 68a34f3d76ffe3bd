"""sf_gated_ffn and sf_gated_ffn_grad against the formulas in 64 bits.

Bounds.  A sum of n products in 32 bits, in any order and with partial sums cut
off instead of rounded, is within 2 (n + 16) 2^-24 of the sum of the products'
magnitudes.  An activation of g and its derivative move with g by at most 1.3
times as much, and are themselves good to 2^-18 of max(|g|, 1) times their size
bound (1.2 |g| and 1.2) where 16 bits are stored.  Each stored value is rounded
once: half a step, eps / 2 of it, and the smallest number of its type.  dg and du
are stored between the products, and that rounding goes through them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def mat(gen, n, m, dtype, scale, ld=None, offset=0):
    """A matrix of the generator's values in a buffer of its own: (buffer, view)."""
    ld = m if ld is None else ld
    flat = torch.full((offset + n * ld + 64,), 7.0, dtype=TYPES[dtype], device="cuda")
    t = torch.as_strided(flat, (n, m), (ld, 1), offset)
    t.copy_(torch.randn((n, m), generator=gen, device="cuda") * scale)
    return flat, t


def act64(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    if act == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    return g.clamp(min=0), (g > 0).double()


def sums(n):
    return 2 * (n + 16) * 2.0 ** -24


def reference(x, wg, wu, act, dtype, dh=None):
    """Values and their bounds: {name: (value, bound)}."""
    half, tiny = torch.finfo(TYPES[dtype]).eps / 2, TINY[dtype]
    x, wg, wu = x.double(), wg.double(), wu.double()
    T, H, F = x.shape[0], x.shape[1], wg.shape[0]
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = sums(H) * (x.abs() @ wg.abs().t()), sums(H) * (x.abs() @ wu.abs().t())
    a, slope = act64(g, act)
    if act == "relu":  # its slope jumps at 0: where the sign is not certain, either is right
        jump = (g.abs() <= eg).double()
    else:
        jump = torch.zeros_like(g)
    own = 2.0 ** -18 * 1.2 * g.abs().clamp(min=1)
    ea = 1.3 * eg + own * g.abs().clamp(max=1) + 2.0 ** -18 * a.abs()
    es = 1.3 * eg + own + jump
    r = {}
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + ea * eu
    r["h"] = (h, eh + half * (h.abs() + eh) + tiny)
    if dh is None:
        return r
    d = dh.double()
    dg, du = d * u * slope, d * a
    edg = d.abs() * (u.abs() * es + eu * (slope.abs() + es))
    edu = d.abs() * ea
    edg = edg + half * (dg.abs() + edg) + tiny
    edu = edu + half * (du.abs() + edu) + tiny
    value = dg @ wg + du @ wu
    e = edg @ wg.abs() + edu @ wu.abs() + sums(2 * F) * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs())
    r["dx"] = (value, e + half * (value.abs() + e) + tiny)
    for name, q, eq in (("dw_gate", dg, edg), ("dw_up", du, edu)):
        value = q.t() @ x
        e = eq.t() @ x.abs() + sums(T) * ((q.abs() + eq).t() @ x.abs())
        r[name] = (value, e + half * (value.abs() + e) + tiny)
    return r


def within(got, want, name):
    value, bound = want
    off = (got.double() - value).abs()
    worst = float((off / bound).max()) if off.numel() else 0.0
    assert bool((off <= bound).all()), f"{name}: {worst:.3f} of the bound"


def inputs(T, H, F, dtype, seed, grad=False, pad=0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = mat(gen, T, H, dtype, 1.0, H + pad, offset)[1]
    wg, wu = (mat(gen, F, H, dtype, H ** -0.5, H + pad, offset)[1] for _ in range(2))
    dh = mat(gen, T, F, dtype, 0.0625, F + pad, offset)[1] if grad else None
    return x, wg, wu, dh


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 4096, 300), (2, 8, 16), (3, 1000, 1001), (5, 33, 7), (8, 72, 640), (16, 256, 128),
          (17, 257, 129), (48, 2048, 1024), (64, 64, 8), (100, 520, 1000), (128, 128, 128), (129, 130, 191),
          (255, 96, 65), (256, 1024, 2048), (257, 1001, 333), (300, 512, 700), (513, 64, 1100), (1357, 200, 2731),
          (2049, 136, 72), (2305, 2296, 1301), (8200, 40, 50), (33, 64, 3001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,F", SHAPES)
def test_forward(sf, T, H, F, dtype):
    act = ACTS[(T + F) % 4]
    x, wg, wu, _ = inputs(T, H, F, dtype, T + H)
    st = sf.new_status("cuda")
    h = sf.sf_gated_ffn(x, wg, wu, act=act, status=st)
    assert int(st.item()) == 0
    within(h, reference(x, wg, wu, act, dtype)["h"], "h")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,F", SHAPES)
def test_gradient(sf, T, H, F, dtype):
    act = ACTS[(T + H) % 4]
    x, wg, wu, dh = inputs(T, H, F, dtype, T + F, grad=True)
    st = sf.new_status("cuda")
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act=act, want=("dx", "dw", "h"), status=st)
    assert int(st.item()) == 0
    for name, want in reference(x, wg, wu, act, dtype, dh).items():
        within(getattr(r, name), want, name)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations(sf, act, dtype):
    x, wg, wu, dh = inputs(70, 64, 96, dtype, 5, grad=True)
    wg.mul_(4)  # far into both tails
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act=act, want=("dx", "dw", "h"))
    for name, want in reference(x, wg, wu, act, dtype, dh).items():
        within(getattr(r, name), want, name)
    within(sf.sf_gated_ffn(x, wg, wu, act=act), reference(x, wg, wu, act, dtype)["h"], "h")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 6, 40, 300])
@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (3, 0), (8, 1), (0, 5)])
def test_spacing_and_surroundings(sf, T, pad, offset, dtype):
    """Rows of any spacing and start; what lies around the outputs stays."""
    H, F = 136, 200
    x, wg, wu, dh = inputs(T, H, F, dtype, 11 + pad + offset, grad=True, pad=pad, offset=offset)
    ref = reference(x, wg, wu, "silu", dtype, dh)
    gen = torch.Generator(device="cuda").manual_seed(1)
    outs = {n: mat(gen, *s, dtype, 1.0, s[1] + pad, offset) for n, s in
            (("h", (T, F)), ("dx", (T, H)), ("dw_gate", (F, H)), ("dw_up", (F, H)))}
    before = {n: flat.clone() for n, (flat, _) in outs.items()}
    sf.sf_gated_ffn(x, wg, wu, h=outs["h"][1])
    within(outs["h"][1], ref["h"], "h")
    first = outs["h"][1].clone()
    sf.sf_gated_ffn_grad(x, wg, wu, dh, **{n: t for n, (_, t) in outs.items()})
    for n, (flat, t) in outs.items():
        within(t, ref[n], n)
        torch.as_strided(before[n], t.shape, t.stride(), t.storage_offset()).copy_(t)
        assert torch.equal(before[n], flat), n
    within(first, ref["h"], "h")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 5, 600])
def test_accumulate_and_f32_weights(sf, T, dtype):
    H, F = 320, 264
    x, wg, wu, dh = inputs(T, H, F, dtype, 21, grad=True)
    ref = reference(x, wg, wu, "silu", dtype, dh)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    for dt in (torch.float32, TYPES[dtype]):
        a, b = torch.randn((F, H), device="cuda").to(dt), torch.randn((F, H), device="cuda").to(dt)
        was = {"dw_gate": a.double(), "dw_up": b.double()}
        r = sf.sf_gated_ffn_grad(x, wg, wu, dh, dw_gate=a, dw_up=b, accumulate=True, want=())
        assert r.dx is None and r.h is None
        for n in was:
            value, bound = ref[n]
            # the reference's own rounding covers that of the product, not that of the sum
            within(getattr(r, n), (value + was[n], bound + 2 * eps * (was[n].abs() + value.abs())), n)
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dw",), dw_dtype=torch.float32)
    assert r.dw_gate.dtype == torch.float32
    for n in ("dw_gate", "dw_up"):
        within(getattr(r, n), ref[n], n)


@pytest.mark.parametrize("want", [("dx",), ("dw",), ("h",)])
def test_single_outputs(sf, want):
    x, wg, wu, dh = inputs(77, 128, 192, "bf16", 3, grad=True)
    every = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dx", "dw", "h"))
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=want)
    for n in ("dx", "dw_gate", "dw_up", "h"):
        v = getattr(r, n)
        assert v is None or torch.equal(v, getattr(every, n))
        assert (v is not None) == (n[:2] in want or n in want)


@pytest.mark.parametrize("dtype", TYPES)
def test_differences(sf, dtype):
    """The gradient of a sum of h against differences in 64 bits: one direction through all inputs."""
    x, wg, wu, dh = inputs(30, 48, 56, dtype, 31, grad=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    dirs = [torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) for t in (x, wg, wu)]

    def f(e):
        a, b, c = (t.double() + e * v for t, v in zip((x, wg, wu), dirs))
        return float((act64(a @ b.t(), "gelu")[0] * (a @ c.t()) * dh.double()).sum())

    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, act="gelu")
    got = sum(float((getattr(r, n).double() * v).sum()) for n, v in zip(("dx", "dw_gate", "dw_up"), dirs))
    ref = reference(x, wg, wu, "gelu", dtype, dh)
    bound = sum(float((ref[n][1] * v.abs()).sum()) for n, v in zip(("dx", "dw_gate", "dw_up"), dirs))
    e = 1e-4  # the third derivative times e^2 is some 1e-6 of the first
    numeric = (8 * (f(e) - f(-e)) - (f(2 * e) - f(-2 * e))) / (12 * e)
    assert abs(got - numeric) <= bound + 1e-6 * abs(numeric)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [3, 8, 40, 400])
def test_infinite_and_nan_tokens(sf, T, dtype):
    """A token's NaN or infinity goes to its own rows and to the weights' gradients, nowhere else."""
    x, wg, wu, dh = inputs(T, 96, 130, dtype, 41, grad=True)
    clean = sf.sf_gated_ffn(x, wg, wu)
    ref = sf.sf_gated_ffn_grad(x, wg, wu, dh)
    x[1, 5] = float("nan")
    h = sf.sf_gated_ffn(x, wg, wu)
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh)
    keep = torch.arange(T, device="cuda") != 1
    assert bool(h[1].isnan().all()) and torch.equal(h[keep], clean[keep])
    assert bool(r.dx[1].isnan().all()) and torch.equal(r.dx[keep], ref.dx[keep])
    assert bool(r.dw_gate.isnan().all()) and bool(r.dw_up.isnan().all())
    x[1, 5] = float("inf")
    h = sf.sf_gated_ffn(x, wg, wu, act="relu")
    g, u = wg[:, 5].double(), wu[:, 5].double()
    if dtype == "f32" and T > 32:  # products by parts: an infinity meets parts that are 0
        assert not bool(h[1].isfinite().any()) and bool(h[keep].isfinite().all())
        return
    assert bool((h[1][(g > 0) & (u > 0)] == float("inf")).all())
    assert bool((h[1][(g > 0) & (u < 0)] == float("-inf")).all())


def test_calls_repeat(sf):
    for T, H, F, dtype in ((1, 2048, 1000, "bf16"), (48, 2048, 1024, "bf16"), (700, 520, 900, "f16"), (90, 64, 64, "f32")):
        x, wg, wu, dh = inputs(T, H, F, dtype, 51, grad=True)
        h, r = sf.sf_gated_ffn(x, wg, wu), sf.sf_gated_ffn_grad(x, wg, wu, dh)
        for _ in range(5):
            assert torch.equal(sf.sf_gated_ffn(x, wg, wu), h)
            o = sf.sf_gated_ffn_grad(x, wg, wu, dh)
            assert all(torch.equal(getattr(o, n), getattr(r, n)) for n in ("dx", "dw_gate", "dw_up"))


@pytest.mark.parametrize("T,H,F,dtype", [(4, 512, 600, "bf16"), (333, 264, 500, "bf16"), (50, 71, 90, "f16")])
def test_graph_and_streams(sf, T, H, F, dtype):
    x, wg, wu, dh = inputs(T, H, F, dtype, 61, grad=True)
    h = torch.empty((T, F), dtype=TYPES[dtype], device="cuda")
    outs = dict(dx=torch.empty_like(x), dw_gate=torch.empty((F, H), dtype=TYPES[dtype], device="cuda"),
                dw_up=torch.empty((F, H), dtype=TYPES[dtype], device="cuda"))

    def call(**kw):
        sf.sf_gated_ffn(x, wg, wu, h=h, **kw)
        sf.sf_gated_ffn_grad(x, wg, wu, dh, **outs, **kw)

    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    x.copy_(torch.randn(T, H, device="cuda"))
    dh.copy_(torch.randn(T, F, device="cuda"))
    call()
    want = [t.clone() for t in (h, *outs.values())]
    for t in (h, *outs.values()):
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (h, *outs.values())))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for t in (h, *outs.values()):
        t.zero_()
    torch.cuda.synchronize()
    one = sf.sf_gated_ffn(x, wg, wu, stream=a)  # two calls at once, workspaces of their own
    two = sf.sf_gated_ffn_grad(x, wg, wu, dh, stream=b)
    torch.cuda.synchronize()
    assert torch.equal(one, want[0]) and torch.equal(two.dx, want[1]) and torch.equal(two.dw_up, want[3])


def test_no_tokens(sf):
    x, wg, wu, dh = inputs(1, 40, 50, "bf16", 71, grad=True)
    assert sf.sf_gated_ffn(x[:0], wg, wu).shape == (0, 50)
    r = sf.sf_gated_ffn_grad(x[:0], wg, wu, dh[:0])
    assert r.dx.shape == (0, 40) and not r.dw_gate.any() and not r.dw_up.any()
    a, b = torch.ones((50, 40), device="cuda"), torch.ones((50, 40), device="cuda")
    sf.sf_gated_ffn_grad(x[:0], wg, wu, dh[:0], dw_gate=a, dw_up=b, accumulate=True)
    assert bool((a == 1).all()) and bool((b == 1).all())
    sf.sf_gated_ffn_grad(x[:0], wg, wu, dh[:0], dw_gate=a, dw_up=b)
    assert not a.any() and not b.any()


@pytest.mark.parametrize("T,H,F,dtype", [(180001, 64, 12296, "bf16"), (60001, 64, 12296, "f32")])
def test_long(sf, T, H, F, dtype):
    """Tensors whose offsets pass 32 bits: the last rows, and the last features' gradients summed over all tokens."""
    x, wg, wu, dh = inputs(T, H, F, dtype, 91, grad=True)
    st = sf.new_status("cuda")
    r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dx", "dw", "h"), status=st)
    h = sf.sf_gated_ffn(x, wg, wu, status=st)
    assert int(st.item()) == 0
    for at in (slice(0, 40), slice(T - 40, T)):
        ref = reference(x[at], wg, wu, "silu", dtype, dh[at])
        for name, got in (("h", h), ("h", r.h), ("dx", r.dx)):
            within(got[at], ref[name], name)
    few = slice(F - 5, F)
    total = None
    for a in range(0, T, 60000):
        ref = reference(x[a:a + 60000], wg[few], wu[few], "silu", dtype, dh[a:a + 60000, few])
        part = {n: ref[n] for n in ("dw_gate", "dw_up")}
        total = part if total is None else {n: (total[n][0] + part[n][0], total[n][1] + part[n][1]) for n in part}
    for n, got in (("dw_gate", r.dw_gate), ("dw_up", r.dw_up)):
        within(got[few], (total[n][0], total[n][1] * (1 + T / 60000)), n)  # sums as long as all tokens


def test_refusals(sf):
    x, wg, wu, dh = inputs(8, 64, 72, "bf16", 81, grad=True)
    before = sf.launch_count()
    with pytest.raises(ValueError):
        sf.sf_gated_ffn(x, wg, wu, act="tanh")
    for bad in ((x[:, :63], wg, wu), (x, wg[:5], wu), (x, wg.float(), wu), (x, wg, wu[:, :60]), (x.float(), wg, wu)):
        with pytest.raises(ValueError):
            sf.sf_gated_ffn(*bad)
    with pytest.raises(TypeError):
        sf.sf_gated_ffn(x.double(), wg, wu)
    with pytest.raises(TypeError):
        sf.sf_gated_ffn(x, wg.t().contiguous().t(), wu)
    with pytest.raises(ValueError):
        sf.sf_gated_ffn(x, wg, wu, h=torch.empty((8, 71), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        sf.sf_gated_ffn(x, wg, wu, h=torch.empty((8, 72), device="cuda"))
    with pytest.raises(ValueError):
        sf.sf_gated_ffn_grad(x, wg, wu, dh[:7])
    with pytest.raises(ValueError):
        sf.sf_gated_ffn_grad(x, wg, wu, dh, accumulate=True)
    with pytest.raises(ValueError):
        sf.sf_gated_ffn_grad(x, wg, wu, dh, dw_gate=torch.empty_like(wg))
    with pytest.raises(ValueError):
        sf.sf_gated_ffn_grad(x, wg, wu, dh, dw_dtype=torch.float16)
    with pytest.raises(sf.SFError) as err:
        sf.sf_gated_ffn_grad(x, wg, wu, dh, want=())
    assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError) as err:
        sf.sf_gated_ffn_grad(x, wg, wu, dh, dx=x)
    assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError) as err:
        sf.sf_gated_ffn_grad(x, wg, wu, dh, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert err.value.code == sf.SF_EWORKSPACE
    assert sf.launch_count() == before
