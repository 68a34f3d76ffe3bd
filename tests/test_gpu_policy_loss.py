"""sf_policy_loss against the formulas in 64 bits, and its gradient also
against differences of the loss.

Tolerances, from the arithmetic: the kernel's exponentials are good to 2^-22
and its sums of S terms add at most a few hundred roundings of 2^-24, so log S
is within 1e-5; z_y - m rounds once.  What a log-probability's error does to
the loss and to the gradient's factor is at most the error times their own
derivative."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LO, HI, BETA, TAU = 0.2, 0.25, 0.1, 0.8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9, "f16": 2.0 ** -12}  # of values in [0.5, 1): half a unit, doubled below
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -25}
DLP = 1e-5  # error of a log-probability beside that of its largest term


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def make(N, V, dtype, seed, ld=None, offset=0, spread=2.0):
    """Inputs on the host (64-bit values that the type holds), logits on the GPU with rows `ld` apart."""
    rng = np.random.default_rng(seed)
    ld = V if ld is None else ld
    flat = torch.zeros(offset + N * ld, dtype=TYPES[dtype], device="cuda")
    z = torch.as_strided(flat, (N, V), (ld, 1), offset)
    z.copy_(torch.from_numpy(spread * rng.standard_normal((N, V))))
    x = z.double().cpu().numpy()
    y = rng.integers(0, V, N)
    A = rng.standard_normal(N)
    lp = logprob(x * TAU)[np.arange(N), y]
    # ratios on both sides of both bounds (logs -0.22 and 0.22) and far enough from them
    old = (lp - rng.choice([-0.5, -0.1, 0.05, 0.6], N)).astype(np.float32)
    ref = (lp + 0.3 * rng.standard_normal(N)).astype(np.float32)
    w = rng.uniform(0.5, 1.5, N).astype(np.float32)
    return z, dict(x=x, y=y, A=A.astype(np.float32), old=old, ref=ref, w=w)


def logprob(x):
    m = x.max(1, keepdims=True)
    return x - m - np.log(np.exp(x - m).sum(1, keepdims=True))


def reference(h, beta=BETA, ref=True, g=1.0, tau=TAU):
    x, y, w = h["x"] * tau, h["y"], h["w"].astype(np.float64)
    on = w != 0
    n = np.arange(len(y))
    with np.errstate(all="ignore"):
        logp = logprob(x)
        lp = logp[n, y]
        A, u = h["A"].astype(np.float64), h["ref"].astype(np.float64) - lp
        r = np.exp(lp - h["old"].astype(np.float64))
        held = np.clip(r, 1 - LO, 1 + HI)
        clipped = held * A < r * A
        pg = -np.minimum(r * A, held * A)
        kl = np.expm1(u) - u if ref else np.zeros_like(u)
        loss = pg + (beta * kl if ref else 0.0)
        c = np.where(clipped, 0.0, -r * A) - (beta * np.expm1(u) if ref else 0.0)
        slope = np.abs(r * A) + (beta * np.exp(u) if ref else 0.0)
        f = np.where(on, c * w * g * tau, 0.0)
        p = np.exp(logp)
        d = -f[:, None] * p
        d[n, y] += f
    terms = np.stack([loss, pg, kl, clipped.astype(np.float64)])
    zero = lambda v: np.where(on, v, 0.0)  # noqa: E731
    stats = np.where(on, terms * w, 0.0).sum(1)
    return dict(logp=zero(lp), loss=zero(loss), slope=zero(slope), stats=stats, d=d, p=np.where(on[:, None], p, 0.0),
                f=f, absf=np.where(on, slope * np.abs(w * g) * tau, 0.0), w=np.abs(w), terms=zero(np.abs(terms)))


def on_gpu(h):
    t = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    return dict(target=t(h["y"]), old_logp=t(h["old"]), advantage=t(h["A"]), ref_logp=t(h["ref"]), weight=t(h["w"]))


def call(sf, z, h, kl_coef=BETA, **kw):
    st = sf.new_status("cuda")
    r = sf.sf_policy_loss(z, clip=(LO, HI), kl_coef=kl_coef, inv_temperature=TAU, status=st, **{**on_gpu(h), **kw})
    torch.cuda.synchronize()
    return r, int(st.item())


def check(r, e, dtype, grad=True):
    got = lambda t: t.double().cpu().numpy()  # noqa: E731
    lp = np.where(np.isfinite(e["logp"]), e["logp"], 0.0)
    dlp = DLP + 4e-7 * np.abs(lp)
    fin = np.isfinite(e["logp"])
    assert np.array_equal(np.isfinite(got(r.logp)), fin)
    assert np.all(np.abs(got(r.logp) - e["logp"])[fin] <= dlp[fin])
    bound = dlp * (1 + e["slope"]) + 1e-6 * np.abs(e["loss"])
    assert np.all(np.abs(got(r.token_loss) - e["loss"]) <= bound)
    kl_bound = dlp * (1 + e["slope"] / BETA)
    total = [(bound * e["w"]).sum(), (bound * e["w"]).sum(), (kl_bound * e["w"]).sum(), 0.0]
    for q in range(4):
        assert abs(got(r.stats)[q] - e["stats"][q]) <= total[q] + 1e-6 * (e["terms"][q] * e["w"]).sum() + 1e-12, q
    if not grad:
        return
    d = got(r.dlogits)
    at = np.zeros_like(e["p"])
    at[np.arange(len(e["f"])), e["y"]] = 1.0
    # the factor's error, the probability's, and one rounding to the type
    err = 4 * dlp[:, None] * (e["absf"] + np.abs(e["f"]))[:, None] * (e["p"] + at)
    err += 1e-6 * np.abs(e["f"])[:, None] * (e["p"] + at)
    assert np.all(np.abs(d - e["d"]) <= err + 2.1 * HALF_ULP[dtype] * np.abs(e["d"]) + TINY[dtype])


SIZES = [(1, 1), (1, 2), (3, 7), (2, 33), (5, 1000), (40, 4099), (700, 257), (1, 65536), (3, 50001), (9, 32768),
         (2, 131072), (3, 262144), (2, 300007), (2, 136001), (90, 50001), (400, 8), (333, 5), (310, 8192), (317, 16387),
         (650, 4099)]


@pytest.mark.parametrize("N,V", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_loss_and_gradient(sf, N, V, dtype):
    z, h = make(N, V, dtype, N + V)
    if N > 4:
        h["w"][::3] = 0.0
    e = reference(h)
    e["y"] = h["y"]
    r, st = call(sf, z, h, grad=True)
    assert st == 0
    check(r, e, dtype)
    f, st = call(sf, z, h)  # without gradients: the same numbers
    assert st == 0 and f.dlogits is None
    check(f, e, dtype, grad=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ld,offset", [(1000, 1008, 0), (1000, 1001, 0), (1001, 1001, 1), (8190, 8200, 3), (5, 9, 2),
                                         (40001, 40003, 5)])
@pytest.mark.parametrize("N", [7, 320])
def test_strides_and_offsets(sf, dtype, V, ld, offset, N):
    z, h = make(N, V, dtype, V, ld, offset)
    e = reference(h)
    e["y"] = h["y"]
    r, _ = call(sf, z, h, grad=True)
    check(r, e, dtype)
    # gradients with a row spacing of their own, nothing written between the rows
    flat = torch.full((4 + N * (V + 3),), 7.0, dtype=TYPES[dtype], device="cuda")
    d = torch.as_strided(flat, (N, V), (V + 3, 1), 4)
    r, _ = call(sf, z, h, dlogits=d)
    check(r, e, dtype)
    rest = flat.clone()
    torch.as_strided(rest, (N, V), (V + 3, 1), 4).fill_(7.0)
    assert bool((rest == 7.0).all())
    # in place
    r, _ = call(sf, z, h, dlogits=z)
    check(r, e, dtype)


@pytest.mark.parametrize("N,V", [(6, 50), (5, 9001), (4, 40000)])
def test_optional_inputs(sf, N, V):
    z, h = make(N, V, "f32", V)
    h["w"][:] = np.float32(1.0 / N)
    e = reference(h)
    e["y"] = h["y"]
    r, st = call(sf, z, h, weight=None, grad=True)
    assert st == 0
    check(r, e, "f32")
    e = reference(h, beta=0.0, ref=False, g=-3.0)
    e["y"] = h["y"]
    r, st = call(sf, z, h, ref_logp=None, grad=True, grad_out=torch.tensor([-3.0], device="cuda"))
    assert st == 0
    check(r, e, "f32")
    e = reference(h, beta=0.0)  # the KL term is reported, not charged
    e["y"] = h["y"]
    r, st = call(sf, z, h, kl_coef=0.0, grad=True)
    assert st == 0
    check(r, e, "f32")


@pytest.mark.parametrize("V", [64, 5000, 70001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [12, 700])
def test_masked_rows_are_not_read(sf, V, dtype, N):
    if N * V > 10 ** 7:
        V = 9001
    z, h = make(N, V, dtype, V)
    h["w"][[0, 3, 4, 11]] = 0.0
    h["w"][12:690] = 0.0  # a long run of them
    e = reference(h)
    e["y"] = h["y"]
    z[0] = math.nan
    z[3] = math.inf
    z[11] = -math.inf
    a = on_gpu(h)
    for k in ("old_logp", "advantage", "ref_logp"):
        a[k][3] = math.nan
    a["target"][4] = -1
    a.pop("weight")
    r, st = call(sf, z, h, grad=True, **a)
    assert st == 0
    check(r, e, dtype)
    assert not r.dlogits[[0, 3, 4, 11]].any() and not r.logp[[0, 3, 4, 11]].any()
    h["w"][:] = 0.0  # nothing left: no loss, no gradient
    r, st = call(sf, z, h, grad=True)
    assert st == 0 and not r.stats.any() and not r.dlogits.any()


@pytest.mark.parametrize("V", [64, 5000, 70001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N", [6, 330])
def test_ruled_out_tokens(sf, V, dtype, N):
    """-inf and the type's lowest value as masks, and a row of nothing but the latter."""
    V = V if N * V < 10 ** 7 else 9001
    z, h = make(N, V, dtype, V + 1)
    low = torch.finfo(TYPES[dtype]).min
    z[0, 1::2] = -math.inf
    z[1, : V // 2] = low
    z[2] = low
    z[3, :-1] = -math.inf
    z[4, 5:] = -math.inf
    h["y"][[0, 1, 2, 3, 4]] = [0, V - 1, 3, V - 1, 2]
    h["x"] = z.double().cpu().numpy()
    with np.errstate(all="ignore"):
        lp = logprob(h["x"] * TAU)[np.arange(N), h["y"]]
    h["old"] = (lp + 0.1).astype(np.float32)
    h["ref"] = (lp - 0.2).astype(np.float32)
    e = reference(h)
    e["y"] = h["y"]
    r, st = call(sf, z, h, grad=True)
    assert st == 0
    check(r, e, dtype)
    assert not r.dlogits[0, 1::2].any() and not r.dlogits[4, 5:].any()


@pytest.mark.parametrize("V", [64, 5000, 70001])
def test_chosen_token_ruled_out(sf, V):
    """Probability 0: ratio 0, no gradient (without a KL term)."""
    z, h = make(4, V, "f32", V + 2)
    z[1, 3] = -math.inf
    h["y"][1] = 3
    h["x"] = z.double().cpu().numpy()
    e = reference(h, beta=0.0, ref=False)
    e["y"] = h["y"]
    r, st = call(sf, z, h, ref_logp=None, grad=True)
    assert st == 0
    check(r, e, "f32")
    assert not r.dlogits[1].any()


@pytest.mark.parametrize("V", [64, 5000, 70001, 300001])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("N", [9, 400])
def test_faulty_rows_are_left_out(sf, V, grad, N):
    V = V if N * V < 10 ** 7 else 9001
    z, h = make(N, V, "bf16", V + 3)
    bad = h.copy()
    bad["w"] = h["w"].copy()
    bad["w"][[1, 2, 3]] = 0.0
    e = reference(bad)
    e["y"] = h["y"]
    z[1] = -math.inf
    z[2, V - 1] = math.nan
    z[3, V // 2] = math.inf
    r, st = call(sf, z, h, grad=grad)
    assert st == sf.SF_ST_NONFINITE
    check(r, e, "bf16", grad)
    a = on_gpu(h)
    a["target"][1], a["target"][2], a["target"][3] = V, -1, 1 << 40
    z[1:4] = 0.0
    r, st = call(sf, z, h, grad=grad, target=a["target"])
    assert st == sf.SF_ST_INDEX
    check(r, e, "bf16", grad)


@pytest.mark.parametrize("N,V", [(3, 11), (2, 5000)])
def test_gradient_against_differences(sf, N, V):
    """The loss along a direction: differences of step 0.01 have an error of
    about 1e-4 of the loss's third derivative, and 1e-6 / 0.02 of rounding."""
    z, h = make(N, V, "f32", 5 * V)
    rng = np.random.default_rng(1)
    D = torch.from_numpy(rng.standard_normal((N, V)).astype(np.float32)).cuda()
    step = 1e-2
    r, _ = call(sf, z, h, grad=True)
    slope = float((r.dlogits.double() * D.double()).sum())
    up, _ = call(sf, z + step * D, h)
    down, _ = call(sf, z - step * D, h)
    diff = (float(up.stats[0]) - float(down.stats[0])) / (2 * step)
    assert abs(diff - slope) <= 2e-3 * (1 + abs(slope))


@pytest.mark.parametrize("N,V", [(300, 1000), (40, 33000), (20000, 64)])
def test_same_bits_again_and_on_another_stream(sf, N, V):
    z, h = make(N, V, "bf16", V + N)
    a, _ = call(sf, z, h, grad=True)
    b, _ = call(sf, z, h, grad=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c, _ = call(sf, z, h, grad=True)
    d, _ = call(sf, z, h, grad=True, stream=s)
    for o in (b, c, d):
        for k in ("logp", "token_loss", "stats", "dlogits"):
            assert torch.equal(getattr(a, k), getattr(o, k)), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(3, 1000), (320, 1000), (3, 140000)])
@pytest.mark.parametrize("level", [1e36, -1e36, 3e38, -3e38])
def test_far_out_logits(sf, dtype, N, V, level):
    """Rows at the end of the type's range: what counts is the differences."""
    z, h = make(N, V, dtype, 17)
    z[1] = level
    z[1, V // 2:] = z[1, 0] * (0.5 if level > 0 else 1.125) if abs(level) < 1e38 else -level
    h["x"] = z.double().cpu().numpy()
    h["y"][1] = 3 if level > 0 or abs(level) < 1e38 else V - 1
    lp = logprob(h["x"] * TAU)[np.arange(N), h["y"]]
    h["old"][1] = lp[1] + 0.1
    h["ref"][1] = lp[1] - 0.2
    e = reference(h)
    e["y"] = h["y"]
    r, st = call(sf, z, h, grad=True)
    assert st == 0
    check(r, e, dtype)


def test_many_rows(sf):
    """More rows than one CTA's share of the sums: against the rows' own losses in 64 bits."""
    N = 70001
    z, h = make(N, 5, "f32", 9)
    e = reference(h)
    e["y"] = h["y"]
    r, st = call(sf, z, h, grad=True)
    assert st == 0
    check(r, e, "f32")


@pytest.mark.parametrize("N,V", [(17000, 131072), (1100, 2000003)])
def test_offsets_beyond_32_bits(sf, N, V):
    """More than 2^31 logits, in place: the last rows against the same rows alone."""
    z = torch.zeros((N, V), dtype=torch.bfloat16, device="cuda")
    last, h = make(8, V, "bf16", 21)
    e = reference(h)
    e["y"] = h["y"]
    z[-8:] = last
    t = {k: torch.zeros(N, dtype=v.dtype, device="cuda") for k, v in on_gpu(h).items()}
    for k, v in on_gpu(h).items():
        t[k][-8:] = v
    st = sf.new_status("cuda")
    r = sf.sf_policy_loss(z, clip=(LO, HI), kl_coef=BETA, inv_temperature=TAU, status=st, dlogits=z, **t)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and not z[:100].any()
    r.logp, r.token_loss, r.dlogits = r.logp[-8:], r.token_loss[-8:], z[-8:]
    check(r, e, "bf16")


@pytest.mark.parametrize("N,V", [(1, 40), (1, 70001), (5, 1000), (900, 300), (9000, 40)])
def test_sums_with_and_without_log_probabilities(sf, N, V):
    """The sums are taken from logp where it is asked for, else from a workspace."""
    z, h = make(N, V, "bf16", N)
    if N > 3:
        z[1] = math.nan
        h["w"][2] = 0.0
    a, sa = call(sf, z, h, grad=True)
    b, sb = call(sf, z, h, grad=True, want=("token_loss",))
    c, _ = call(sf, z, h, grad=True, want=())
    assert sa == sb == (sf.SF_ST_NONFINITE if N > 3 else 0) and b.logp is None and c.token_loss is None
    for o in (b, c):
        assert torch.equal(a.stats, o.stats) and torch.equal(a.dlogits, o.dlogits)
    size = sf.lib().sf_policy_loss_workspace_size(N, V)
    d, _ = call(sf, z, h, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a.stats, d.stats)


def test_no_rows(sf):
    z = torch.empty((0, 16), device="cuda")
    f = lambda n, t=torch.float32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
    r = sf.sf_policy_loss(z, f(0, torch.int64), f(0), f(0), stats=torch.ones(4, device="cuda"), grad=True)
    assert not r.stats.any() and r.dlogits.shape == (0, 16)


def test_refusals(sf):
    z, h = make(4, 16, "f32", 0)
    a = on_gpu(h)

    def code(**kw):
        k = dict(a)
        k.update(kw)
        with pytest.raises(sf.SFError) as err:
            sf.sf_policy_loss(z, **k)
        return err.value.code

    before = sf.launch_count()
    for kw in (dict(clip=(-0.1, 0.2)), dict(clip=(1.1, 0.2)), dict(clip=(0.2, math.nan)), dict(kl_coef=-1.0),
               dict(kl_coef=math.inf), dict(inv_temperature=0.0), dict(inv_temperature=math.inf)):
        assert code(**kw) == sf.SF_EINVAL
    assert code(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")) == sf.SF_EWORKSPACE
    flat = torch.empty(200, device="cuda")
    part = torch.as_strided(flat, (4, 16), (16, 1), 8)
    whole = torch.as_strided(flat, (4, 16), (16, 1), 0)
    with pytest.raises(sf.SFError) as err:
        sf.sf_policy_loss(whole, dlogits=part, **a)
    assert err.value.code == sf.SF_EINVAL
    for bad in (z.double(), z.cpu(), z[0], z.t()):
        with pytest.raises(TypeError):
            sf.sf_policy_loss(bad, **a)
    with pytest.raises(TypeError):
        sf.sf_policy_loss(z, **dict(a, target=a["target"].int()))
    with pytest.raises(ValueError):
        sf.sf_policy_loss(z, **dict(a, weight=a["weight"][:3]))
    with pytest.raises(ValueError):
        sf.sf_policy_loss(z, dlogits=torch.empty(4, 15, device="cuda"), **a)
    assert sf.launch_count() == before


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,V,ld,offset,ldd", [(320, 40001, 40003, 5, 40001), (320, 40008, 40008, 0, 40009),
                                               (320, 40008, 40008, 0, 40008), (640, 20001, 20001, 0, 20001)])
def test_calls_repeat(sf, dtype, N, V, ld, offset, ldd):
    # every call the same bits: no pack of a chunk that came later
    z, h = make(N, V, dtype, V + ldd, ld, offset)
    flat = torch.empty(N * ldd, dtype=TYPES[dtype], device="cuda")
    d = torch.as_strided(flat, (N, V), (ldd, 1), 0)
    e = reference(h)
    e["y"] = h["y"]
    first = None
    for _ in range(12):
        flat.fill_(7.0)
        r, st = call(sf, z, h, dlogits=d)
        assert st == 0
        if first is None:
            check(r, e, dtype)
            first = d.clone(), r.logp.clone(), r.stats.clone()
        for a, b in zip(first, (d, r.logp, r.stats)):
            assert torch.equal(a, b)


SUM_UNITS = 64  # roundings of 2^-24 in a row's sum, whatever the row's length: see test_equal_terms


def loss_of_rows(sf, z, y, lp, rows, grad, tau=1.0):
    """sf_policy_loss of the given rows of z, the others without weight; the gradient's factor."""
    N = z.shape[0]
    w = torch.zeros(N, device="cuda")
    w[rows] = 1.0
    old = torch.full((N,), lp + 0.1, device="cuda")
    st = sf.new_status("cuda")
    r = sf.sf_policy_loss(z, torch.full((N,), y, device="cuda"), old, torch.ones(N, device="cuda"), weight=w,
                          clip=(LO, HI), inv_temperature=tau, grad=grad, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return r, -math.exp(lp - float(old[0]))


@pytest.mark.parametrize("N,V", [(40, 131072), (2, 2000003), (2, 1 << 24)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("grad", [False, True])
def test_equal_terms(sf, N, V, dtype, grad):
    """Rows of two values: a run at the maximum, then terms so small beside its
    sum that each addition to a sum in 32 bits rounds the same way.  Held to
    what does not grow with the row: sums of at most 16 terms (15 roundings),
    their halves (1), a compensated sum (3), reductions over lanes and warps
    with one exponential each (2 (5 + 5)), the terms' own exponentials (4, and
    15 for an argument of 22) and the last reductions' products (2): 60 units
    of 2^-24; then 4 units of log S for the logarithm and the result."""
    z = torch.zeros((N, V), dtype=TYPES[dtype], device="cuda")
    rows = [0, N - 1]
    for first in (8192, 15872):
        for low in (13.9375, 14.625, 15.3125):  # half a unit of sums of 16, 8 and 4, a little less
            z[rows] = -low
            z[rows, :first] = 0.0
            S = first + (V - first) * math.exp(-low)
            lp = -math.log(S)
            r, f = loss_of_rows(sf, z, 5, lp, rows, grad)
            tol = 2.0 ** -24 * (SUM_UNITS + 4 * abs(lp))
            assert float((r.logp[rows].double() - lp).abs().max()) <= tol
            if not grad:
                continue
            for at, p in ((6, 1 / S), (first - 1, 1 / S), (first, math.exp(-low) / S), (V - 1, math.exp(-low) / S)):
                want = -f * p
                err = abs(want) * (4 * tol + 1e-6 + 2.1 * HALF_ULP[dtype]) + TINY[dtype]
                assert float((r.dlogits[rows, at].double() - want).abs().max()) <= err


def test_equal_terms_far_out(sf):
    """The same in a row that is computed by exact differences from its maximum: neighbours in 32 bits near -1e30."""
    N, V, first = 2, 2000003, 8192
    top = np.float32(-1.1e30)
    low = np.nextafter(top, np.float32(-np.inf))
    tau = float(np.float32(14.625 / (float(top) - float(low))))
    z = torch.full((N, V), float(low), device="cuda")
    z[:, :first] = float(top)
    lp = -math.log(first + (V - first) * math.exp((float(low) - float(top)) * tau))
    r, _ = loss_of_rows(sf, z, 5, lp, [0, 1], False, tau)
    assert float((r.logp.double() - lp).abs().max()) <= 2.0 ** -24 * (SUM_UNITS + 4 * abs(lp))


@pytest.mark.parametrize("N,V", [(40, 131072), (2, 2000003), (2, 1 << 24)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("grad", [False, True])
def test_rising_rows(sf, N, V, dtype, grad):
    """A maximum that rises from chunk to chunk, and what was summed is scaled
    again and again: at most six times while the old part still counts, by an
    exponential and a product of 5 units together."""
    z = torch.zeros((N, V), dtype=TYPES[dtype], device="cuda")
    rows = [0, N - 1]
    for rise in (1.0, 6.0, 40.0):
        z[rows] = torch.linspace(-rise, 0.0, V, dtype=torch.float64, device="cuda").to(TYPES[dtype])
        x = z[0].double()
        lp = float(x[V - 1] - x.logsumexp(0))
        r, _ = loss_of_rows(sf, z, V - 1, lp, rows, grad)
        assert float((r.logp[rows].double() - lp).abs().max()) <= 2.0 ** -24 * (SUM_UNITS + 30 + 4 * abs(lp)), rise


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,V", [(3, 1000), (320, 1000), (2, 140000)])
@pytest.mark.parametrize("below", [8, 100, 120, 125])
def test_logits_just_below_the_reference(sf, dtype, N, V, below):
    """A row whose largest logit times tau log2(e) lies a little below -2^20, the
    least reference of 16-bit rows: no power of 2 there may stand for its sum."""
    z = torch.zeros((N, V), dtype=TYPES[dtype], device="cuda")
    z[0] = -2.0
    z[0, 10:14] = -1.0
    tau = float(np.float32((2.0 ** 20 + below) * math.log(2.0)))
    lp = -math.log(4.0)
    w = torch.zeros(N, device="cuda")
    w[0] = 0.05
    y, old = torch.full((N,), 11, device="cuda"), torch.full((N,), lp + 0.1, device="cuda")
    st = sf.new_status("cuda")
    r = sf.sf_policy_loss(z, y, old, torch.ones(N, device="cuda"), weight=w, clip=(LO, HI), inv_temperature=tau,
                          grad=True, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert abs(float(r.logp[0]) - lp) <= DLP
    f = -math.exp(-0.1) * tau * 0.05
    want = np.zeros(V)
    want[10:14] = -f / 4
    want[11] += f
    err = np.abs(want) * (8 * DLP + 2.1 * HALF_ULP[dtype])
    assert np.all(np.abs(r.dlogits[0].double().cpu().numpy() - want) <= err)


@pytest.mark.parametrize("N", [3, 2000, 20000])
@pytest.mark.parametrize("sign", [1, -1])
def test_sums_beyond_the_result_type(sf, N, sign):
    """Finite rows whose sum is not: infinite, as one addition of 32 bits would be, whatever form adds up."""
    z = torch.zeros((N, 4), device="cuda")
    y = torch.zeros(N, dtype=torch.int64, device="cuda")
    old = torch.full((N,), -math.log(4.0), device="cuda")
    A = torch.full((N,), -sign * 2.5e38, device="cuda")
    st = sf.new_status("cuda")
    for want in (("logp", "token_loss"), ()):
        r = sf.sf_policy_loss(z, y, old, A, ref_logp=old, weight=torch.ones(N, device="cuda"), status=st, want=want)
        torch.cuda.synchronize()
        stats = r.stats.tolist()
        assert int(st.item()) == 0
        assert stats[0] == stats[1] == sign * math.inf
        assert 0 <= stats[2] <= 1e-6 * N and stats[3] == 0.0
