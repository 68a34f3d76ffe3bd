"""sf_route_experts and its gradient against the formulas in 64 bits.

Logits and biases lie on coarse grids, so that equal choice values are exactly
equal and others are apart; the rare token two of whose values differ by less
than 1e-6 (a sigmoid plus a bias in 32 bits has half of that) is left out of
the comparison of indices.  A weight is a quotient of exponentials good to a
few roundings of 2^-24 and sums of at most 1024 / 32 + 5 of them: 1e-5 of its
value; a gradient's terms have that relative error each."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -23, "bf16": 2.0 ** -7, "f16": 2.0 ** -10}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}
REL = 1e-5


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def make(T, E, dtype, seed, ld=None, offset=0, step=8):
    rng = np.random.default_rng(seed)
    ld = E if ld is None else ld
    flat = torch.zeros(offset + T * ld, dtype=TYPES[dtype], device="cuda")
    z = torch.as_strided(flat, (T, E), (ld, 1), offset)
    z.copy_(torch.from_numpy(np.round(2.0 * rng.standard_normal((T, E)) * step) / step))
    bias = rng.choice([0.0, 0.25, -0.125], E).astype(np.float32)
    return z, bias


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def choose(z, bias, k, score, groups, top_groups, group_top):
    """(indices, tokens whose choice rounding may change), a token at a time."""
    T, E = z.shape
    per = E // groups
    index, close = np.full((T, k), -1), np.zeros(T, bool)
    for t in range(T):
        u = (sigmoid(z[t]) if score == "sigmoid" else z[t]) + bias
        u = np.where((z[t] == -np.inf) | (bias == -np.inf), -np.inf, u)
        if top_groups < groups:
            value = np.full(groups, -np.inf)
            for g in range(groups):
                best = sorted((v for v in u[g * per:(g + 1) * per] if v > -np.inf), reverse=True)[:group_top]
                if best:
                    value[g] = sum(best)
            order = sorted(range(groups), key=lambda g: (-value[g], g))
            kept = set(order[:top_groups])
            a, b = value[order[top_groups - 1]], value[order[top_groups]]
            close[t] |= a != b and abs(a - b) < 1e-6
            u = np.array([u[e] if e // per in kept else -np.inf for e in range(E)])
        order = np.lexsort((np.arange(E), -u))
        top = u[order[:k + 1]]
        with np.errstate(invalid="ignore"):
            d = np.abs(np.diff(top))
        close[t] |= bool(np.any((d > 0) & (d < 1e-6)))
        got = [e for e in order[:k] if u[e] > -np.inf]
        index[t, :len(got)] = got
    return index, close


def weights(z, index, score, renorm, scale):
    T, k = index.shape
    on = index >= 0
    zi = np.where(on, np.take_along_axis(z, np.maximum(index, 0), 1), -np.inf)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            s = np.where(on, sigmoid(zi), 0.0)
            total = s.sum(1, keepdims=True) if renorm else 1.0
        else:
            m = (zi if renorm else z).max(1, keepdims=True)
            s = np.where(on, np.exp(zi - m), 0.0)
            total = (s if renorm else np.exp(z - m)).sum(1, keepdims=True)
        return np.where(on & (s > 0), scale * s / total, 0.0)


def gradient(z, index, dw, score, renorm, scale):
    """The weights' Jacobian, applied token by token."""
    d, mag = np.zeros_like(z), np.zeros_like(z)
    for t in range(z.shape[0]):
        i = index[t][index[t] >= 0]
        if len(i) == 0:
            continue
        g = dw[t][index[t] >= 0]
        if score == "sigmoid":
            s = sigmoid(z[t, i])
            slope = s * sigmoid(-z[t, i])
            if renorm:
                if s.sum() == 0:
                    continue
                q = s / s.sum()
                d[t, i] = scale * slope / s.sum() * (g - (g * q).sum())
                mag[t, i] = scale * slope / s.sum() * (np.abs(g) + (np.abs(g) * q).sum())
            else:
                d[t, i] = scale * slope * g
                mag[t, i] = np.abs(d[t, i])
            continue
        at = i if renorm else np.arange(z.shape[1])
        m = z[t, at].max()
        if m == -np.inf:
            continue
        p = np.zeros(z.shape[1])
        p[at] = np.exp(z[t, at] - m)
        p /= p.sum()
        inner = (p[i] * g).sum()
        full = np.zeros(z.shape[1])
        full[i] = g
        d[t] = scale * p * (full - inner)
        mag[t] = scale * p * (np.abs(full) + (p[i] * np.abs(g)).sum())
    return d, mag


def route(sf, z, bias, k, **kw):
    st = sf.new_status("cuda")
    b = None if bias is None else torch.from_numpy(bias).cuda()
    r = sf.sf_route_experts(z, k, bias=b, status=st, **kw)
    torch.cuda.synchronize()
    return r, int(st.item())


def check(sf, z, bias, k, score, groups=1, top_groups=1, group_top=2, renorm=True, scale=1.0, status=0, host=None):
    r, st = route(sf, z, bias, k, score=score, groups=groups, top_groups=top_groups, group_top=group_top,
                  renorm=renorm, scale=scale)
    assert st == status
    x = z.double().cpu().numpy() if host is None else host
    T, E = x.shape
    b = np.zeros(E) if bias is None else bias.astype(np.float64)
    index, close = choose(x, b, k, score, groups, top_groups, group_top)
    got = r.index.cpu().numpy()
    assert close.mean() <= 0.01
    assert np.array_equal(got[~close], index[~close])
    w = weights(x, got, score, renorm, scale)
    assert np.all(np.abs(r.weight.double().cpu().numpy() - w) <= REL * np.abs(w))
    assert np.array_equal(r.load.cpu().numpy(), np.bincount(got[got >= 0], minlength=E))
    return r


CASES = [  # T, E, k, groups, top_groups, group_top
    (1, 1, 1, 1, 1, 2), (1, 64, 6, 1, 1, 2), (3, 7, 7, 1, 1, 2), (9, 8, 2, 1, 1, 1), (130, 33, 5, 1, 1, 2),
    (70, 60, 4, 6, 3, 2), (65, 256, 8, 8, 4, 2), (64, 256, 8, 8, 4, 1), (41, 160, 6, 8, 3, 2), (17, 475, 9, 5, 2, 2),
    (20, 512, 12, 16, 1, 2), (33, 32, 3, 32, 5, 2), (11, 1024, 32, 32, 32, 2), (10, 1000, 32, 4, 3, 2),
    (300, 128, 8, 4, 4, 2), (12, 96, 8, 3, 2, 2), (5, 1023, 31, 31, 9, 1), (13, 24, 24, 2, 2, 2)]


@pytest.mark.parametrize("T,E,k,groups,top_groups,group_top", CASES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_routing(sf, T, E, k, groups, top_groups, group_top, score, dtype):
    z, bias = make(T, E, dtype, T + E)
    check(sf, z, bias, k, score, groups, top_groups, group_top)
    check(sf, z, None, k, score, groups, top_groups, group_top, renorm=False, scale=2.5)


@pytest.mark.parametrize("T,E,k,groups,top_groups", [(3000, 256, 8, 8, 4), (20000, 64, 6, 1, 1), (2500, 100, 4, 1, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_many_tokens(sf, T, E, k, groups, top_groups, score):
    z, bias = make(T, E, "bf16", T)
    check(sf, z, bias, k, score, groups, top_groups)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,ld,offset", [(64, 72, 0), (64, 65, 0), (65, 65, 1), (256, 260, 3), (30, 31, 5)])
def test_strides_and_offsets(sf, dtype, E, ld, offset):
    z, bias = make(37, E, dtype, E, ld, offset)
    check(sf, z, bias, 4, "sigmoid")
    r = check(sf, z, bias, 4, "softmax", renorm=False)
    dw = torch.randn(37, 4, device="cuda")
    flat = torch.full((3 + 37 * (E + 2),), 7.0, dtype=TYPES[dtype], device="cuda")
    d = torch.as_strided(flat, (37, E), (E + 2, 1), 3)
    a = sf.sf_route_experts_grad(z, r.index, dw, renorm=False)
    sf.sf_route_experts_grad(z, r.index, dw, renorm=False, dlogits=d)
    assert torch.equal(a, d)
    d.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_equal_values_go_to_the_lowest(sf):
    z = torch.zeros(5, 100, device="cuda")
    for kw in (dict(), dict(groups=10, top_groups=2), dict(score="sigmoid")):
        r, _ = route(sf, z, None, 7, **kw)
        assert r.index.cpu().tolist() == [list(range(7))] * 5
    z[:, ::2] = -0.0  # both zeros are equal
    r, _ = route(sf, z, None, 7)
    assert r.index.cpu().tolist() == [list(range(7))] * 5


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,groups,top_groups", [(40, 1, 1), (40, 4, 2), (256, 8, 4)])
def test_experts_that_are_not_available(sf, score, dtype, E, groups, top_groups):
    """Masks that leave fewer than k experts, one, or none; the type's lowest value as a mask."""
    z, bias = make(12, E, dtype, E + 1)
    z[0] = -math.inf
    z[1, 1:] = -math.inf
    z[2, 3:] = -math.inf
    z[3, : E - 2] = -math.inf
    z[4, ::2] = -math.inf
    z[5, E // 2:] = torch.finfo(TYPES[dtype]).min
    bias[7] = -np.inf
    for renorm in (True, False):
        r = check(sf, z, bias, 6, score, groups, top_groups, renorm=renorm)
        assert bool((r.index[0] == -1).all()) and not r.weight[0].any()
        dw = torch.randn(12, 6, device="cuda")
        st = sf.new_status("cuda")
        d = sf.sf_route_experts_grad(z, r.index, dw, score=score, renorm=renorm, status=st)
        e, mag = gradient(z.double().cpu().numpy(), r.index.cpu().numpy(), dw.double().cpu().numpy(), score, renorm, 1.0)
        assert int(st.item()) == 0
        assert np.all(np.abs(d.double().cpu().numpy() - e) <= 4 * REL * mag + 0.51 * ULP[dtype] * np.abs(e) + TINY[dtype])
        assert not d[0].any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_faulty_values(sf, score):
    z, bias = make(6, 50, "f32", 3)
    z[1, 4] = math.nan
    host = z.double().cpu().numpy()
    host[1, 4] = -np.inf
    check(sf, z, bias, 5, score, renorm=True, status=sf.SF_ST_NONFINITE, host=host)
    z[1, 4] = math.inf
    if score == "softmax":
        check(sf, z, bias, 5, score, renorm=False, status=sf.SF_ST_NONFINITE, host=host)
    else:
        check(sf, z, bias, 5, score, renorm=False)  # a score of 1
    z[1, 4] = 0.0
    bias[9] = np.nan
    r, st = route(sf, z, bias, 5, score=score)
    assert st == sf.SF_ST_NONFINITE and not bool((r.index == 9).any())


@pytest.mark.parametrize("big", [math.inf, 3e38])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_infinite_choice_values(sf, score, big):
    """Biases that force an expert, and groups whose values are infinite together."""
    z, bias = make(9, 64, "f32", 8)
    bias[[5, 20, 21, 40, 41]] = big
    r, st = route(sf, z, bias, 3, score=score, groups=4, top_groups=1)
    assert st == 0
    # groups 1 and 2 have two such experts each (group 0 one): the lower of equal ones is kept, in 32 bits
    # 3e38 + 3e38 is infinite, and so is the sum of group 0 only where the bias is
    first = 0 if big == math.inf else 16
    assert bool(((r.index >= first) & (r.index < first + 16)).all())
    r, st = route(sf, z, bias, 6, score=score)
    got = np.sort(r.index.cpu().numpy(), 1)
    assert st == 0 and all(set([5, 20, 21, 40, 41]) <= set(row) for row in got.tolist())


def test_offsets_beyond_32_bits(sf):
    """More than 2^31 logits: the last tokens against the same tokens alone."""
    T, E, k = (1 << 23) + 1000, 256, 8
    z = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    z[-500:] = torch.randn(500, E, device="cuda").to(torch.bfloat16)
    a = sf.sf_route_experts(z, k)
    b = sf.sf_route_experts(z[-500:], k)
    assert torch.equal(a.index[-500:], b.index) and torch.equal(a.weight[-500:], b.weight)
    assert int(a.load.sum()) == T * k and bool((a.index[:1000] == torch.arange(8, device="cuda")).all())
    dw = torch.randn(T, k, device="cuda")
    for renorm in (True, False):
        d = sf.sf_route_experts_grad(z, a.index, dw, renorm=renorm)
        assert torch.equal(d[-500:], sf.sf_route_experts_grad(z[-500:], b.index, dw[-500:], renorm=renorm))


def test_saturated_scores(sf):
    """Sigmoids that are 0 in 32 bits: a sum of 0, weights and gradients of 0."""
    z = torch.full((3, 40), -200.0, device="cuda")
    z[1, 5] = 3.0
    r, st = route(sf, z, None, 4, score="sigmoid")
    assert st == 0 and not r.weight[0].any() and r.index[0].tolist() == [0, 1, 2, 3]
    assert r.weight[1].tolist() == [1.0, 0.0, 0.0, 0.0]
    d = sf.sf_route_experts_grad(z, r.index, torch.ones(3, 4, device="cuda"), score="sigmoid")
    assert not d[0].any() and bool(torch.isfinite(d).all())
    z = -z  # all 1
    r, st = route(sf, z, None, 4, score="sigmoid")
    assert st == 0 and r.weight[0].tolist() == [0.25] * 4
    z = torch.full((2, 40), -3e38, device="cuda")
    z[:, 7] = 3e38
    r, st = route(sf, z, None, 3)
    assert st == 0 and r.index[0].tolist() == [7, 0, 1] and r.weight[0].tolist() == [1.0, 0.0, 0.0]


def test_loads_accumulate(sf):
    z, bias = make(2000, 70, "bf16", 5)
    load = torch.full((70,), 5, dtype=torch.int32, device="cuda")
    a = check(sf, z, bias, 4, "sigmoid")
    b = torch.from_numpy(bias).cuda()
    sf.sf_route_experts(z, 4, bias=b, score="sigmoid", load=load, accumulate=True)
    assert torch.equal(load, a.load + 5)
    for n in (1, 8, 9, 100):
        load.fill_(3)
        r = sf.sf_route_experts(z[:n], 4, bias=b, score="sigmoid", load=load)
        assert torch.equal(load.long(), torch.bincount(r.index.flatten().long(), minlength=70))
        sf.sf_route_experts(z[:n], 4, bias=b, score="sigmoid", load=load, accumulate=True)
        assert torch.equal(load.long(), 2 * torch.bincount(r.index.flatten().long(), minlength=70))
    r = sf.sf_route_experts(z, 4, bias=b, score="sigmoid", want=())
    assert r.load is None and torch.equal(r.index, a.index)


@pytest.mark.parametrize("T,E,k", [(1, 64, 6), (37, 33, 5), (200, 160, 6), (9, 1000, 32), (5, 7, 7), (2000, 256, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gradient(sf, T, E, k, score, renorm, dtype):
    z, bias = make(T, E, dtype, T + E)
    r, _ = route(sf, z, bias, k, score=score, renorm=renorm)
    dw = torch.randn(T, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(T))
    st = sf.new_status("cuda")
    d = sf.sf_route_experts_grad(z, r.index, dw, score=score, renorm=renorm, scale=1.5, status=st)
    e, mag = gradient(z.double().cpu().numpy(), r.index.cpu().numpy(), dw.double().cpu().numpy(), score, renorm, 1.5)
    assert int(st.item()) == 0
    assert np.all(np.abs(d.double().cpu().numpy() - e) <= 4 * REL * mag + 0.51 * ULP[dtype] * np.abs(e) + TINY[dtype])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(sf, score, renorm):
    """Along a direction that leaves the choice as it is: differences of step
    1/256 have an error of 1e-5 of the third derivative and 1e-6 * 128 of rounding."""
    T, E, k = 50, 24, 24
    z, _ = make(T, E, "f32", 11)
    g = torch.Generator(device="cuda").manual_seed(1)
    dw = torch.randn(T, k, device="cuda", generator=g).double()
    D = torch.randn(T, E, device="cuda", generator=g)
    step = 1.0 / 256

    def value(x):  # all experts are chosen: put the weights in the experts' order
        r = sf.sf_route_experts(x, k, score=score, renorm=renorm)
        return (torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, r.index.long(), r.weight.double()) * dw)

    order = torch.arange(E, dtype=torch.int32, device="cuda").repeat(T, 1)
    d = sf.sf_route_experts_grad(z, order, dw.float(), score=score, renorm=renorm)
    slope = (d.double() * D.double()).sum(1)
    diff = (value(z + step * D).sum(1) - value(z - step * D).sum(1)) / (2 * step)
    assert bool(((slope - diff).abs() <= 2e-3 * (1 + slope.abs())).all())


def test_gradient_of_faulty_inputs(sf):
    z, _ = make(6, 40, "f32", 2)
    r, _ = route(sf, z, None, 4)
    index = r.index.clone()
    dw = torch.ones(6, 4, device="cuda")
    dw[:, 0] = 2.0
    for bad in (40, -2, 1 << 30):
        index[2, 1] = bad
        ref = r.index.cpu().numpy().copy()
        ref[2, 1] = -1
        st = sf.new_status("cuda")
        d = sf.sf_route_experts_grad(z, index, dw, status=st)
        e, mag = gradient(z.double().cpu().numpy(), ref, dw.double().cpu().numpy(), "softmax", True, 1.0)
        assert int(st.item()) == sf.SF_ST_INDEX
        assert np.all(np.abs(d.double().cpu().numpy() - e) <= 5 * REL * mag + TINY["f32"])
    for v in (math.nan, math.inf):
        z[3, r.index[3, 0].item()] = v
        for renorm in (True, False):
            st = sf.new_status("cuda")
            d = sf.sf_route_experts_grad(z, r.index, dw, renorm=renorm, status=st)
            assert int(st.item()) == sf.SF_ST_NONFINITE and not d[3].any() and bool(torch.isfinite(d).all())


def test_same_bits_again_and_on_another_stream(sf):
    z, bias = make(5000, 128, "bf16", 6)
    b = torch.from_numpy(bias).cuda()
    f = lambda **kw: sf.sf_route_experts(z, 8, bias=b, score="sigmoid", groups=4, top_groups=2, **kw)  # noqa: E731
    a = f()
    dw = torch.randn(5000, 8, device="cuda")
    da = sf.sf_route_experts_grad(z, a.index, dw, renorm=False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = f()
        db = sf.sf_route_experts_grad(z, o.index, dw, renorm=False)
    p = f(stream=s)
    torch.cuda.synchronize()
    for x in (o, p):
        assert torch.equal(a.index, x.index) and torch.equal(a.weight, x.weight) and torch.equal(a.load, x.load)
    assert torch.equal(da, db)


def test_no_tokens(sf):
    z = torch.empty((0, 16), device="cuda")
    load = torch.ones(16, dtype=torch.int32, device="cuda")
    r = sf.sf_route_experts(z, 2, load=load, accumulate=True)
    assert r.index.shape == (0, 2) and bool((load == 1).all())
    sf.sf_route_experts(z, 2, load=load)
    assert not load.any()
    assert sf.sf_route_experts_grad(z, r.index, r.weight).shape == (0, 16)


def test_refusals(sf):
    z = torch.zeros((4, 64), device="cuda")
    before = sf.launch_count()
    for k, kw in ((0, {}), (33, {}), (65, {}), (4, dict(groups=3)), (4, dict(groups=64, top_groups=8)),
                  (4, dict(groups=4, top_groups=5)), (4, dict(groups=4, top_groups=0)), (4, dict(group_top=3)),
                  (9, dict(groups=8, top_groups=1)), (4, dict(scale=math.nan)), (4, dict(scale=math.inf))):
        with pytest.raises(sf.SFError) as err:
            sf.sf_route_experts(z, k, **kw)
        assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError) as err:
        sf.sf_route_experts(torch.zeros((2, 1025), device="cuda"), 4)
    assert err.value.code == sf.SF_EINVAL
    with pytest.raises(ValueError):
        sf.sf_route_experts(z, 4, score="linear")
    with pytest.raises(ValueError):
        sf.sf_route_experts(z, 4, accumulate=True)
    with pytest.raises(ValueError):
        sf.sf_route_experts(z, 4, bias=torch.zeros(63, device="cuda"))
    with pytest.raises(TypeError):
        sf.sf_route_experts(z.double(), 4)
    with pytest.raises(TypeError):
        sf.sf_route_experts(z.t(), 4)
    index = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    dw = torch.zeros((4, 2), device="cuda")
    with pytest.raises(TypeError):
        sf.sf_route_experts_grad(z, index.long(), dw)
    with pytest.raises(ValueError):
        sf.sf_route_experts_grad(z, index, dw[:3])
    with pytest.raises(ValueError):
        sf.sf_route_experts_grad(z, index[:3], dw)
    with pytest.raises(sf.SFError) as err:
        sf.sf_route_experts_grad(z, index, dw, dlogits=z)
    assert err.value.code == sf.SF_EINVAL
    assert sf.launch_count() == before
