"""sf_verify_draft against the rule in 64 bits, sequence by sequence.

Whole numbers have to be equal, so the inputs are made with no uniform number
within 1e-4 of the ratio that it is compared with and no winner of a race within
1e-4 of the next (a probability in 32 bits is good to some 1e-6 of its value; the
difference p - q loses at most the factor p / (p - q), which `make` keeps below
50 for the two leading entries).  A log-probability is a difference of numbers of
up to |tau (z - max)| + log V and the logarithm of a sum good to 1e-6: within
4e-6 + 2^-22 of those magnitudes."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def softmax(z, tau):
    x = z.astype(np.float64) * tau
    m = x.max()
    e = np.exp(x - m)
    return e / e.sum(), x - m - math.log(e.sum())


def sequence(z, zq, y, u, e, tau):
    """(tokens, accepted, log-probabilities, closeness, ok) of one sequence by the rule; zq None: looked up;
    e None: greedy.  closeness: the least relative distance of any decision from its border."""
    out, lps, close = [], [], np.inf
    for k in range(len(y) + 1):
        if np.isnan(z[k]).any() or z[k].max() in (np.inf, -np.inf):
            return out + [-1], k, lps + [0.0], close, False
        p, lp = softmax(z[k], tau)
        if e is None:
            best = int(z[k].argmax())
            if k < len(y) and y[k] == best:
                out.append(best)
                lps.append(lp[best])
                continue
            return out + [best], k, lps + [lp[best]], close, True
        r = p
        if k < len(y):
            if 0 <= y[k] < len(p):
                if zq is None:
                    q = np.zeros_like(p)
                    q[y[k]] = 1.0
                else:
                    if np.isnan(zq[k]).any() or zq[k].max() in (np.inf, -np.inf):
                        return out + [-1], k, lps + [0.0], close, False
                    q = softmax(zq[k], tau)[0]
                with np.errstate(all="ignore"):
                    close = min(close, abs(u[k] * q[y[k]] - p[y[k]]) / max(p[y[k]], 1e-300))
                if u[k] * q[y[k]] < p[y[k]]:
                    out.append(int(y[k]))
                    lps.append(lp[y[k]])
                    continue
                r = np.maximum(p - q, 0.0)
                if zq is None:
                    r = np.where(np.arange(len(p)) == y[k], 0.0, p)
                if not (r > 0).any():
                    r = p
        with np.errstate(all="ignore"):
            v = np.where((r > 0) & (e > 0), r / e, 0.0)
        if not (v > 0).any():
            return out + [-1], k, lps + [0.0], close, False
        j = int(v.argmax())
        rest = np.delete(v, j)
        second = int(rest.argmax()) if len(rest) else 0
        if len(rest) and rest[second] > 0:
            lead = min(r[j] / p[j], np.delete(r, j)[second] / np.delete(p, j)[second])
            close = min(close, (1 - rest[second] / v[j]) * min(1.0, 50 * lead))
        return out + [j], k, lps + [lp[j]], close, True


def make(B, L, V, dtype, seed, draft=True, greedy=False, ragged=False, tau=0.9, pad=0, near=0.7):
    """Inputs as numbers; sequences whose decisions lie close to a border are drawn again."""
    rng = np.random.default_rng(seed)
    to = lambda a: torch.from_numpy(a.astype(np.float32)).to(TYPES[dtype]).float().numpy()  # noqa: E731
    s = dict(z=np.zeros((B, L + 1, V), np.float32), y=np.zeros((B, L), np.int64), u=np.zeros((B, L), np.float32),
             e=np.ones((B, V), np.float32), n=np.full(B, L, np.int32), tau=tau, dtype=dtype, greedy=greedy, pad=pad,
             zq=np.zeros((B, L, V), np.float32) if draft else None)
    for b in range(B):
        for _ in range(100):
            z = rng.standard_normal((L + 1, V)) * 2
            z[np.arange(L + 1), rng.integers(0, V, L + 1)] += 6
            s["z"][b] = to(z)
            if draft:
                s["zq"][b] = to(z[:L] + rng.standard_normal((L, V)) * near)
            s["u"][b] = rng.random(L).astype(np.float32)
            s["e"][b] = rng.exponential(size=V).astype(np.float32) + np.float32(1e-20)
            for k in range(L):
                if draft and not greedy:
                    s["y"][b, k] = rng.choice(V, p=softmax(s["zq"][b, k], tau)[0])
                else:
                    s["y"][b, k] = s["z"][b, k].argmax() if rng.random() < 0.8 else rng.integers(0, V)
            if ragged:
                s["n"][b] = rng.integers(0, L + 1)
            if want_of(s, b)[3] > 1e-4:
                break
        else:
            raise AssertionError("no sequence away from the borders")
    return s


def want_of(s, b):
    n = min(max(int(s["n"][b]), 0), s["y"].shape[1])
    zq = s["zq"]
    return sequence(s["z"][b], None if zq is None else zq[b], s["y"][b][:n], s["u"][b],
                    None if s["greedy"] else s["e"][b], s["tau"])


def padded(a, dtype, pad):
    B, n, V = a.shape
    t = torch.full((B, n, V + pad), float("nan"), dtype=dtype, device="cuda")
    t[:, :, pad // 2:pad // 2 + V] = torch.from_numpy(a).to(dtype).cuda()
    return t[:, :, pad // 2:pad // 2 + V]


def call(sf, s, **kw):
    st = sf.new_status("cuda")
    to = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    r = sf.sf_verify_draft(padded(s["z"], TYPES[s["dtype"]], s["pad"]), to(s["y"]),
                           draft=None if s["zq"] is None else padded(s["zq"], TYPES[s["dtype"]], s["pad"]),
                           lengths=to(s["n"]), uniform=None if s["greedy"] else to(s["u"]),
                           noise=None if s["greedy"] else to(s["e"]), inv_temperature=s["tau"], status=st, **kw)
    torch.cuda.synchronize()
    return r, int(st.item())


def check(sf, s, status=0):
    r, st = call(sf, s)
    assert st == status
    token, accepted, logp = (t.cpu().numpy() for t in (r.token, r.accepted, r.logp))
    B, L = s["y"].shape
    for b in range(B):
        out, k, lps, _, _ = want_of(s, b)
        assert accepted[b] == k, b
        assert token[b].tolist() == out + [-1] * (L + 1 - len(out)), b
        for i in range(L + 1):
            if i < len(out) and out[i] >= 0:
                z = s["z"][b, i].astype(np.float64)
                size = s["tau"] * abs(z[out[i]] - z.max()) + math.log(len(z))
                assert abs(logp[b, i] - lps[i]) <= 4e-6 + 2.0 ** -22 * size
            else:
                assert logp[b, i] == 0
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,L,V", [(1, 0, 1), (1, 1, 2), (3, 2, 33), (2, 4, 1000), (5, 3, 4096), (2, 2, 4097), (1, 1, 50001),
                                   (40, 3, 257), (2, 64, 100), (400, 1, 64), (3, 0, 9000), (1, 3, 131072)])
@pytest.mark.parametrize("form", ["draft", "lookup", "greedy"])
def test_rule(sf, B, L, V, dtype, form):
    check(sf, make(B, L, V, dtype, B * 7 + L + V, draft=form != "lookup", greedy=form == "greedy", ragged=L > 1 and B > 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [1, 6, 16])
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
def test_spacing_and_temperature(sf, dtype, pad, tau):
    check(sf, make(6, 3, 777, dtype, pad, ragged=True, tau=tau, pad=pad))
    check(sf, make(2, 2, 9999, dtype, pad, tau=tau, pad=pad))


def test_masked_entries(sf):
    """Entries of -inf are never drawn or accepted; a row of one entry gives it; the lowest finite numbers are no masks."""
    s = make(8, 2, 500, "f32", 3)
    s["z"][:, :, 100:] = -np.inf
    s["y"][:4] %= 100
    s["y"][4:] = 300  # drafted, but ruled out
    s["z"][7, 0, :] = -np.inf
    s["z"][7, 0, 17] = -40.0
    s["z"][6, 0, :] = np.finfo(np.float32).min
    s["u"][:] = 0.5
    for b in range(8):
        if want_of(s, b)[3] <= 1e-4 and b != 6:
            s["e"][b] = np.random.default_rng(b).exponential(size=500) + 1e-3
    r = check(sf, s)
    assert r.accepted[[4, 5, 7]].tolist() == [0] * 3 and r.token[7, 0] == 17
    assert 0 <= int(r.token[:7].max()) < 500 and bool((r.token[:6] < 100).all())


def test_equal_rows_draw_from_the_policy(sf):
    """p = q leaves nothing of p - q: a token that is rejected all the same is replaced by one from p."""
    s = make(20, 1, 5000, "bf16", 5)
    s["zq"] = s["z"][:, :1].copy()
    s["u"][:] = 1.0  # outside [0, 1): the only way to reject
    for b in range(20):
        p = softmax(s["z"][b, 0], s["tau"])[0]
        s["e"][b, (p / s["e"][b]).argmax()] *= 0.5
    r, st = call(sf, s)
    assert st == 0 and not r.accepted.any()
    for b in range(20):
        p = softmax(s["z"][b, 0], s["tau"])[0]
        assert int(r.token[b, 0]) == (p / s["e"][b]).argmax()


def test_ties_go_to_the_lowest(sf):
    z = np.zeros((3, 2, 9000), np.float32)
    for form in ("greedy", "race"):
        s = dict(z=z, y=np.full((3, 1), 8999, np.int64), u=np.full((3, 1), 0.99999, np.float32), e=np.ones((3, 9000), np.float32),
                 n=np.zeros(3, np.int32), tau=1.0, dtype="f32", greedy=form == "greedy", pad=0, zq=None)
        z[1, 0, 5000] = z[1, 0, 7000] = 1
        z[2, 0, 8998:] = 2
        r, st = call(sf, s)
        assert st == 0 and r.token[:, 0].tolist() == [0, 5000, 8998]
        z[:] = 0


def test_faulty_rows(sf):
    """NaN, +inf or nothing in a row that is needed ends that sequence; rows that are not needed do not matter."""
    s = make(9, 2, 600, "f32", 8)
    s["u"][:] = 0.0  # all drafted tokens are accepted
    s["n"][:] = [2, 2, 2, 1, 0, 2, 2, 2, 2]
    s["z"][0, 0, 3] = np.nan
    s["z"][1, 1, 599] = np.inf
    s["z"][2, 2, :] = -np.inf
    s["z"][3, 2, 0] = np.nan   # behind the length
    s["z"][4, 1:, 0] = np.nan
    s["zq"][4, :, 0] = np.nan
    s["zq"][5, 1, 7] = np.nan
    s["zq"][6, 0, :] = -np.inf
    s["e"][7, :] = 0.0         # nothing can be drawn
    s["e"][8, :] = np.nan
    for b in (3, 4):
        w = want_of(s, b)
        assert w[4] and w[3] > 1e-4
    r = check(sf, s, status=sf.SF_ST_NONFINITE)
    assert r.accepted.tolist() == [0, 1, 2, 1, 0, 1, 0, 2, 2]
    s["greedy"] = True
    r, st = call(sf, s)
    assert st == sf.SF_ST_NONFINITE and int(r.token[0, 0]) == -1


def test_bad_tokens_and_lengths(sf):
    s = make(5, 3, 300, "bf16", 9)
    s["y"][0, 0], s["y"][1, 1], s["y"][2, 0] = 300, -1, 1 << 40
    s["u"][1, 0] = 0.0
    s["n"][3], s["n"][4] = -7, 9
    for b in (0, 1, 2):
        k = 1 if b == 1 else 0
        p = softmax(s["z"][b, k], s["tau"])[0]
        s["e"][b, (p / s["e"][b]).argmax()] *= 0.5
    p = softmax(s["z"][3, 0], s["tau"])[0]
    s["e"][3, (p / s["e"][3]).argmax()] *= 0.5
    r = check(sf, s, status=sf.SF_ST_INDEX)
    assert r.accepted[:4].tolist() == [0, 1, 0, 0]


def test_distribution(sf):
    """What is kept is distributed as the policy's own samples: the first and second token's counts over many
    sequences lie within five standard deviations."""
    B, V, tau = 60000, 6, 1.0
    rng = np.random.default_rng(12)
    z, zq = rng.standard_normal((1, 2, V)), rng.standard_normal((1, 1, V))
    q = softmax(zq[0, 0], tau)[0]
    for draft in (True, False):
        s = dict(z=np.repeat(z, B, 0).astype(np.float32), zq=np.repeat(zq, B, 0).astype(np.float32) if draft else None,
                 y=rng.choice(V, size=(B, 1), p=q) if draft else np.full((B, 1), 2), u=rng.random((B, 1)).astype(np.float32),
                 e=rng.exponential(size=(B, V)).astype(np.float32) + np.float32(1e-20), n=np.ones(B, np.int32), tau=tau,
                 dtype="f32", greedy=False, pad=0)
        r, st = call(sf, s)
        assert st == 0
        token = r.token.cpu().numpy()
        for col, row in ((0, z[0, 0]), (1, z[0, 1])):
            got = token[token[:, col] >= 0, col]
            p = softmax(row, tau)[0]
            n = len(got)
            assert n > 1000
            assert (np.abs(np.bincount(got, minlength=V) - n * p) < 5 * np.sqrt(n * p * (1 - p))).all()


def test_log_probabilities_are_the_policy_losss(sf):
    s = make(4, 3, 5000, "bf16", 13)
    r, _ = call(sf, s)
    rows = padded(s["z"], TYPES["bf16"], 0).view(16, 5000)
    used = r.token.view(-1) >= 0
    zero = torch.zeros(16, device="cuda")
    o = sf.sf_policy_loss(rows, r.token.view(-1).clamp(min=0), zero, zero, inv_temperature=s["tau"])
    assert bool(((o.logp - r.logp.view(-1)).abs()[used] < 2e-5).all())


def test_graph_streams_and_repeats(sf):
    s = make(12, 4, 40000, "bf16", 14, ragged=True)
    other = make(12, 4, 40000, "bf16", 15, ragged=True)
    to = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    t = dict(z=padded(s["z"], TYPES["bf16"], 0), zq=padded(s["zq"], TYPES["bf16"], 0), y=to(s["y"]), u=to(s["u"]),
             e=to(s["e"]), n=to(s["n"]))
    out = dict(out_token=torch.empty((12, 5), dtype=torch.int64, device="cuda"),
               accepted=torch.empty(12, dtype=torch.int32, device="cuda"), logp=torch.empty((12, 5), device="cuda"))
    f = lambda **kw: sf.sf_verify_draft(t["z"], t["y"], draft=t["zq"], lengths=t["n"], uniform=t["u"], noise=t["e"],  # noqa: E731
                                        inv_temperature=0.9, **kw)
    first = f()
    for _ in range(5):
        r = f()
        assert all(torch.equal(getattr(r, n), getattr(first, n)) for n in ("token", "accepted", "logp"))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    r = f(stream=st)
    torch.cuda.synchronize()
    assert torch.equal(r.token, first.token) and torch.equal(r.logp, first.logp)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(**out)
    for n in t:
        t[n].copy_(padded(other[n], TYPES["bf16"], 0) if n in ("z", "zq") else to(other[n]))
    g.replay()
    r, _ = call(sf, other)
    assert torch.equal(out["out_token"], r.token) and torch.equal(out["accepted"], r.accepted)
    assert torch.equal(out["logp"], r.logp)


def test_many_sequences(sf):
    """More rows than a grid's second axis takes."""
    B, V = 70000, 8
    rng = np.random.default_rng(16)
    z = torch.from_numpy(rng.standard_normal((B, 1, V)).astype(np.float32)).cuda()
    y = torch.empty((B, 0), dtype=torch.int64, device="cuda")
    r = sf.sf_verify_draft(z, y)
    assert torch.equal(r.token[:, 0], z[:, 0].argmax(1)) and not r.accepted.any()


def test_long_rows(sf):
    """Rows whose offsets pass 32 bits."""
    B, V = 2, 1 << 24
    z = torch.zeros((B * 65, V), dtype=torch.bfloat16, device="cuda").view(B, 65, V)
    y = torch.zeros((B, 64), dtype=torch.int64, device="cuda")
    z[1, 64, V - 1] = 20
    z[0, 64, 12345] = 20
    r = sf.sf_verify_draft(z, y)
    assert r.accepted.tolist() == [64, 64] and r.token[:, 64].tolist() == [12345, V - 1]
    assert abs(float(r.logp[0, 0]) + math.log(V)) < 1e-4


def test_empty_and_refusals(sf):
    z = torch.zeros((2, 3, 64), device="cuda")
    y = torch.zeros((2, 2), dtype=torch.int64, device="cuda")
    u, e = torch.zeros((2, 2), device="cuda"), torch.ones((2, 64), device="cuda")
    before = sf.launch_count()
    assert sf.sf_verify_draft(z[:0], y[:0]).token.shape == (0, 3)
    for kw in (dict(uniform=u), dict(noise=e), dict(uniform=u[:1], noise=e), dict(draft=z), dict(draft=z[:, :2].half()),
               dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            sf.sf_verify_draft(z, y, **kw)
    with pytest.raises(ValueError):
        sf.sf_verify_draft(z[:, :2], y)
    with pytest.raises(TypeError):
        sf.sf_verify_draft(torch.zeros((2, 64, 3), device="cuda").transpose(1, 2), y)
    with pytest.raises(TypeError):
        sf.sf_verify_draft(z, y.int())
    for tau in (0.0, -1.0, float("nan"), 2e6):
        with pytest.raises(sf.SFError) as err:
            sf.sf_verify_draft(z, y, inv_temperature=tau)
        assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError) as err:
        sf.sf_verify_draft(torch.zeros((1, 66, 8), device="cuda"), torch.zeros((1, 65), dtype=torch.int64, device="cuda"))
    assert err.value.code == sf.SF_EINVAL
    assert sf.launch_count() == before
