"""sf_grad_norm and sf_grad_clip against the formulas in 64 bits.

Tolerances: a sum of squares is exact to 32 roundings of 2^-24 on its way into
64 bits, so its root is within 16 of them and the rounding of the result:
2e-6 of the norm.  The clipped value has the coefficient's error (that of the
norm and three roundings) and one rounding to its type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10}
TINY = {torch.float32: 2.0 ** -148, torch.bfloat16: 2.0 ** -132, torch.float16: 2.0 ** -24}
REL = 2e-6


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def tensors(sizes, types, seed, packed=True, scale=1.0):
    """Tensors as views of one buffer a type: packed, they start at any element."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    at, out = {}, []
    for n, t in zip(sizes, types):
        at[t] = at.get(t, 1) + n if packed else -(-(at.get(t, 0) + n) // 64) * 64
    flat = {t: torch.randn(n, generator=g, device="cuda").mul_(scale).to(TYPES[t]) for t, n in at.items()}
    at = {t: 1 if packed else 0 for t in flat}
    for n, t in zip(sizes, types):
        out.append(flat[t][at[t]:at[t] + n])
        at[t] += n if packed else -(-n // 64) * 64
        at[t] = at[t] if packed else -(-at[t] // 64) * 64
    return out, flat


def norms(grads):
    each = np.array([math.sqrt(float(g.double().square().sum())) if g.numel() else 0.0 for g in grads])
    return math.sqrt(float((each ** 2).sum())), each


def check(sf, grads, max_norm=None, out=None, eps=1e-6):
    total, each = norms(grads)
    before = [g.double() for g in grads]
    st = sf.new_status("cuda")
    if max_norm is None:
        r = sf.sf_grad_norm(grads, per_tensor=True, status=st)
    else:
        r = sf.sf_grad_clip(grads, max_norm, out=out, eps=eps, per_tensor=True, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert abs(float(r.norm) - total) <= REL * total
    assert np.all(np.abs(r.tensor_norm.double().cpu().numpy() - each) <= REL * each)
    if max_norm is None:
        return r
    coef = min(1.0, max_norm / (total + eps)) if total + eps > 0 else 1.0
    assert abs(float(r.coef) - coef) <= 2 * REL * coef
    for b, g in zip(before, grads if out is None else out):
        err = (b * coef).abs() * (2 * REL + 0.51 * ULP[g.dtype]) + TINY[g.dtype]
        assert bool(((g.double() - b * coef).abs() <= err).all())
    return r


LISTS = [([1], ["f32"]), ([0], ["bf16"]), ([5], ["bf16"]), ([17, 0, 3], ["f16", "f32", "bf16"]),
         ([4095, 4096, 4097, 1, 2, 7], ["bf16"] * 6), ([1000003], ["f32"]), ([20000001, 333], ["bf16", "f32"]),
         ([4096 * 8, 100001, 9, 64, 100], ["f16", "bf16", "f32", "f32", "f16"])]


@pytest.mark.parametrize("sizes,types", LISTS)
@pytest.mark.parametrize("packed", [False, True])
def test_norms(sf, sizes, types, packed):
    check(sf, tensors(sizes, types, 1, packed)[0])


@pytest.mark.parametrize("sizes,types", LISTS)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clip_in_place(sf, sizes, types, packed, max_norm):
    grads, flat = tensors(sizes, types, 2, packed)
    rest = {t: f.clone() for t, f in flat.items()}
    check(sf, grads, max_norm)
    if packed:  # the element before the first tensor
        for t in flat:
            assert torch.equal(flat[t][:1], rest[t][:1])


@pytest.mark.parametrize("sizes,types", LISTS)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_clip_into_other_tensors(sf, sizes, types, shift):
    """Results that start at another element than the gradients do."""
    grads, flat = tensors(sizes, types, 3)
    kept = {t: f.clone() for t, f in flat.items()}
    full = [torch.full((n + 8,), 7.0, dtype=TYPES[t], device="cuda") for n, t in zip(sizes, types)]
    out = [f[1 + shift:1 + shift + n] for f, n in zip(full, sizes)]
    check(sf, grads, 0.5, out)
    for t in flat:
        assert torch.equal(flat[t], kept[t])
    for f, n in zip(full, sizes):
        assert bool((f[:1 + shift] == 7).all()) and bool((f[1 + shift + n:] == 7).all())
    full = [f.clone() for f in full]
    check(sf, grads, 1e9, [f[1 + shift:1 + shift + n] for f, n in zip(full, sizes)])  # unclipped: a copy


@pytest.mark.parametrize("n", [63, 64, 65, 1024, 1025, 2500])
def test_many_tensors(sf, n):
    rng = np.random.default_rng(n)
    sizes = [int(v) for v in rng.integers(0, 3000, n)]
    types = [["f32", "bf16", "f16"][int(v)] for v in rng.integers(0, 3, n)]
    grads, _ = tensors(sizes, types, n)
    check(sf, grads)
    check(sf, grads, 2.0)


@pytest.mark.parametrize("n,each", [(24, 50000), (960, 1000), (961, 1000), (3, 1048576), (3, 1048577), (200, 7)])
@pytest.mark.parametrize("packed", [False, True])
def test_around_the_size_of_one_launch(sf, n, each, packed):
    """Up to 6 MB in up to 960 tensors go by one cluster, without a workspace; the same bits with one."""
    sizes = [each + (i % 3 - 1) * (i % 5) for i in range(n)] if n > 3 else [each] * n
    grads, _ = tensors(sizes, [["bf16", "f32", "f16"][i % 3] for i in range(n)] if n > 3 else ["bf16"] * n, n, packed)
    check(sf, grads)
    a = sf.sf_grad_norm(grads, per_tensor=True)
    ws = torch.empty(sf.lib().sf_grad_workspace_size(n), dtype=torch.uint8, device="cuda")
    b = sf.sf_grad_norm(grads, per_tensor=True, workspace=ws)
    assert torch.equal(a.norm, b.norm) and torch.equal(a.tensor_norm, b.tensor_norm)
    check(sf, grads, 0.5, [torch.empty_like(g) for g in grads])
    check(sf, grads, 0.5)


def test_equal_values(sf):
    """Sums of equal squares, which round the same way over and over in 32 bits."""
    for t, v in (("f32", 0.1), ("bf16", 1.1015625), ("f16", 0.3)):
        check(sf, [torch.full((30000000,), v, dtype=TYPES[t], device="cuda")])


@pytest.mark.parametrize("t,big,small", [("f32", 3e36, 1e-30), ("bf16", 3e36, 1e-30), ("f16", 6e4, 6e-8)])
def test_range(sf, t, big, small):
    """Squares beyond and below 32 bits."""
    for v in (big, small):
        g = torch.full((5000,), v, dtype=TYPES[t], device="cuda")
        g[::2] = 0.0
        other = torch.randn(4096 * 3 + 1, device="cuda").to(TYPES[t]).mul_(v if v == small else 1e-3)
        check(sf, [g, other])
        check(sf, [g, other], 0.5)
    zero = torch.zeros(100000, dtype=TYPES[t], device="cuda")
    check(sf, [zero, zero.clone()[1:]], 1.0, eps=0.0)


@pytest.mark.parametrize("v", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [9, 70000])
def test_not_finite(sf, v, t, n):
    good = torch.ones(n, dtype=TYPES[t], device="cuda")
    bad = torch.ones(n, dtype=TYPES[t], device="cuda")
    bad[n // 2] = v
    kept = bad.clone()
    st = sf.new_status("cuda")
    r = sf.sf_grad_clip([good, bad], 0.5, per_tensor=True, status=st)
    assert int(st.item()) == sf.SF_ST_NONFINITE and math.isnan(float(r.coef))
    assert not math.isfinite(float(r.norm)) and not math.isfinite(float(r.tensor_norm[1]))
    assert abs(float(r.tensor_norm[0]) - math.sqrt(n)) <= REL * math.sqrt(n)
    assert bool((good == 1).all()) and torch.equal(bad.view(torch.uint8), kept.view(torch.uint8))
    out = [torch.empty_like(good), torch.empty_like(bad)]
    sf.sf_grad_clip([good, bad], 0.5, out=out)
    assert bool((out[0] == 1).all())
    assert torch.equal(out[1].nan_to_num(5.0), bad.nan_to_num(5.0))


def test_norm_beyond_the_result_type(sf):
    g = torch.full((1000,), 3e38, device="cuda")
    st = sf.new_status("cuda")
    r = sf.sf_grad_norm([g], status=st)
    assert int(st.item()) == sf.SF_ST_NONFINITE and math.isinf(float(r.norm))


def test_more_than_32_bits_of_elements(sf):
    n = (1 << 31) + 12345
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g[-3:] = 100.0
    r = sf.sf_grad_clip([g[:77], g[77:]], 1.0, per_tensor=True)
    total = math.sqrt(n - 3 + 3e4)
    assert abs(float(r.norm) - total) <= REL * total
    assert abs(float(r.tensor_norm[1]) - math.sqrt(n - 80 + 3e4)) <= REL * total
    want = torch.tensor([1.0, 100.0], device="cuda").mul(1.0 / total).bfloat16()
    assert bool((g[:-3] == want[0]).all()) and bool((g[-3:] == want[1]).all())


def test_no_tensors(sf):
    r = sf.sf_grad_norm([], per_tensor=True)
    assert float(r.norm) == 0.0 and r.tensor_norm.numel() == 0
    r = sf.sf_grad_clip([], 1.0)
    assert float(r.norm) == 0.0 and float(r.coef) == 1.0


def test_same_bits_again_and_on_another_stream(sf):
    grads, _ = tensors([3000001, 70001, 12], ["bf16", "f32", "f16"], 7)
    out = [torch.empty_like(g) for g in grads]
    a = sf.sf_grad_clip(grads, 1.0, out=out, per_tensor=True)
    kept = [o.clone() for o in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = sf.sf_grad_clip(grads, 1.0, out=out, per_tensor=True)
    c = sf.sf_grad_clip(grads, 1.0, out=out, per_tensor=True, stream=s)
    torch.cuda.synchronize()
    for o in (b, c):
        assert torch.equal(a.norm, o.norm) and torch.equal(a.coef, o.coef) and torch.equal(a.tensor_norm, o.tensor_norm)
    assert all(torch.equal(x, y) for x, y in zip(kept, out))


def test_in_a_graph(sf):
    """Captured once, replayed on new gradients."""
    grads, _ = tensors([100001, 4097], ["bf16", "f32"], 8)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    norm, coef = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    sf.sf_grad_clip(grads, 1.0, norm=norm, coef=coef, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sf.sf_grad_clip(grads, 1.0, norm=norm, coef=coef, workspace=ws)
    for g in grads:
        g.normal_()
    total, _ = norms(grads)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(norm) - total) <= REL * total
    after, _ = norms(grads)
    assert abs(after - 1.0) <= 1e-3


def test_refusals(sf):
    g = [torch.ones(8, device="cuda"), torch.ones(5, device="cuda")]
    before = sf.launch_count()
    for kw in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(max_norm=1.0, eps=-1.0),
               dict(max_norm=1.0, eps=math.inf)):
        with pytest.raises(sf.SFError) as err:
            sf.sf_grad_clip(g, **kw)
        assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError) as err:
        sf.sf_grad_norm(g, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert err.value.code == sf.SF_EWORKSPACE
    flat = torch.ones(20, device="cuda")
    with pytest.raises(sf.SFError) as err:
        sf.sf_grad_clip([flat[:8]], 1.0, out=[flat[4:12]])
    assert err.value.code == sf.SF_EINVAL
    for bad in (torch.ones(8), torch.ones(8, dtype=torch.float64, device="cuda"),
                torch.ones((4, 4), device="cuda").t()[:3]):
        with pytest.raises(TypeError):
            sf.sf_grad_norm([bad])
    for out in ([g[0]], [g[0], torch.ones(6, device="cuda")], [g[0], g[1].bfloat16()]):
        with pytest.raises(ValueError):
            sf.sf_grad_clip(g, 1.0, out=out)
    assert sf.launch_count() == before


def ragged(n, total, seed):
    """Sizes of n tensors (a few large ones, many small and empty ones, odd counts) and their types."""
    rng = np.random.default_rng(seed)
    share = rng.lognormal(0.0, 2.0, n)
    sizes = [int(v) for v in share / share.sum() * total]
    sizes[3::11] = [i % 3 for i in range(len(sizes[3::11]))]
    return sizes, [["bf16", "f32", "f16"][int(v)] for v in rng.integers(0, 3, n)]


@pytest.mark.parametrize("n,total", [(5, 150000001), (60, 140000001), (1100, 260000003)])
@pytest.mark.parametrize("packed", [False, True])
def test_ranges_of_whole_ctas(sf, n, total, packed):
    """Lists above 160 MB: a range is a CTA's and its warps take the blocks in
    turn.  Random values of every type, ragged, in place and into results that
    start elsewhere, with what lies around them; 1100 tensors are two lists."""
    sizes, types = ragged(n, total, n)
    grads, flat = tensors(sizes, types, n, packed)
    # the first list's bytes: each of up to 152 * 4 * 8 warps' 2048 packs of 16
    assert sum(g.numel() * g.element_size() for g in grads[:960]) > 160e6
    check(sf, grads)
    kept = {t: f.clone() for t, f in flat.items()}
    for shift in (0, 1, 3):
        full = {t: torch.full((sum(m + 8 for m, u in zip(sizes, types) if u == t),), 7.0, dtype=TYPES[t], device="cuda")
                for t in flat}
        guard = {t: torch.ones(f.numel(), dtype=torch.bool, device="cuda") for t, f in full.items()}
        at, out = {t: 0 for t in flat}, []
        for m, t in zip(sizes, types):
            a = at[t] + 1 + shift
            out.append(full[t][a:a + m])
            guard[t][a:a + m] = False
            at[t] += m + 8
        check(sf, grads, 0.5, out)
        for t in flat:
            assert torch.equal(flat[t], kept[t]) and bool((full[t][guard[t]] == 7).all())
        del full, guard, out
    check(sf, grads, 0.5)
