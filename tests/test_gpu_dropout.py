"""sf_dropout against its definition: the mask bit for bit from a generator
written here, the values with the two roundings of 32 bits and the one to the
type that the definition has, so that results are equal."""
import numpy as np
import pytest
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def philox(counter, key):
    """Philox4x32-10 on arrays: counter [4][...], key [2] numbers."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k0, k1 = key
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def keep(N, D, p, seed, offset):
    packs = (D + 7) // 8
    pack, row = np.meshgrid(np.arange(packs), np.arange(N))
    full = lambda v: np.full((N, packs), v)  # noqa: E731
    w = philox([pack, row, full(offset & 0xFFFFFFFF), full(offset >> 32)], (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack([v for u in w for v in (u & np.uint64(0xFFFF), u >> np.uint64(16))], -1).reshape(N, packs * 8)[:, :D]
    return bits >= int(np.floor(np.float32(p).astype(np.float64) * 65536 + 0.5))


def expected(x, p, seed, offset, residual=None):
    N, D = x.shape
    t = int(np.floor(np.float64(np.float32(p)) * 65536 + 0.5))
    scale = np.float32(65536 / (65536 - t)) if t < 65536 else np.float32(0)
    kept = torch.from_numpy(keep(N, D, p, seed, offset))
    y = torch.where(kept, x.cpu().float() * torch.tensor(scale), torch.zeros(()))
    if residual is not None:
        y = y + residual.cpu().float()
    return y.to(x.dtype)


def test_generator_has_the_published_vectors():
    """The generator's known answers (counter and key all zeros, all ones, and digits of pi)."""
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(v) for v in philox(counter, key)) == want


def key_of(seed, offset):
    signed = lambda v: v - (1 << 64) if v >= 1 << 63 else v  # noqa: E731
    return torch.tensor([signed(seed), signed(offset)], dtype=torch.int64, device="cuda")


def rows(N, D, dtype, gen, ld=None, offset=0):
    ld = D if ld is None else ld
    flat = torch.full((offset + N * ld + 64,), 7.0, dtype=TYPES[dtype], device="cuda")
    t = torch.as_strided(flat, (N, D), (ld, 1), offset)
    t.copy_(torch.randn((N, D), generator=gen, device="cuda"))
    return flat, t


def same(a, b):
    v = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.cpu().contiguous().view(v), b.cpu().contiguous().view(v))


SEED, OFFSET = 0xFEDCBA9876543210, (5 << 32) + 77


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D,ld,offset", [(1, 1, None, 0), (1, 7, None, 0), (3, 8, None, 0), (2, 9, None, 1),
                                           (5, 255, 256, 0), (5, 256, 264, 8), (4, 257, 257, 3), (300, 100, 104, 0),
                                           (7, 4096, None, 0), (33, 5001, None, 0), (2000, 33, 40, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_values(sf, dtype, N, D, ld, offset, residual):
    gen = torch.Generator(device="cuda").manual_seed(N * 1000 + D)
    _, x = rows(N, D, dtype, gen, ld, offset)
    r = rows(N, D, dtype, gen, ld, offset)[1] if residual else None
    flat, out = rows(N, D, dtype, gen, ld, offset)
    before = flat.clone()
    sf.sf_dropout(x, 0.3, key_of(SEED, OFFSET), residual=r, out=out)
    want = expected(x, 0.3, SEED, OFFSET, r)
    assert same(out, want)
    torch.as_strided(before, out.shape, out.stride(), out.storage_offset()).copy_(out)
    assert torch.equal(flat, before)  # nothing else was written
    assert same(sf.sf_dropout(x, 0.3, key_of(SEED, OFFSET), residual=r), want)  # rows of another spacing


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.5, 0.999999, 1.0])
def test_probabilities(sf, p):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = rows(40, 300, "f32", gen)[1]
    out = sf.sf_dropout(x, p, key_of(1, 2))
    assert same(out, expected(x, p, 1, 2))
    if p == 0.0:
        assert torch.equal(out, x)
    if p == 1.0:
        assert not out.any()


@pytest.mark.gpu
def test_share_kept(sf):
    """Of 2^22 values with p = 0.1 as many are dropped as five standard deviations allow; rows, neighbouring
    offsets and seeds have masks of their own."""
    x = torch.ones((1024, 4096), device="cuda")
    a = sf.sf_dropout(x, 0.1, key_of(9, 0))
    t = round(0.1 * 65536) / 65536
    dropped = int((a == 0).sum())
    assert abs(dropped - t * 2 ** 22) < 5 * (t * (1 - t) * 2 ** 22) ** 0.5
    for other in (sf.sf_dropout(x, 0.1, key_of(9, 1)), sf.sf_dropout(x, 0.1, key_of(10, 0)), a.roll(1, 0), a.roll(1, 1)):
        both = int(((a == 0) & (other == 0)).sum())
        assert abs(both - t * t * 2 ** 22) < 5 * (t * t * 2 ** 22) ** 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("D", [320, 321])
def test_in_place(sf, D):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, r = rows(9, D, "bf16", gen)[1], rows(9, D, "bf16", gen)[1]
    want = expected(x, 0.25, 5, 6, r)
    y = x.clone()
    assert sf.sf_dropout(y, 0.25, key_of(5, 6), residual=r, out=y) is y and same(y, want)
    y = r.clone()
    sf.sf_dropout(x, 0.25, key_of(5, 6), residual=y, out=y)
    assert same(y, want)


@pytest.mark.gpu
def test_dropped_values_do_not_matter(sf):
    kept = torch.from_numpy(keep(6, 500, 0.5, 7, 8)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = rows(6, 500, "f32", gen)[1].clone()
    y = torch.where(kept, x, torch.full_like(x, float("nan")))
    assert same(sf.sf_dropout(y, 0.5, key_of(7, 8)), sf.sf_dropout(x, 0.5, key_of(7, 8)))


@pytest.mark.gpu
def test_gradient(sf):
    """The backward call is the forward call's derivative: the map is linear, so differences are exact but for roundings."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, d, up = (rows(16, 130, "f32", gen)[1] for _ in range(3))
    key = key_of(11, 12)
    f = lambda v: sf.sf_dropout(v, 0.2, key, residual=x).double()  # noqa: E731
    numeric = ((f(x + d) - f(x - d)) * up.double()).sum() / 2
    analytic = (sf.sf_dropout(up, 0.2, key).double() * d.double()).sum()
    # values below 16, four roundings each, 2080 terms
    assert abs(float(numeric - analytic)) < 2080 * 4 * 16 * 4 * 2.0 ** -24


@pytest.mark.gpu
def test_graph_draws_anew(sf):
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = rows(20, 640, "bf16", gen)[1]
    key, out = key_of(21, 0), torch.empty_like(x)
    sf.sf_dropout(x, 0.1, key, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sf.sf_dropout(x, 0.1, key, out=out)
        key[1] += 3
    for k in range(3):
        g.replay()
        assert same(out, expected(x, 0.1, 21, 3 * k))


@pytest.mark.gpu
def test_streams_and_no_rows(sf):
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = rows(20, 640, "bf16", gen)[1]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = sf.sf_dropout(x, 0.1, key_of(1, 1), stream=s)
    torch.cuda.synchronize()
    assert same(out, expected(x, 0.1, 1, 1))
    before = sf.launch_count()
    assert sf.sf_dropout(x[:0], 0.1, key_of(1, 1)).shape == (0, 640)
    assert sf.launch_count() == before


@pytest.mark.gpu
def test_long_tensor(sf):
    """Rows whose offsets pass 32 bits."""
    N, D = 70000, 32776
    x = torch.ones((N, D), dtype=torch.bfloat16, device="cuda")
    out = sf.sf_dropout(x, 0.5, key_of(1, 1), out=x)
    for a in (0, 65530, N - 5):  # the counter's row is the tensor's: the tail against a view of the mask
        pack, row = np.meshgrid(np.arange(D // 8), np.arange(a, a + 5))
        z = np.zeros_like(pack)
        w = philox([pack, row, z + 1, z], (1, 0))
        bits = np.stack([v for u in w for v in (u & np.uint64(0xFFFF), u >> np.uint64(16))], -1).reshape(5, D)
        assert np.array_equal(out[a:a + 5].float().cpu().numpy(), np.where(bits >= 32768, 2.0, 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("start", [0, 3])
def test_longest_row(sf, start):
    """A row of 2^31 - 1 columns, from a 16-byte boundary and from within: its last columns."""
    D = (1 << 31) - 1
    flat = torch.ones(D + 16, dtype=torch.bfloat16, device="cuda")
    x = flat[start:start + D].view(1, D)
    sf.sf_dropout(x, 0.5, key_of(1, 1), out=x)
    for pack in (0, (1 << 28) - 2):
        at = np.arange(pack, pack + 2)[None]
        z = np.zeros_like(at)
        w = philox([at, z, z + 1, z], (1, 0))
        bits = np.stack([v for u in w for v in (u & np.uint64(0xFFFF), u >> np.uint64(16))], -1).reshape(-1)
        got = x[0, pack * 8:pack * 8 + 16].float().cpu().numpy()
        assert np.array_equal(got, np.where(bits >= 32768, 2.0, 0.0)[:len(got)])
    assert bool((flat[start + D:] == 1).all()) and bool((flat[:start] == 1).all())


@pytest.mark.gpu
def test_refusals(sf):
    x = torch.zeros((4, 64), device="cuda")
    key = key_of(1, 1)
    before = sf.launch_count()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(sf.SFError) as err:
            sf.sf_dropout(x, p, key)
        assert err.value.code == sf.SF_EINVAL
    flat = torch.zeros(1024, device="cuda")
    with pytest.raises(sf.SFError) as err:
        sf.sf_dropout(flat[:256].view(4, 64), 0.1, key, out=flat[8:264].view(4, 64))
    assert err.value.code == sf.SF_EINVAL
    with pytest.raises(sf.SFError):
        sf.sf_dropout(flat[:256].view(4, 64), 0.1, key, residual=flat[512:768].view(4, 64), out=flat[500:756].view(4, 64))
    for bad in (dict(residual=x[:3]), dict(out=x.bfloat16())):
        with pytest.raises(ValueError):
            sf.sf_dropout(x, 0.1, key, **bad)
    with pytest.raises(ValueError):
        sf.sf_dropout(x, 0.1, key[:1])
    with pytest.raises(TypeError):
        sf.sf_dropout(x, 0.1, key.int())
    with pytest.raises(TypeError):
        sf.sf_dropout(x.t(), 0.1, key)
    assert sf.launch_count() == before
