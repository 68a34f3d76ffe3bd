"""Host refusals of the operators around a policy's layers, without a GPU."""
import pytest

from paper_2606_06751_gb300 import build as B

A = 1 << 20   # well-aligned addresses, far apart, that are never dereferenced: every call fails validation
at = lambda k: A + (k << 24)  # noqa: E731


@pytest.fixture(scope="module")
def sf():
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def test_gated_ffn(sf):
    L = sf.lib()

    def call(x=at(0), dtype=sf.SF_BF16, T=8, H=64, ldx=64, wg=at(1), wu=at(2), F=72, ldw=64, act=0, h=at(3), ldh=72,
             ws=None, n=0):
        return L.sf_gated_ffn(x, dtype, T, H, ldx, wg, wu, F, ldw, act, h, ldh, ws, n, None, None)

    for kw in (dict(dtype=3), dict(T=-1), dict(H=0), dict(ldx=63), dict(ldw=63), dict(F=0), dict(act=4), dict(act=-1),
               dict(ldh=71), dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(h=at(0)), dict(h=at(1)),
               dict(h=at(2) + 128), dict(T=1 << 31)):
        assert call(**kw) == sf.SF_EINVAL, kw
    assert call(x=at(0) + 1) == sf.SF_EINVAL_ALIGN and call(dtype=sf.SF_F32, h=at(3) + 2) == sf.SF_EINVAL_ALIGN
    assert call(T=1 << 20, H=1 << 20, ldx=1 << 20, ldw=1 << 20) == sf.SF_EUNSUPPORTED
    assert call(T=0, x=None, h=None) == sf.SF_OK


def test_gated_ffn_grad(sf):
    L = sf.lib()

    def call(x=at(0), dtype=sf.SF_BF16, T=8, H=64, wg=at(1), wu=at(2), F=72, act=0, dh=at(3), dx=at(4), dwg=at(5),
             dwu=at(6), dwt=sf.SF_BF16, lddw=64, acc=0, h=None, ws=at(8), n=1 << 23):
        return L.sf_gated_ffn_grad(x, dtype, T, H, 64, wg, wu, F, 64, act, dh, 72, dx, 64, dwg, dwu, dwt, lddw, acc, h,
                                   72, ws, n, None, None)

    for kw in (dict(dh=None), dict(dwg=None), dict(dwu=None), dict(dx=None, dwg=None, dwu=None), dict(dwt=sf.SF_F16),
               dict(lddw=63), dict(acc=2), dict(dx=at(0)), dict(dx=at(3)), dict(dwu=at(5)), dict(dwg=at(1)), dict(h=at(4)),
               dict(h=at(3))):
        assert call(**kw) == sf.SF_EINVAL, kw
    assert call(ws=None) == sf.SF_EWORKSPACE and call(n=8) == sf.SF_EWORKSPACE
    assert call(ws=at(8) + 8) == sf.SF_EINVAL_ALIGN and call(dwt=sf.SF_F32, dwg=at(5) + 2) == sf.SF_EINVAL_ALIGN


def test_ffn_workspace(sf):
    size = sf.lib().sf_gated_ffn_workspace_size
    assert size(sf.SF_BF16, 0, 64, 64, 1, 1) == 0 and size(7, 8, 64, 64, 1, 1) == 0 and size(sf.SF_BF16, 8, 0, 64, 1, 1) == 0
    assert size(sf.SF_BF16, 8, 64, 64, 1, 0) == 0 and size(sf.SF_F32, 8, 65, 64, 0, 0) == 0
    for dtype, b in ((sf.SF_BF16, 2), (sf.SF_F32, 4)):
        assert size(dtype, 100, 64, 333, 1, 1) >= 2 * 100 * 333 * b


def test_dropout(sf):
    L = sf.lib()

    def call(x=at(0), dtype=sf.SF_BF16, N=8, D=64, ldx=64, p=0.1, key=at(1), res=None, ldr=64, out=at(2), ldo=64):
        return L.sf_dropout(x, dtype, N, D, ldx, p, key, res, ldr, out, ldo, None)

    for kw in (dict(dtype=-1), dict(N=-1), dict(D=0), dict(ldx=63), dict(ldo=63), dict(res=at(3), ldr=63), dict(p=-1e-9),
               dict(p=1.5), dict(p=float("nan")), dict(x=None), dict(key=None), dict(out=None), dict(out=at(0) + 2),
               dict(out=at(0), ldo=65), dict(res=at(3), out=at(3) + 64), dict(out=at(1))):
        assert call(**kw) == sf.SF_EINVAL, kw
    for kw in (dict(x=at(0) + 1), dict(key=at(1) + 4), dict(out=at(2) + 1)):
        assert call(**kw) == sf.SF_EINVAL_ALIGN, kw
    assert call(N=0, x=None, key=None, out=None) == sf.SF_OK


def test_verify(sf):
    L = sf.lib()

    def call(z=at(0), dtype=sf.SF_BF16, B=2, Ld=3, V=64, ldt=64, q=at(1), ldq=64, y=at(2), n=None, u=at(3), e=at(4),
             tau=1.0, t=at(5), acc=at(6), lp=at(7)):
        return L.sf_verify_draft(z, dtype, B, Ld, V, ldt, q, ldq, y, n, u, e, tau, t, acc, lp, None, None)

    for kw in (dict(dtype=3), dict(B=-1), dict(Ld=65), dict(Ld=-1), dict(V=0), dict(V=(1 << 24) + 1), dict(ldt=63),
               dict(ldq=63), dict(z=None), dict(y=None), dict(t=None), dict(acc=None), dict(u=None), dict(e=None),
               dict(tau=0.0), dict(tau=float("inf")), dict(t=at(2)), dict(lp=at(3)), dict(lp=at(5)), dict(t=at(0) + 64),
               dict(B=1 << 30)):
        assert call(**kw) == sf.SF_EINVAL, kw
    for kw in (dict(z=at(0) + 1), dict(y=at(2) + 4), dict(t=at(5) + 4), dict(lp=at(7) + 2)):
        assert call(**kw) == sf.SF_EINVAL_ALIGN, kw
    assert call(B=0, z=None, y=None, t=None, acc=None) == sf.SF_OK
