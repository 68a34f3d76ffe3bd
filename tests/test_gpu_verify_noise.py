"""sf_verify_draft where a part of the noise cannot be drawn by (0, negative, NaN):
the race falls back to p only where no entry of max(p - q, 0) is above 0, not where
those that are above 0 cannot win."""
import numpy as np
import pytest
import torch
from test_gpu_verify import call, sf, want_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [0.0, -1.0, float("nan")])
@pytest.mark.parametrize("V,dtype,pad", [(40, "f32", 0), (500, "f32", 3), (9001, "f32", 0), (40000, "bf16", 0), (40001, "f16", 1)])
def test_residual_without_noise(sf, V, dtype, pad, bad):  # noqa: F811
    """p is uniform and q has a peak at the drafted token y: p - q is above 0 everywhere but at y."""
    B, y = 5, V // 2
    z, zq = np.zeros((B, 2, V), np.float32), np.zeros((B, 1, V), np.float32)
    zq[:, 0, y] = 5
    zq[2:4] = z[2:4, :1]                   # equal rows: nothing is left of p - q
    e = np.full((B, V), bad, np.float32)
    e[0, y] = 1                            # only an entry without residual can be drawn
    e[1, y], e[1, V - 3] = 0.001, 1        # one that has a residual can
    e[2, y], e[2, 7] = 1, 2                # the policy's own draw
    u = np.full((B, 1), 1.0, np.float32)   # rejected for certain
    s = dict(z=z, zq=zq, y=np.full((B, 1), y, np.int64), u=u, e=e, n=np.ones(B, np.int32), tau=1.0, dtype=dtype, greedy=False, pad=pad)
    r, st = call(sf, s)
    assert st == sf.SF_ST_NONFINITE and not r.accepted.any()
    assert r.token[:, 0].tolist() == [-1, V - 3, y, -1, -1] and bool((r.token[:, 1] == -1).all())
    assert r.token[:, 0].tolist() == [want_of(s, b)[0][0] for b in range(B)]
    assert bool((r.logp[[0, 3, 4], 0] == 0).all())


@pytest.mark.parametrize("V,dtype", [(40, "f32"), (9001, "bf16")])
def test_looked_up_without_noise(sf, V, dtype):  # noqa: F811
    """q is 1 at the drafted token: it is what can be drawn only where p has nothing else.  Probabilities are held in
    32 bits, where exp(-300) = 5e-131 is 0 (the least number above 0 is 2^-149); the rule in 64 bits keeps it."""
    y = V // 2
    z = np.zeros((3, 2, V), np.float32)
    z[1:, 0, y] = 300
    e = np.zeros((3, V), np.float32)
    e[:2, y] = 1
    s = dict(z=z, zq=None, y=np.full((3, 1), y, np.int64), u=np.full((3, 1), 1.0, np.float32), e=e, n=np.ones(3, np.int32), tau=1.0,
             dtype=dtype, greedy=False, pad=0)
    r, st = call(sf, s)
    assert st == sf.SF_ST_NONFINITE and not r.accepted.any()
    assert r.token[:, 0].tolist() == [-1, y, -1]
    assert want_of(s, 0)[0] == [-1] and want_of(s, 2)[0] == [-1]
