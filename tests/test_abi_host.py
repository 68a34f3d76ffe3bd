"""The C ABI library without a GPU: it loads, exports every declared entry
point, and rejects bad arguments on the host before touching CUDA."""
import ctypes
import os
import re

import pytest

from paper_2606_06751_gb300 import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def sf():
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


def declared_symbols():
    names = set()
    inc = os.path.join(ROOT, "include")
    for f in os.listdir(inc):
        if f.endswith(".h"):
            txt = open(os.path.join(inc, f)).read()
            txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
            names |= set(re.findall(r"\b(sf_[a-z0-9_]+)\s*\(", txt))
    return names


def test_exports_every_declared_symbol(sf):
    syms = declared_symbols()
    assert {"sf_frontier", "sf_window_aggregate", "sf_topk_suspects", "sf_label_windows"} <= syms
    lib = ctypes.CDLL(sf.LIB_PATH)
    missing = [s for s in sorted(syms) if not hasattr(lib, s)]
    assert not missing, missing


def test_status_strings_and_helpers(sf):
    L = sf.lib()
    assert L.sf_status_str(0) == b"ok"
    assert L.sf_status_str(-5).startswith(b"workspace")
    assert sf.num_windows(0, 100, 10) == 10
    assert sf.num_windows(5, 37, 7) == 6
    assert sf.num_windows(0, 0, 7) == 0
    c = sf.default_config()
    assert (c.gamma_A.num, c.gamma_A.den) == (2, 5) and (c.tau_C.num, c.tau_C.den) == (4, 5)
    assert L.sf_label_windows_workspace_size(1000, 8, 6, 100) > 10 * 8 * 6 * 8
    assert L.sf_label_windows_workspace_size(0, 8, 6, 100) == 0


FAKE = 1 << 20  # a well-aligned address that is never dereferenced: every call below fails validation


def test_host_validation(sf):
    L = sf.lib()
    # tie-set sizes: null d / a / ties, bad shape, misaligned d
    assert L.sf_frontier_ties(None, 10, 4, 4, FAKE, FAKE, None, None) == sf.SF_EINVAL
    assert L.sf_frontier_ties(FAKE, 10, 4, 4, None, FAKE, None, None) == sf.SF_EINVAL
    assert L.sf_frontier_ties(FAKE, 10, 4, 4, FAKE, None, None, None) == sf.SF_EINVAL
    assert L.sf_frontier_ties(FAKE, 0, 4, 4, FAKE, FAKE, None, None) == sf.SF_EINVAL
    assert L.sf_frontier_ties(FAKE + 8, 10, 4, 4, FAKE, FAKE, None, None) == sf.SF_EINVAL_ALIGN
    # null input, bad shapes, no outputs
    assert L.sf_frontier(None, 10, 4, 4, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_frontier(FAKE, 0, 4, 4, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_frontier(FAKE, 10, 65537, 4, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_frontier(FAKE, 10, 4, 33, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_frontier(FAKE, 10, 4, 4, None, None, None, None, None) == sf.SF_EINVAL
    # alignment
    assert L.sf_frontier(FAKE + 8, 10, 4, 4, FAKE, None, None, None, None) == sf.SF_EINVAL_ALIGN
    assert L.sf_frontier(FAKE, 10, 4, 4, FAKE + 4, None, None, None, None) == sf.SF_EINVAL_ALIGN
    # window aggregate: W out of range, accumulate flag, missing X
    agg = L.sf_window_aggregate
    assert agg(FAKE, 10, 4, 4, 0, 0, FAKE, FAKE, None, None, None, 0, None, None) == sf.SF_EINVAL
    assert agg(FAKE, 10, 4, 4, 0, 65537, FAKE, FAKE, None, None, None, 0, None, None) == sf.SF_EINVAL
    assert agg(FAKE, 10, 4, 4, 0, 5, FAKE, FAKE, None, None, None, 2, None, None) == sf.SF_EINVAL
    assert agg(FAKE, 10, 4, 4, -1, 5, FAKE, FAKE, None, None, None, 0, None, None) == sf.SF_EINVAL
    assert agg(FAKE, 10, 4, 4, 0, 5, None, FAKE, None, None, None, 0, None, None) == sf.SF_EINVAL
    # top-k: k range, pairs without E
    assert L.sf_topk_suspects(FAKE, FAKE, 3, 4, 4, 0, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_topk_suspects(FAKE, FAKE, 3, 4, 4, 33, FAKE, None, None, None, None) == sf.SF_EINVAL
    assert L.sf_topk_suspects(FAKE, None, 3, 4, 4, 2, None, None, FAKE, None, None) == sf.SF_EINVAL
    # labeler: bad config, workspace too small or misaligned
    cfg = sf.default_config()
    bad = sf.default_config()
    bad.tau_C.den = 0
    lw = L.sf_label_windows
    assert lw(FAKE, 10, 4, 4, 5, None, None, None, -1, ctypes.byref(bad), FAKE, 1 << 20, FAKE, FAKE,
              FAKE, None, None, None, None, None, None, None) == sf.SF_EINVAL
    assert lw(FAKE, 10, 4, 4, 5, None, None, None, 4, ctypes.byref(cfg), FAKE, 1 << 20, FAKE, FAKE,
              FAKE, None, None, None, None, None, None, None) == sf.SF_EINVAL
    assert lw(FAKE, 10, 4, 4, 5, None, None, None, -1, ctypes.byref(cfg), FAKE, 16, FAKE, FAKE,
              FAKE, None, None, None, None, None, None, None) == sf.SF_EWORKSPACE
    assert lw(FAKE, 10, 4, 4, 5, None, None, None, -1, ctypes.byref(cfg), FAKE + 16, 1 << 20, FAKE,
              FAKE, FAKE, None, None, None, None, None, None, None) == sf.SF_EINVAL_ALIGN
    # evidence pass: bad eta ratio and residual stage index
    dg = L.sf_direct_gain
    assert dg(FAKE, 10, 4, 4, 5, FAKE, None, -1, sf.Ratio(1, 0), FAKE, FAKE, FAKE, None, None, FAKE, None,
              None, None) == sf.SF_EINVAL
    assert dg(FAKE, 10, 4, 4, 5, FAKE, None, -2, sf.Ratio(1, 20), FAKE, FAKE, FAKE, None, None, FAKE, None,
              None, None) == sf.SF_EINVAL
    assert dg(FAKE, 10, 4, 4, 5, FAKE, None, -1, sf.Ratio(1, 20), FAKE, FAKE, FAKE, FAKE + 4, None, FAKE,
              None, None, None) == sf.SF_EINVAL_ALIGN
    assert L.sf_window_median(FAKE, 10, 4, 4, 0, FAKE, None, None) == sf.SF_EINVAL
    # cross-rank order statistics: no outputs, bad window, misaligned output
    assert L.sf_rank_lag(FAKE, 10, 4, 4, None, None, None, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_rank_lag(FAKE, 10, 4, 4, FAKE + 4, None, None, FAKE, 1 << 20, None, None) == sf.SF_EINVAL_ALIGN
    assert L.sf_rank_lag(FAKE, 10, 4, 4, FAKE, None, None, FAKE + 16, 1 << 20, None, None) == sf.SF_EINVAL_ALIGN
    assert L.sf_rank_lag(FAKE, 10, 4, 4, FAKE, None, None, FAKE, 64, None, None) == sf.SF_EWORKSPACE
    assert L.sf_rank_lag(FAKE, 10, 4, 4, FAKE, None, None, None, 1 << 20, None, None) == sf.SF_EWORKSPACE
    assert L.sf_raw_spread(FAKE, 10, 4, 4, 0, 0, FAKE, 0, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_raw_spread(FAKE, 10, 4, 4, 0, 5, None, 0, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_raw_spread(FAKE, 10, 4, 4, 0, 5, FAKE, 3, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_raw_spread(FAKE, 10, 4, 4, 0, 5, FAKE + 4, 0, FAKE, 1 << 20, None, None) == sf.SF_EINVAL_ALIGN
    assert L.sf_rank_lag_windows(FAKE, 10, 4, 4, 0, 5, None, None, 0, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_rank_lag_windows(FAKE, 10, 4, 4, 0, 0, FAKE, None, 0, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_rank_lag_windows(FAKE, 10, 4, 4, 0, 5, FAKE, None, 0, FAKE, 8, None, None) == sf.SF_EWORKSPACE
    assert L.sf_rank_workspace_size(8192, 8192, 8) >= 8 * 8192 * 4
    assert L.sf_rank_workspace_size(0, 8, 8) == 0
    # role groups: group count, G*S limit, stage-group ids (host array)
    ga = L.sf_group_aggregate
    assert ga(FAKE, 10, 4, 4, FAKE, 0, 0, 5, FAKE, FAKE, 0, None, None) == sf.SF_EINVAL
    assert ga(FAKE, 10, 4, 8, FAKE, 1000, 0, 5, FAKE, FAKE, 0, None, None) == sf.SF_EINVAL
    assert ga(FAKE, 10, 4, 4, None, 2, 0, 5, FAKE, FAKE, 0, None, None) == sf.SF_EINVAL
    assert ga(FAKE, 10, 4, 4, FAKE + 2, 2, 0, 5, FAKE, FAKE, 0, None, None) == sf.SF_EINVAL_ALIGN
    sg = (ctypes.c_int32 * 4)(0, 1, 0, 5)
    assert L.sf_stage_group_sum(FAKE, 3, 4, sg, 2, FAKE, None) == sf.SF_EINVAL
    sg = (ctypes.c_int32 * 4)(0, 1, 0, 1)
    assert L.sf_stage_group_sum(FAKE, 3, 4, sg, 33, FAKE, None) == sf.SF_EINVAL
    assert L.sf_stage_group_sum(FAKE + 4, 3, 4, sg, 2, FAKE, None) == sf.SF_EINVAL_ALIGN
    # rank-major ingest: block length, in-place conversion, alignment
    assert L.sf_gathered_to_steps(FAKE, 10, 4, 4, 0, FAKE + (1 << 16), None) == sf.SF_EINVAL
    assert L.sf_gathered_to_steps(FAKE, 10, 4, 4, 5, FAKE + 64, None) == sf.SF_EINVAL
    assert L.sf_gathered_to_steps(FAKE + 8, 10, 4, 4, 5, FAKE + (1 << 16), None) == sf.SF_EINVAL_ALIGN
    # nothing was launched by any of the rejected calls
    assert sf.launch_count() == 0


def test_no_cpu_fallback_in_binding():
    src = open(os.path.join(ROOT, "paper_2606_06751_gb300", "stagefrontier.py")).read()
    assert "oracle" not in src and "numpy" not in src


def test_host_validation_of_training_step_operators(sf):
    """Refusals before anything is enqueued: null pointers, alignment, shapes, configurations, workspaces."""
    L = sf.lib()
    ok = sf.PolicyConfig(0.2, 0.2, 0.1, 1.0)

    def loss(logits=FAKE, dtype=1, N=4, V=16, ld=16, target=FAKE, old=FAKE, adv=FAKE, cfg=ok, stats=FAKE, d=None, ldd=16,
             ws=FAKE, size=1 << 20, logp=None):
        return L.sf_policy_loss(logits, dtype, N, V, ld, target, old, None, adv, None,
                                None if cfg is None else ctypes.byref(cfg), None, logp, None, stats, d, ldd, ws, size,
                                None, None)

    for kw in (dict(logits=None), dict(dtype=3), dict(dtype=-1), dict(N=-1), dict(V=0), dict(V=(1 << 30) + 1, ld=1 << 31),
               dict(ld=15), dict(target=None), dict(old=None), dict(adv=None), dict(cfg=None), dict(stats=None),
               dict(d=FAKE + 32), dict(d=FAKE, ldd=15), dict(d=FAKE, ldd=17), dict(N=1 << 31),
               dict(cfg=sf.PolicyConfig(-0.1, 0.2, 0.0, 1.0)), dict(cfg=sf.PolicyConfig(0.2, -0.2, 0.0, 1.0)),
               dict(cfg=sf.PolicyConfig(0.2, 0.2, 0.0, 2e6))):
        assert loss(**kw) == sf.SF_EINVAL, kw
    for kw in (dict(logits=FAKE + 1), dict(target=FAKE + 4), dict(old=FAKE + 2), dict(stats=FAKE + 2), dict(ws=FAKE + 8),
               dict(logp=FAKE + 1)):
        assert loss(**kw) == sf.SF_EINVAL_ALIGN, kw
    assert loss(ws=None) == sf.SF_EWORKSPACE and loss(size=63) == sf.SF_EWORKSPACE
    assert L.sf_policy_loss_workspace_size(4, 16) == 64 and L.sf_policy_loss_workspace_size(0, 16) == 0
    assert L.sf_policy_loss_workspace_size(-1, 16) == 0 and L.sf_policy_loss_workspace_size(4, 0) == 0

    def route(logits=FAKE, T=4, E=64, ld=64, k=4, score=0, groups=1, top=1, best=2, renorm=1, scale=1.0, index=FAKE,
              weight=FAKE, load=None, acc=0, cfg=True):
        c = sf.RouteConfig(k, score, groups, top, best, renorm, scale)
        return L.sf_route_experts(logits, 0, T, E, ld, None, ctypes.byref(c) if cfg else None, index, weight, load, acc,
                                  None, None)

    for kw in (dict(logits=None), dict(T=-1), dict(E=0), dict(E=1025, ld=1025), dict(ld=63), dict(k=0), dict(k=33),
               dict(k=9, groups=8), dict(score=2), dict(groups=0), dict(groups=33, E=66, ld=66), dict(groups=5),
               dict(top=2), dict(top=0), dict(best=0), dict(best=3), dict(renorm=2), dict(scale=float("inf")),
               dict(index=None), dict(weight=None), dict(acc=2), dict(cfg=False)):
        assert route(**kw) == sf.SF_EINVAL, kw
    for kw in (dict(logits=FAKE + 2), dict(index=FAKE + 2), dict(weight=FAKE + 1), dict(load=FAKE + 2)):
        assert route(**kw) == sf.SF_EINVAL_ALIGN, kw
    c = sf.RouteConfig(4, 0, 1, 1, 1, 1, 1.0)
    grad = lambda z, i, w, d, ldd: L.sf_route_experts_grad(z, 0, 4, 64, 64, i, w, ctypes.byref(c), d, ldd, None, None)  # noqa: E731
    far = FAKE + (1 << 16)
    assert grad(None, FAKE, FAKE, far, 64) == sf.SF_EINVAL and grad(FAKE, None, FAKE, far, 64) == sf.SF_EINVAL
    assert grad(FAKE, FAKE, None, far, 64) == sf.SF_EINVAL and grad(FAKE, FAKE, FAKE, None, 64) == sf.SF_EINVAL
    assert grad(FAKE, FAKE, FAKE, FAKE, 64) == sf.SF_EINVAL and grad(FAKE, FAKE, FAKE, FAKE + 128, 64) == sf.SF_EINVAL
    assert grad(FAKE, FAKE, FAKE, far, 63) == sf.SF_EINVAL
    assert grad(FAKE, FAKE + 1, FAKE, far, 64) == sf.SF_EINVAL_ALIGN

    def clip(data=(FAKE, far), out=None, numel=(8, 5), dtype=(0, 1), norm=FAKE, ws=FAKE, size=1 << 20, most=1.0, eps=0.0):
        n = len(numel)
        p = (ctypes.c_void_p * n)(*data)
        o = None if out is None else (ctypes.c_void_p * n)(*out)
        s, t = (ctypes.c_int64 * n)(*numel), (ctypes.c_int32 * n)(*dtype)
        if most is None:
            return L.sf_grad_norm(p, s, t, n, norm, None, ws, size, None, None)
        return L.sf_grad_clip(p, o, s, t, n, most, eps, norm, None, None, ws, size, None, None)

    for most in (None, 1.0):
        for kw in (dict(data=(None, far)), dict(numel=(-1, 5)), dict(numel=(1 << 40, 5)), dict(dtype=(0, 3)),
                   dict(norm=None)):
            assert clip(most=most, **kw) == sf.SF_EINVAL, kw
        for kw in (dict(data=(FAKE + 2, far)), dict(data=(FAKE, far + 1)), dict(norm=FAKE + 2), dict(ws=FAKE + 8)):
            assert clip(most=most, **kw) == sf.SF_EINVAL_ALIGN, kw
        assert clip(most=most, size=64) == sf.SF_EWORKSPACE
        assert clip(most=most, ws=None, numel=(2 << 20, 5)) == sf.SF_EWORKSPACE  # smaller lists need none
    for kw in (dict(most=0.0), dict(most=float("nan")), dict(eps=-1.0), dict(eps=float("inf")),
               dict(out=(FAKE + 16, far)), dict(out=(None, far))):
        assert clip(**kw) == sf.SF_EINVAL, kw
    assert L.sf_grad_norm(None, None, None, 1, FAKE, None, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_grad_norm(None, None, None, (1 << 20) + 1, FAKE, None, FAKE, 1 << 20, None, None) == sf.SF_EINVAL
    assert L.sf_grad_workspace_size(-1) == 0 and L.sf_grad_workspace_size(10) > 0
    sizes, types = (ctypes.c_int64 * 2)(3 << 20, 16), (ctypes.c_int32 * 2)(1, 0)
    assert L.sf_grad_needs_workspace(sizes, types, 1) == 0 and L.sf_grad_needs_workspace(sizes, types, 2) == 1
    assert L.sf_grad_needs_workspace(None, None, 0) == 0
    assert sf.launch_count() == 0


def test_which_gradient_lists_need_no_workspace(sf):
    """As the header says: by tensors and by packs of 16 bytes, the last of each tensor counted whole."""
    def needs(numel, dtype):
        n = len(numel)
        return sf.lib().sf_grad_needs_workspace((ctypes.c_int64 * n)(*numel), (ctypes.c_int32 * n)(*dtype), n)

    packs = 393216
    for dtype, per in ((sf.SF_F32, 4), (sf.SF_BF16, 8), (sf.SF_F16, 8)):
        assert needs([packs * per], [dtype]) == 0 and needs([packs * per + 1], [dtype]) == 1
        assert needs([(packs - 1) * per, 1], [dtype] * 2) == 0 and needs([(packs - 1) * per + 1, 1], [dtype] * 2) == 1
    assert needs([1] * 960, [sf.SF_F32] * 960) == 0 and needs([1] * 961, [sf.SF_F32] * 961) == 1
    assert needs([0] * 961, [sf.SF_F32] * 961) == 1
    for n, dtype in ((961, sf.SF_F32), (1, 3)):  # a null workspace is refused there, bad arguments too
        p, s, t = (ctypes.c_void_p * n)(*[FAKE] * n), (ctypes.c_int64 * n)(*[1] * n), (ctypes.c_int32 * n)(*[dtype] * n)
        code = sf.lib().sf_grad_norm(p, s, t, n, FAKE, None, None, 0, None, None)
        assert code == (sf.SF_EWORKSPACE if n == 961 else sf.SF_EINVAL)
