"""A layer of experts from the operators: the router, the gated product of each
expert on its tokens (a call an expert; how many tokens it has is read on the
host), and their gradients, against the same layer in 64 bits.  Products in 32
bits: 1e-4 of a tensor's norm, some hundred times what their roundings add up to."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,H,F,E,k", [(96, 64, 80, 4, 2), (700, 72, 130, 8, 3), (5, 33, 50, 6, 1)])
def test_layer_of_experts(sf, T, H, F, E, k, score):
    gen = torch.Generator(device="cuda").manual_seed(T)
    n = lambda *s, by=1.0: torch.randn(s, generator=gen, device="cuda") * by  # noqa: E731
    x, router = n(T, H), n(E, H, by=H ** -0.5)
    wg, wu, wd = n(E, F, H, by=H ** -0.5), n(E, F, H, by=H ** -0.5), n(E, H, F, by=F ** -0.5)
    dy = n(T, H)
    bias = torch.zeros(E, device="cuda")
    bias[E - 1] = -100  # an expert without tokens
    status = sf.new_status("cuda")

    logits = x @ router.t()
    route = sf.sf_route_experts(logits, k, bias=bias, score=score, status=status)
    load = route.load.tolist()
    assert sum(load) == T * k and load[E - 1] == 0
    y, dx = torch.zeros((T, H), device="cuda"), torch.zeros((T, H), device="cuda")
    dweight = torch.zeros((T, k), device="cuda")
    dwg, dwu = torch.empty_like(wg), torch.empty_like(wu)
    for e in range(E):
        t, slot = (route.index == e).nonzero(as_tuple=True)
        assert len(t) == load[e]
        xe, weight = x[t], route.weight[t, slot][:, None]
        h = sf.sf_gated_ffn(xe, wg[e], wu[e], status=status)
        out = h @ wd[e].t()
        y.index_add_(0, t, weight * out)
        dweight[t, slot] = (out * dy[t]).sum(1)
        g = sf.sf_gated_ffn_grad(xe, wg[e], wu[e], weight * (dy[t] @ wd[e]), dw_gate=dwg[e], dw_up=dwu[e], status=status)
        dx.index_add_(0, t, g.dx)
    dlogits = sf.sf_route_experts_grad(logits, route.index, dweight, score=score, status=status)
    dx += dlogits @ router
    assert int(status.item()) == 0

    leaves = x64, r64, g64, u64 = [v.double().requires_grad_() for v in (x, router, wg, wu)]
    z = x64 @ r64.t()
    p = torch.softmax(z, 1) if score == "softmax" else torch.sigmoid(z)
    index = route.index.long()
    w = p.gather(1, index)
    w = w / w.sum(1, keepdim=True)
    want = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    for e in range(E):
        h = torch.nn.functional.silu(x64 @ g64[e].t()) * (x64 @ u64[e].t())
        want = want + (h @ wd[e].double().t()) * (w * (index == e)).sum(1, keepdim=True)
    grads = torch.autograd.grad((want * dy.double()).sum(), leaves)
    # k = 1: a weight is p / p = 1 and its gradient 0, of which the reference's roundings leave 2^-53 of its terms
    near = lambda a, b: float((a.double() - b).norm()) <= 1e-4 * float(b.norm()) + 1e-12  # noqa: E731
    assert near(y, want.detach()) and near(dx, grads[0]) and near(dlogits.t() @ x, grads[1])
    assert near(dwg, grads[2]) and near(dwu, grads[3])
    assert not dwg[E - 1].any() and not dwu[E - 1].any()
