"""The operators around a policy's layers together, as a policy step uses them:
drafted tokens are verified, the tokens pass a gated layer with dropout, the loss
takes the verified log-probabilities, and the gradients come back the same way.
Gradients against the same step in 64 bits (products in 32 bits: 1e-4 of a
tensor's norm, some hundred times what their roundings add up to), captured and
from several threads against the eager calls, bit for bit."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

P, TAU, KL = 0.25, 0.8, 0.05


@pytest.fixture(scope="module")
def sf():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


class Step:
    """B sequences of L drafted tokens through a layer of widths H and F and a head over V tokens."""

    def __init__(self, sf, B, L, H, F, V, dtype, seed):
        self.sf, self.sizes, self.dtype = sf, (B, L, H, F, V), dtype
        self.T = T = B * (L + 1)
        f = lambda *s, d=dtype: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.x, self.wg, self.wu, self.wd, self.head = f(T, H), f(F, H), f(F, H), f(H, F), f(V, H)
        self.rows, self.draft = f(B, L + 1, V), f(B, L, V)
        self.token = f(B, L, d=torch.int64)
        self.uniform, self.noise, self.advantage = f(B, L, d=f32), f(B, V, d=f32), f(T, d=f32)
        self.key = f(2, d=torch.int64)
        self.out = dict(token=f(B, L + 1, d=torch.int64), accepted=f(B, d=torch.int32), logp=f(B, L + 1, d=f32),
                        h=f(T, F), y=f(T, H), stats=f(4, d=f32), dlogits=f(T, V), dh=f(T, F), dx=f(T, H),
                        dw_gate=f(F, H, d=f32), dw_up=f(F, H, d=f32), norm=f(1, d=f32), coef=f(1, d=f32))
        self.status = sf.new_status("cuda")
        lib, n = sf.lib(), {torch.float32: 0, torch.bfloat16: 1}[dtype]
        bytes_ = lambda k: torch.empty(max(k, 16), dtype=torch.uint8, device="cuda")  # noqa: E731
        even = 1 if H % 8 == 0 else 0
        self.ws = [bytes_(lib.sf_gated_ffn_workspace_size(n, T, H, F, even, g)) for g in (0, 1)]
        self.ws_loss = bytes_(lib.sf_policy_loss_workspace_size(T, V))
        self.refill(seed)

    def refill(self, seed):
        B, L, H, F, V = self.sizes
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda t, s: t.copy_(torch.randn(t.shape, generator=g, device="cuda") * s)  # noqa: E731
        n(self.x, 1.0), n(self.wg, H ** -0.5), n(self.wu, H ** -0.5), n(self.wd, F ** -0.5), n(self.head, H ** -0.5)
        n(self.rows, 1.5), n(self.draft, 1.0)
        self.draft.add_(self.rows[:, :L])
        self.token.random_(0, V, generator=g)
        self.uniform.uniform_(generator=g)
        self.noise.exponential_(generator=g).clamp_(min=1e-20)
        n(self.advantage, 1.0)
        self.key[0], self.key[1] = seed, 3

    def run(self):
        sf, o = self.sf, self.out
        v = sf.sf_verify_draft(self.rows, self.token, draft=self.draft, uniform=self.uniform, noise=self.noise,
                               inv_temperature=TAU, out_token=o["token"], accepted=o["accepted"], logp=o["logp"],
                               status=self.status)
        weight = (v.token.view(-1) >= 0).float() / self.T
        target = v.token.view(-1).clamp(min=0)
        sf.sf_gated_ffn(self.x, self.wg, self.wu, h=o["h"], workspace=self.ws[0], status=self.status)
        sf.sf_dropout(o["h"] @ self.wd.t(), P, self.key, residual=self.x, out=o["y"])
        logits = o["y"] @ self.head.t()
        old = v.logp.view(-1)
        sf.sf_policy_loss(logits, target, old, self.advantage, ref_logp=old, weight=weight, kl_coef=KL,
                          inv_temperature=TAU, stats=o["stats"], dlogits=o["dlogits"], workspace=self.ws_loss,
                          status=self.status)
        dy = o["dlogits"] @ self.head
        o["dh"].copy_(sf.sf_dropout(dy, P, self.key) @ self.wd)
        sf.sf_gated_ffn_grad(self.x, self.wg, self.wu, o["dh"], dx=o["dx"], dw_gate=o["dw_gate"], dw_up=o["dw_up"],
                             workspace=self.ws[1], status=self.status)
        o["dx"].add_(dy)
        sf.sf_grad_clip([o["dx"], o["dw_gate"], o["dw_up"]], 0.01, norm=o["norm"], coef=o["coef"], status=self.status)
        return [t.clone() for t in o.values()]


def plain_gradients(s):
    """The step's unclipped gradients by elementary operations in 64 bits, with the masks of sf_dropout."""
    B, L, H, F, V = s.sizes
    mask = s.sf.sf_dropout(torch.ones((s.T, H), device="cuda"), P, s.key).double()
    token, old = s.out["token"].view(-1), s.out["logp"].view(-1).double()
    x, wg, wu = (t.double().requires_grad_() for t in (s.x, s.wg, s.wu))
    h = torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())
    y = x + mask * (h @ s.wd.double().t())
    lp = torch.log_softmax(TAU * (y @ s.head.double().t()), 1).gather(1, token.clamp(min=0)[:, None])[:, 0]
    ratio, u, A = torch.exp(lp - old), old - lp, s.advantage.double()
    loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A) + KL * (torch.exp(u) - u - 1)
    loss = (loss * (token >= 0)).sum() / s.T
    return float(loss.detach()), torch.autograd.grad(loss, (x, wg, wu))


@pytest.mark.parametrize("B,L,H,F,V", [(24, 3, 64, 160, 120), (7, 4, 65, 90, 333), (2, 2, 128, 200, 1000)])
def test_gradients_of_a_step(sf, B, L, H, F, V):
    s = Step(sf, B, L, H, F, V, torch.float32, 5)
    s.run()
    assert int(s.status.item()) == 0
    o = s.out
    loss, grads = plain_gradients(s)
    assert abs(float(o["stats"][0]) - loss) <= 1e-4 * (1 + abs(loss))
    norm = float(torch.stack([g.norm() for g in grads]).norm())
    assert abs(float(o["norm"]) - norm) <= 1e-4 * norm
    coef = min(1.0, 0.01 / (norm + 1e-6))
    for got, want in zip((o["dx"], o["dw_gate"], o["dw_up"]), grads):
        assert float((got.double() - coef * want).norm()) <= 1e-4 * coef * float(want.norm())


SHAPES = [(24, 3, 64, 160, 120), (1, 0, 256, 512, 4096), (90, 4, 264, 520, 999), (300, 1, 65, 131, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,L,H,F,V", SHAPES)
def test_captured_step(sf, B, L, H, F, V, dtype):
    s = Step(sf, B, L, H, F, V, dtype, 1)
    s.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for seed in (2, 3):
        s.refill(seed)
        want = s.run()
        for t in s.out.values():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(s.out.values(), want))


def test_two_graphs_at_once(sf):
    """Two captured steps with workspaces of their own, replayed on two streams."""
    steps = [Step(sf, *SHAPES[0], torch.bfloat16, 7), Step(sf, *SHAPES[2], torch.bfloat16, 8)]
    want = [s.run() for s in steps]
    graphs = []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.out.values(), w))


def test_several_threads(sf):
    steps = [Step(sf, *SHAPES[k % 4], (torch.float32, torch.bfloat16)[k % 2], 20 + k) for k in range(6)]
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    errors = []

    def work(s, w):
        try:
            st = torch.cuda.Stream()
            for _ in range(8):
                with torch.cuda.stream(st):
                    got = s.run()
                st.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, w)):
                    errors.append("results differ")
        except Exception as e:  # noqa: BLE001
            errors.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(steps, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not errors and not any(t.is_alive() for t in threads)
