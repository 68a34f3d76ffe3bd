"""Calls on another stream than the current one, with memory that the binding
allocates: every allocation of every entry point comes from the stream that the
work goes to, and calls on two streams at once do not share memory."""
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


def entry_points(sf):
    """(name, call(**kw)) of each entry point that allocates."""
    g = torch.Generator(device="cuda").manual_seed(1)
    T, R, S, W, k = 12, 5, 4, 4, 2
    d = torch.randint(1, 1000, (T, R, S), generator=g, device="cuda")
    host = d.cpu().pin_memory()
    win = sf.sf_window_aggregate(d, W)
    m = sf.sf_window_median(d, W)
    ev = sf.sf_direct_gain(d, W, m)
    group = torch.zeros(R, dtype=torch.int32, device="cuda")
    gathered = torch.cat([d[t:t + W].transpose(0, 1).reshape(-1) for t in range(0, T, W)])
    z = torch.randn((2000, 64), generator=g, device="cuda")
    target = torch.zeros(2000, dtype=torch.int64, device="cuda")
    f = torch.zeros(2000, device="cuda")
    route = sf.sf_route_experts(z, 4)
    grads = [torch.randn(100003 + i, generator=g, device="cuda") for i in range(300)]
    x, w = torch.randn((300, 64), generator=g, device="cuda"), torch.randn((96, 64), generator=g, device="cuda")
    b = torch.randn((300, 65), generator=g, device="cuda").bfloat16()[:, 1:]
    wb = torch.randn((96, 65), generator=g, device="cuda").bfloat16()[:, 1:]
    dh = torch.randn((300, 96), generator=g, device="cuda")
    key = torch.tensor([1, 2], device="cuda")
    rows, token = z[:12].view(4, 3, 64), torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    return [
        ("frontier", lambda **kw: sf.sf_frontier(d, **kw)),
        ("frontier_ties", lambda **kw: sf.sf_frontier_ties(d, **kw)),
        ("window_aggregate", lambda **kw: sf.sf_window_aggregate(d, W, **kw)),
        ("topk", lambda **kw: sf.sf_topk_suspects(win.X, win.E, k, **kw)),
        ("window_median", lambda **kw: sf.sf_window_median(d, W, **kw)),
        ("direct_gain", lambda **kw: sf.sf_direct_gain(d, W, m, other_stage=1, lead_credit=True, **kw)),
        ("label_gates", lambda **kw: sf.sf_label_gates(T, R, S, W, ev, **kw)),
        ("label_windows", lambda **kw: sf.sf_label_windows(d, W, **kw)),
        ("stream_windows", lambda **kw: sf.sf_stream_windows(host, W, k, W, **kw)),
        ("stream_gathered", lambda **kw: sf.sf_stream_gathered_windows(gathered.cpu().pin_memory(), T, R, S, W, k, W, **kw)),
        ("baselines", lambda **kw: sf.sf_window_baselines(d, W, **kw)),
        ("rank_lag", lambda **kw: sf.sf_rank_lag(d, **kw)),
        ("rank_lag_windows", lambda **kw: sf.sf_rank_lag_windows(d, W, **kw)),
        ("raw_spread", lambda **kw: sf.sf_raw_spread(d, W, **kw)),
        ("group_aggregate", lambda **kw: sf.sf_group_aggregate(d, group, 1, W, **kw)),
        ("stage_group_sum", lambda **kw: sf.sf_stage_group_sum(win.X, [0, 0, 1, 1], 2, **kw)),
        ("gathered_to_steps", lambda **kw: sf.sf_gathered_to_steps(gathered, T, R, S, W, **kw)),
        ("policy_loss", lambda **kw: sf.sf_policy_loss(z, target, f, f, grad=True, **kw)),
        ("route", lambda **kw: sf.sf_route_experts(z, 4, **kw)),
        ("route_grad", lambda **kw: sf.sf_route_experts_grad(z, route.index, route.weight, **kw)),
        ("grad_norm", lambda **kw: sf.sf_grad_norm(grads, per_tensor=True, **kw)),
        ("grad_clip", lambda **kw: sf.sf_grad_clip(grads, 1e9, per_tensor=True, **kw)),
        ("gated_ffn", lambda **kw: sf.sf_gated_ffn(x, w, w, **kw)),
        ("gated_ffn_uneven", lambda **kw: sf.sf_gated_ffn(b, wb, wb, **kw)),
        ("gated_ffn_grad", lambda **kw: sf.sf_gated_ffn_grad(x, w, w, dh, want=("dx", "dw", "h"), **kw)),
        ("dropout", lambda **kw: sf.sf_dropout(x, 0.1, key, **kw)),
        ("verify", lambda **kw: sf.sf_verify_draft(rows, token, **kw)),
    ]


def test_allocations_on_the_works_stream(sf, monkeypatch):
    side, copies = torch.cuda.Stream(), torch.cuda.Stream()
    empty, made = torch.empty, []

    def watched(*a, **kw):
        made.append(torch.cuda.current_stream())
        return empty(*a, **kw)

    calls = entry_points(sf)
    torch.cuda.synchronize()
    for name, call in calls:
        made.clear()
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", watched)
            call(stream=side)
        assert made and all(s == side for s in made), name
        torch.cuda.synchronize()
        if name.startswith("stream_"):  # the staging is the copies' first
            made.clear()
            with monkeypatch.context() as m:
                m.setattr(torch, "empty", watched)
                call(stream=side, copy_stream=copies)
            assert made[0] == copies and all(s == side for s in made[1:]), name
            made.clear()
            with monkeypatch.context() as m:
                m.setattr(torch, "empty", watched)
                call(copy_stream=copies)
            here = torch.cuda.current_stream()
            assert made[0] == copies and all(s == here for s in made[1:]), name
            torch.cuda.synchronize()


def test_results_are_held_for_the_caller(sf):
    """A result of a call on another stream that the current one still reads is not given away when it is dropped."""
    side = torch.cuda.Stream()
    x = torch.ones((4096, 4096), device="cuda")
    key = torch.tensor([1, 2], device="cuda")
    torch.cuda.synchronize()
    y = sf.sf_dropout(x, 0.0, key, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    a = torch.randn((4096, 4096), device="cuda")
    for _ in range(8):
        a = a @ a * 1e-4  # keeps the current stream busy for a while
    z = y + a * 0
    del y
    other = sf.sf_dropout(x, 1.0, key, stream=side)  # at once: zeros
    torch.cuda.synchronize()
    assert bool((z == 1).all()) and not other.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_streams_at_once(sf, dtype):
    """A call on the current stream, then at once another one on a side stream: the first one's workspace
    and dropped results are not the second one's while its kernels run."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def problem(T, H, F):
        n = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(dtype)  # noqa: E731
        return n(T, H), n(F, H, k=H ** -0.5), n(F, H, k=H ** -0.5), n(T, F)

    one, two = problem(4096, 1024, 4096), problem(4096, 1024, 4096)
    call = lambda p, **kw: sf.sf_gated_ffn_grad(*p, want=("dx", "dw", "h"), **kw)  # noqa: E731
    names = ("dx", "dw_gate", "dw_up", "h")
    want = [[getattr(r, n).clone() for n in names] for r in (call(one), call(two))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        call(one)  # dropped at once: its memory is free for the current stream's next call
        a = call(one)
        b = call(two, stream=side)
        c = call(one)
        torch.cuda.synchronize()
        for r, w in ((a, want[0]), (b, want[1]), (c, want[0])):
            assert all(torch.equal(getattr(r, n), t) for n, t in zip(names, w))


def test_captured_on_a_forked_stream(sf):
    """A graph whose work goes to a second stream and back: its memory is the graph's, replay after replay, whatever
    other calls allocate in between."""
    g = torch.Generator(device="cuda").manual_seed(9)
    n = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).bfloat16()  # noqa: E731
    x, wg, wu, dh = n(700, 264), n(520, 264, k=0.06), n(520, 264, k=0.06), n(700, 520)
    key = torch.tensor([3, 4], device="cuda")
    names = ("dx", "dw_gate", "dw_up", "h")

    def work(stream=None):
        y = sf.sf_dropout(x, 0.25, key, stream=stream)
        r = sf.sf_gated_ffn_grad(x, wg, wu, dh, want=("dx", "dw", "h"), stream=stream)
        return [y] + [getattr(r, k) for k in names]

    work()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        out = work(side)
        here.wait_stream(side)
        twice = [t * 2 for t in out]
    for k in range(3):
        x.copy_(n(700, 264))
        want = [t.clone() for t in work()]
        work(side)
        torch.cuda.synchronize()
        graph.replay()
        work(side)  # beside the graph
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b * 2) for a, b in zip(twice, want))
