"""The example's training step: its gradients against the same step in plain
64-bit operations, and a run of it with its report."""
import math
import os
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_06751_gb300 import build as B
    B.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import monitored_step
    finally:
        sys.path.pop(0)
    return monitored_step


def plain_gradients(model, batches, k, kl_coef):
    """The step's gradients by elementary operations in 64 bits."""
    p = [q.detach().double().requires_grad_() for q in model.parameters()]
    embedding, router, up, head = p
    x = embedding[torch.cat([b["context"] for b in batches])]
    s = torch.sigmoid(x @ router)
    index = (s + model.bias.double()).sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = s.gather(1, index)
    w = w / w.sum(1, keepdim=True)
    full = torch.zeros_like(s).scatter(1, index, w)
    y = torch.relu(torch.einsum("td,edf->tef", x, up))
    logits = (x + torch.einsum("tef,te->tf", y, full)) @ head
    logp = torch.log_softmax(logits, 1).gather(1, torch.cat([b["target"] for b in batches])[:, None])[:, 0]
    cat = lambda n: torch.cat([b[n] for b in batches]).double()  # noqa: E731
    ratio = torch.exp(logp - cat("old_logp"))
    u = cat("ref_logp") - logp
    loss = -torch.minimum(ratio * cat("advantage"), ratio.clamp(0.8, 1.2) * cat("advantage"))
    loss = ((loss + kl_coef * (torch.exp(u) - u - 1)) * cat("weight")).sum() / len(batches)
    return loss.detach(), torch.autograd.grad(loss, p), index


def test_gradients_of_a_step(example):
    dev = torch.device("cuda", torch.cuda.current_device())
    model = example.Model(200, 32, 16, 3, 3, dev)
    status = example.sf.new_status(dev)
    gen = torch.Generator(device=dev).manual_seed(5)
    _, info = example.step(model, 4, 96, gen, 0.0, 1e9, 0.02, status)
    gen.manual_seed(5)
    batches = [example.batch_of(96, 200, gen, dev) for _ in range(4)]
    model.bias.zero_()  # the step has moved it
    loss, grads, index = plain_gradients(model, batches, 3, 0.02)
    assert int(status.item()) == 0
    assert torch.equal(info["load"].long(), torch.bincount(index.flatten(), minlength=16))
    assert abs(float(info["stats"][0]) - float(loss)) <= 1e-4 * (1 + abs(float(loss)))
    for a, b in zip(info["grads"], grads):  # products in 32 bits (TF32 is off by default)
        assert float((a.double() - b).norm()) <= 1e-4 * float(b.norm())
    norm = float(torch.stack([g.norm() for g in grads]).norm())
    assert abs(float(info["norm"].norm) - norm) <= 1e-4 * norm


def test_run_and_report(example):
    r = example.train(steps=12, ranks=4, tokens=256, vocabulary=300, width=32, experts=16, k=2)
    assert r["status"] == 0
    assert r["log"][-1]["loss"] < r["log"][0]["loss"]
    for g in r["log"]:
        assert int(g["load"].sum()) == 4 * 256 * 2
        assert 0 < g["coef"] <= 1 and g["norm"] > 0
    spread = [float(g["load"].max()) for g in r["log"]]
    assert spread[-1] < spread[0]  # the bias evens the loads out
    d = r["d"]
    assert d.shape == (12, 4, len(example.STAGES)) and bool((d >= 0).all())
    assert torch.equal(r["windows"].X.sum(1), r["windows"].D)  # increments add up to the makespan


def step_operators(sf, N, V, T, E, seed):
    """A call of every operator on inputs of its own and outputs that are kept: (call, refill, outputs)."""
    dev = torch.device("cuda", torch.cuda.current_device())
    f = lambda *s: torch.empty(s, device=dev)  # noqa: E731
    z, old, ref, A = f(N, V), f(N), f(N), f(N)
    router, dw = f(T, E), f(T, 4)
    target = torch.zeros(N, dtype=torch.int64, device=dev)
    grads = [f(5001), f(70).bfloat16(), f(12345)]

    def refill(k):
        g = torch.Generator(device=dev).manual_seed(seed * 100 + k)
        for t in (z, old, ref, A, router, dw, *grads):
            t.normal_(generator=g)
        target.random_(0, V, generator=g)
        old.sub_(math.log(V))
        ref.sub_(math.log(V))

    d, logp, loss, stats = torch.empty_like(z), f(N), f(N), f(4)
    index, weight = torch.empty((T, 4), dtype=torch.int32, device=dev), f(T, 4)
    load, droute = torch.empty(E, dtype=torch.int32, device=dev), torch.empty_like(router)
    norm, coef, each, out = f(1), f(1), f(3), [torch.empty_like(t) for t in grads]
    status = sf.new_status(dev)
    ws = torch.empty(sf.lib().sf_policy_loss_workspace_size(N, V), dtype=torch.uint8, device=dev)

    def call():
        sf.sf_policy_loss(z, target, old, A, ref_logp=ref, kl_coef=0.1, logp=logp, token_loss=loss, stats=stats,
                          dlogits=d, workspace=ws, status=status)
        sf.sf_route_experts(router, 4, score="sigmoid", index=index, weight=weight, load=load, status=status)
        sf.sf_route_experts_grad(router, index, dw, score="sigmoid", dlogits=droute, status=status)
        sf.sf_grad_clip(grads, 1.0, out=out, norm=norm, coef=coef, tensor_norm=each, status=status)

    return call, refill, [d, logp, loss, stats, index, weight, load, droute, norm, coef, each, *out, status]


SHAPES = [(1, 4099, 3, 64), (3, 40000, 100, 64), (700, 1001, 5000, 160), (20000, 33, 700, 8)]


@pytest.mark.parametrize("shape", SHAPES)
def test_operators_in_a_graph(example, shape):
    """Captured once and replayed on new inputs: the bits of calls outside a graph."""
    call, refill, outputs = step_operators(example.sf, *shape, 1)
    refill(0)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in (1, 2):
        refill(k)
        call()
        want = [t.clone() for t in outputs]
        for t in outputs[:-1]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(outputs[-1].item()) == 0
        for a, b in zip(outputs, want):
            assert torch.equal(a, b)


def test_operators_from_several_threads(example):
    """Threads with streams and buffers of their own, at once: the bits of the same calls one after another."""
    work = [step_operators(example.sf, *shape, 2 + i) for i, shape in enumerate(SHAPES)]
    wants = []
    for call, refill, outputs in work:
        refill(0)
        call()
        wants.append([t.clone() for t in outputs])
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        call, _, outputs = work[i]
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    for t in outputs[:-1]:
                        t.zero_()
                    call()
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(outputs, wants[i])):
                        wrong.append(i)
        except Exception as e:  # shown by the assertion
            wrong.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and all(int(o[-1].item()) == 0 for _, _, o in work)
