"""The example's training step: its gradients against the same step in plain
64-bit operations, and a run of it with its report."""
import os
import sys

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
