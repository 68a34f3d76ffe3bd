"""A training job that computes its own report.

A small policy with a layer of experts is trained on one GPU.  Its ranks are a
data axis: each owns a shard of the experts and a micro-batch of tokens, and
each rank's part of every stage is timed by events.  The step's operators are
the library's: routing with the experts' loads, the clipped policy loss with a
KL term, the gradient norm and clipping.  At the end the durations d[T][R][S]
go through the frontier accounting, and the report sets side by side which
(stage, rank) exposed the step's time and what that rank's load was, before and
after the routing bias has balanced it.

    python examples/monitored_step.py [--steps 40]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2606_06751_gb300 import stagefrontier as sf  # noqa: E402

STAGES = ("data", "router", "experts", "loss", "backward", "optimizer")


class Route(torch.autograd.Function):
    """Router logits -> weights of the chosen experts."""

    @staticmethod
    def forward(ctx, logits, bias, k, load, status):
        r = sf.sf_route_experts(logits, k, bias=bias, score="sigmoid", load=load, accumulate=True, status=status)
        ctx.save_for_backward(logits, r.index)
        ctx.status = status
        ctx.mark_non_differentiable(r.index)
        return r.weight, r.index

    @staticmethod
    def backward(ctx, dweight, _):
        logits, index = ctx.saved_tensors
        d = sf.sf_route_experts_grad(logits, index, dweight.contiguous(), score="sigmoid", status=ctx.status)
        return d, None, None, None, None


class Policy(torch.autograd.Function):
    """Logits -> loss; the gradient is computed with the loss and kept."""

    @staticmethod
    def forward(ctx, logits, batch, kl_coef, status):
        r = sf.sf_policy_loss(logits, batch["target"], batch["old_logp"], batch["advantage"],
                              ref_logp=batch["ref_logp"], weight=batch["weight"], kl_coef=kl_coef, grad=True,
                              status=status)
        ctx.save_for_backward(r.dlogits)
        ctx.mark_non_differentiable(r.stats)
        return r.stats[0], r.stats

    @staticmethod
    def backward(ctx, grad, _):
        (dlogits,) = ctx.saved_tensors
        return dlogits * grad, None, None, None


class Model:
    """An embedding, a layer of experts of which a token uses k, and a head."""

    def __init__(self, vocabulary, width, experts, k, seed, device):
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s: (torch.randn(*s, device=device, generator=g) * s[-2] ** -0.5).requires_grad_()  # noqa: E731
        self.k, self.experts = k, experts
        self.embedding, self.router = new(vocabulary, width), new(width, experts)
        self.up, self.head = new(experts, width, width), new(width, vocabulary)
        with torch.no_grad():  # a layer that likes its first experts better
            self.embedding.mul_(vocabulary ** 0.5)
            self.embedding[:, 0] = 1.0
            self.router[0, : experts // 8] += 2.0
        self.bias = torch.zeros(experts, device=device)

    def parameters(self):
        return [self.embedding, self.router, self.up, self.head]

    def experts_of(self, x, index, weight, shard):
        """What the experts in `shard` add to the tokens that were sent to them."""
        out = torch.zeros_like(x)
        for e in shard:
            token, slot = (index == e).nonzero(as_tuple=True)
            if token.numel():
                out = out.index_add(0, token, torch.relu(x[token] @ self.up[e]) * weight[token, slot, None])
        return out


def batch_of(tokens, vocabulary, gen, device):
    """A micro-batch: contexts, the tokens that were chosen, and what the policy that chose them said."""
    context = torch.randint(0, vocabulary, (tokens,), generator=gen, device=device)
    weight = (torch.arange(tokens, device=device) % 32 >= 8).float()  # prompts carry no loss
    uniform = torch.full((tokens,), -float(torch.tensor(vocabulary).log()), device=device)
    return dict(context=context, target=(context * 7 + 3) % vocabulary, old_logp=uniform, ref_logp=uniform.clone(),
                advantage=torch.ones(tokens, device=device), weight=weight / weight.sum())


class Clock:
    """Stage durations of the ranks of one step, by events."""

    def __init__(self):
        self.spans = []

    def __call__(self, rank, stage):
        return _Span(self, rank, stage)

    def durations(self, ranks):
        d = torch.zeros(ranks, len(STAGES), dtype=torch.int64)
        for rank, stage, a, b in self.spans:
            ns = int(a.elapsed_time(b) * 1e6)
            if rank is None:  # all ranks together
                d[:, STAGES.index(stage)] += ns
            else:
                d[rank, STAGES.index(stage)] += ns
        return d


class _Span:
    def __init__(self, clock, rank, stage):
        self.clock, self.key = clock, (rank, stage)

    def __enter__(self):
        self.a = torch.cuda.Event(enable_timing=True)
        self.a.record()

    def __exit__(self, *_):
        b = torch.cuda.Event(enable_timing=True)
        b.record()
        self.clock.spans.append((*self.key, self.a, b))


def step(model, ranks, tokens, gen, lr, max_norm, kl_coef, status):
    """One optimizer step over the ranks' micro-batches; (durations [R][S], what a monitor logs)."""
    device, E = model.bias.device, model.experts
    clock, load = Clock(), torch.zeros(E, dtype=torch.int32, device=device)
    batches, hidden, weights, indices = [], [], [], []
    for r in range(ranks):
        with clock(r, "data"):
            batches.append(batch_of(tokens, model.embedding.shape[0], gen, device))
        with clock(r, "router"):
            x = model.embedding[batches[r]["context"]]
            w, i = Route.apply(x @ model.router, model.bias, model.k, load, status)
        hidden.append(x)
        weights.append(w)
        indices.append(i)
    x, w, i = torch.cat(hidden), torch.cat(weights), torch.cat(indices)
    shard = E // ranks
    added = []
    for r in range(ranks):  # a rank's experts work on all ranks' tokens that were sent to them
        with clock(r, "experts"):
            added.append(model.experts_of(x, i, w, range(r * shard, (r + 1) * shard)))
    h = x + sum(added)
    losses, stats = [], []
    for r in range(ranks):
        with clock(r, "loss"):
            loss, s = Policy.apply(h[r * tokens:(r + 1) * tokens] @ model.head, batches[r], kl_coef, status)
        losses.append(loss)
        stats.append(s)
    with clock(None, "backward"):
        grads = torch.autograd.grad(sum(losses) / ranks, model.parameters())
    with clock(None, "optimizer"):
        grads = [g.contiguous() for g in grads]
        norm = sf.sf_grad_clip(grads, max_norm, per_tensor=True, status=status)
        with torch.no_grad():
            for p, g in zip(model.parameters(), grads):
                p -= lr * g
            model.bias += 0.02 * torch.sign(load.float().mean() - load)  # towards even loads
    torch.cuda.synchronize()
    return clock.durations(ranks), dict(stats=torch.stack(stats).mean(0), load=load, norm=norm, grads=grads)


def train(steps=40, ranks=8, tokens=512, vocabulary=1000, width=64, experts=32, k=4, lr=1.0, max_norm=0.15,
          kl_coef=0.02, seed=0):
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(vocabulary, width, experts, k, seed, device)
    gen = torch.Generator(device=device).manual_seed(seed + 1)
    status = sf.new_status(device)
    step(model, ranks, tokens, gen, 0.0, max_norm, kl_coef, status)  # warm-up: no update
    model.bias.zero_()
    durations, log = [], []
    for _ in range(steps):
        d, info = step(model, ranks, tokens, gen, lr, max_norm, kl_coef, status)
        durations.append(d)
        log.append({"loss": float(info["stats"][0]), "kl": float(info["stats"][2]), "clipped": float(info["stats"][3]),
                    "norm": float(info["norm"].norm), "coef": float(info["norm"].coef), "load": info["load"].cpu()})
    d = torch.stack(durations).to(device)
    window = max(1, steps // 2)
    win = sf.sf_window_aggregate(d, window, status=status)
    top = sf.sf_topk_suspects(win.X, win.E, 1)
    labels = sf.sf_label_windows(d, window, status=status)
    torch.cuda.synchronize()
    return dict(d=d, log=log, windows=win, suspects=top, labels=labels, status=int(status.item()), window=window,
                shard=experts // ranks)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    r = train(a.steps)
    print("device status", r["status"])
    for t in range(0, a.steps, max(1, a.steps // 8)):
        g = r["log"][t]
        print(f"step {t:3d}  loss {g['loss']:8.4f}  kl {g['kl']:.4f}  clipped {g['clipped']:.2f}  "
              f"norm {g['norm']:.3f} x {g['coef']:.3f}")
    share = r["windows"].X.double() / r["windows"].D.double()[:, None]
    for w in range(share.shape[0]):
        stage, rank = r["suspects"].pair[w, 0].tolist()
        experts = STAGES.index("experts")
        lead = int(r["windows"].E[w, experts].argmax())  # the rank that the stage's exposed time is credited to
        logs = r["log"][w * r["window"]:(w + 1) * r["window"]]
        load = torch.stack([g["load"] for g in logs]).sum(0).view(-1, r["shard"]).sum(1).double()
        names = [n for b, n in enumerate(sf.LABEL_NAMES) if int(r["labels"].labels[w]) >> b & 1]
        print(f"window {w}: " + ", ".join(f"{s} {float(v):.0%}" for s, v in zip(STAGES, share[w])))
        print(f"  first suspect {STAGES[stage]} of rank {rank}; {', '.join(names)}")
        print(f"  experts: led by rank {lead}, whose load is {float(load[lead] / load.mean()):.2f} of an even one "
              f"(largest: rank {int(load.argmax())}, {float(load.max() / load.mean()):.2f})")


if __name__ == "__main__":
    main()
