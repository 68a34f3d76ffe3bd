"""Performance cases of the training-step operators: what a monitor inside a
training job computes beside the times of the step's stages.

A case names an operator and its sizes.

  score       sf_policy_loss without gradients: log-probabilities of N chosen
              tokens from logits over V entries, and their loss
  loss        sf_policy_loss with the gradient of the logits
  route       sf_route_experts: T tokens to k of E experts, the experts' loads
  route_grad  sf_route_experts_grad: the gradient of the router's logits
  norm        sf_grad_norm: the norm over n gradient tensors, and each one's
  clip        sf_grad_clip: the norm and the clipped copies of the gradients
"""
import math
import random

import torch

own = False

CELLS = 1 << 26  # logits made, or computed in 64 bits, at a time
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
SEQUENCE = 512  # tokens of a sequence; the first ones are the prompt and carry no loss
CLIP, KL, TAU = (0.2, 0.28), 0.05, 1.0
MAX_NORM, EPS = 1.0, 1e-6


def listed():
    return [
        # the token just generated, scored as it comes: the smallest call there is
        dict(name="score_one_token", kind="score", N=1, V=65536, dtype="bf16", masked=0.0),
        # a batch of responses scored by the policy that wrote them; rows of an odd length
        dict(name="score_batch_odd", kind="score", N=4095, V=50001, dtype="f32", masked=0.0),
        # one sequence of a micro-batch, half of it prompt
        dict(name="loss_one_sequence", kind="loss", N=512, V=32768, dtype="bf16", masked=0.5),
        # a rank's whole micro-batch over a large vocabulary
        dict(name="loss_micro_batch", kind="loss", N=8192, V=131072, dtype="bf16", masked=0.25),
        # one token of a running generation
        dict(name="route_one_token", kind="route", T=1, E=64, k=6, groups=1, top_groups=1, score="softmax",
             renorm=True, dtype="bf16"),
        # a layer's router over a micro-batch, experts in groups by node
        dict(name="route_groups", kind="route", T=65536, E=256, k=8, groups=8, top_groups=4, score="sigmoid",
             renorm=True, dtype="f32"),
        # its backward pass for a smaller micro-batch
        dict(name="route_grad_groups", kind="route_grad", T=16384, E=256, k=8, groups=8, top_groups=4,
             score="sigmoid", renorm=True, dtype="f32"),
        # a token count and an expert count that fill no tile, probabilities of all experts in each gradient
        dict(name="route_grad_ragged", kind="route_grad", T=100003, E=160, k=6, groups=1, top_groups=1,
             score="softmax", renorm=False, dtype="bf16"),
        # an adapter's gradients
        dict(name="norm_adapter", kind="norm", n=24, total=1200000, dtype="f32", packed=False),
        # a rank's gradients of a large model
        dict(name="norm_model", kind="norm", n=400, total=1500000000, dtype="bf16", packed=False),
        # gradients of both types in buckets without padding: views that start anywhere
        dict(name="clip_packed", kind="clip", n=150, total=30000001, dtype="mixed", packed=True),
        # a rank's gradients, clipped into the buffers that the optimizer reads
        dict(name="clip_model", kind="clip", n=300, total=1000000000, dtype="bf16", packed=False),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["score", "loss", "loss", "route", "route_grad", "norm", "clip"])
    if kind in ("score", "loss"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        V = _between(rng, 4096, 131072)
        if rng.random() < 0.5:  # half of the vocabularies are padded
            V = V // 64 * 64
        most = (1 << 30 if dtype != "f32" else 1 << 29) // V
        return dict(kind=kind, N=_between(rng, 1, min(8192, most)), V=V, dtype=dtype,
                    masked=rng.choice([0.0, 0.25, 0.5]))
    if kind in ("route", "route_grad"):
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _between(rng, 8 if groups == 1 else 4, 512 // groups)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(12, E // groups * top_groups))
        return dict(kind=kind, T=_between(rng, 1, (1 << 24) // E), E=E, k=k, groups=groups, top_groups=top_groups,
                    score=rng.choice(["softmax", "sigmoid"]), renorm=rng.random() < 0.7,
                    dtype=rng.choice(["bf16", "f32"]))
    n = _between(rng, 1, 400)
    return dict(kind=kind, n=n, total=_between(rng, max(1000, 4 * n), 1000000000),
                dtype=rng.choice(["bf16", "f16", "f32", "mixed"]), packed=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _active(case):
    """Whether each row carries loss: the first `masked` of every sequence is prompt."""
    L = min(SEQUENCE, case["N"])
    return [i % L >= int(case["masked"] * L) for i in range(case["N"])]


def _loss_inputs(case, seed):
    """Logits around a chosen token of log-probability -10 to 0; the policy that
    wrote the tokens and the reference lie near the present one.  No log ratio is
    within 1e-3 of a clipping bound, where the last bit of a sum in 32 bits
    would say whether a row is clipped."""
    dev, N, V = _device(), case["N"], case["V"]
    gen = torch.Generator(device=dev).manual_seed(seed)
    logits = torch.empty((N, V), dtype=TYPES[case["dtype"]], device=dev)
    target = torch.randint(0, V, (N,), generator=gen, device=dev)
    boost = torch.rand((N, 1), generator=gen, device=dev) * 10 + 4
    logp = torch.empty(N, device=dev)
    step = max(1, CELLS // V)
    for a in range(0, N, step):
        b = min(N, a + step)
        x = torch.randn((b - a, V), generator=gen, device=dev).mul_(2.0)
        x.scatter_add_(1, target[a:b, None], boost[a:b])
        logits[a:b] = x
        x = logits[a:b].float().mul_(TAU)
        logp[a:b] = x.gather(1, target[a:b, None])[:, 0] - x.logsumexp(1)
    ratio = torch.randn(N, generator=gen, device=dev) * 0.2
    for bound in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
        off = ratio - bound
        ratio = torch.where(off.abs() < 1e-3, bound + torch.where(off < 0, -1e-3, 1e-3), ratio)
    per = min(SEQUENCE, N)
    advantage = torch.randn(-(-N // per), generator=gen, device=dev).repeat_interleave(per)[:N].contiguous()
    active = torch.tensor(_active(case), device=dev)
    return dict(logits=logits, target=target, old_logp=logp - ratio, advantage=advantage,
                ref_logp=logp - torch.randn(N, generator=gen, device=dev) * 0.3,
                weight=active.float() / active.sum())


def _route_inputs(case, seed):
    """Router logits with experts that are liked more than others."""
    dev, T, E = _device(), case["T"], case["E"]
    gen = torch.Generator(device=dev).manual_seed(seed)
    logits = torch.randn((T, E), generator=gen, device=dev).mul_(1.5)
    logits += torch.randn(E, generator=gen, device=dev) * 0.5
    bias = torch.randn(E, generator=gen, device=dev) * 0.05
    return dict(logits=logits.to(TYPES[case["dtype"]]), bias=bias), gen


def _sizes(case):
    """Sizes and types of a model's tensors: a few large ones, many small ones."""
    rng = random.Random(case["n"] * 7919 + case["total"])
    share = [rng.lognormvariate(0.0, 2.0) for _ in range(case["n"])]
    scale = case["total"] / sum(share)
    sizes = [max(1, int(s * scale)) for s in share]
    types = [case["dtype"] if case["dtype"] != "mixed" else rng.choice(["bf16", "f32"]) for _ in sizes]
    return sizes, types


def _views(case):
    """The tensors as views of one buffer a type, with their places in it."""
    sizes, types = _sizes(case)
    end, places = {}, []
    for n, t in zip(sizes, types):
        at = end.get(t, 0)
        places.append((t, at, n))
        end[t] = at + n if case["packed"] else -(-(at + n) // 64) * 64
    return places, end


def _gradients(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    places, end = _views(case)
    flat = {t: torch.empty(n, dtype=TYPES[t], device=dev).normal_(generator=gen) for t, n in end.items()}
    grads = [flat[t][at:at + n] for t, at, n in places]
    for g in grads:  # layers differ in the size of their gradients; the norm is a few times MAX_NORM
        g.mul_(3.0 * rng.lognormvariate(0.0, 0.5) / math.sqrt(case["total"]))
    state = dict(grads=grads)
    if case["kind"] == "clip":
        state["flat"] = {t: torch.zeros(n, dtype=TYPES[t], device=dev) for t, n in end.items()}
        state["out"] = [state["flat"][t][at:at + n] for t, at, n in places]
    return state


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("score", "loss"):
        state = _loss_inputs(case, seed)
    elif kind in ("route", "route_grad"):
        state, gen = _route_inputs(case, seed)
        if kind == "route_grad":
            state["index"] = _plain_route(case, state)["index"]
            state["dweight"] = torch.randn(state["index"].shape, generator=gen, device=_device())
    else:
        state = _gradients(case, seed)
    state["case"] = case
    state["status"] = torch.zeros(1, dtype=torch.int32, device=_device())
    return state


# ---------------------------------------------------------------- the plain forms


def _plain_loss(case, s, grad):
    x = s["logits"].float() * TAU
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1)
    active = s["weight"] != 0
    logp = x.gather(1, s["target"][:, None])[:, 0] - m[:, 0] - torch.log(total)
    ratio = torch.exp(logp - s["old_logp"])
    free = ratio * s["advantage"]
    held = ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * s["advantage"]
    clipped = held < free
    diff = s["ref_logp"] - logp
    policy, kl = -torch.minimum(free, held), torch.exp(diff) - diff - 1
    loss = policy + KL * kl
    terms = torch.stack([loss, policy, kl, clipped.float()])
    stats = torch.where(active, terms * s["weight"], 0.0).sum(1)
    out = dict(logp=torch.where(active, logp, 0.0), token_loss=torch.where(active, loss, 0.0), stats=stats)
    if grad:
        c = KL * (1 - torch.exp(diff)) - torch.where(clipped, 0.0, free)
        c = torch.where(active, c * s["weight"] * TAU, 0.0)
        d = e.mul_((-c / total)[:, None])
        d.scatter_add_(1, s["target"][:, None], c[:, None])
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_route(case, s):
    z, (T, E), k, G = s["logits"].float(), s["logits"].shape, case["k"], case["groups"]
    score = 1 / (1 + torch.exp(-z)) if case["score"] == "sigmoid" else z
    choice = score + s["bias"]
    if case["top_groups"] < G:
        best = choice.view(T, G, E // G).sort(dim=2, descending=True).values
        value = best[:, :, 0] + best[:, :, 1] if E // G > 1 else best[:, :, 0]
        kept = value.sort(dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=z.device).scatter_(1, kept, True)
        choice = torch.where(keep.repeat_interleave(E // G, 1), choice, -math.inf)
    index = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    chosen = score.gather(1, index)
    if case["score"] == "softmax":
        chosen = torch.exp(chosen - z.amax(1, keepdim=True))
    if case["renorm"]:
        weight = chosen / chosen.sum(1, keepdim=True)
    elif case["score"] == "softmax":
        weight = chosen / torch.exp(z - z.amax(1, keepdim=True)).sum(1, keepdim=True)
    else:
        weight = chosen
    load = torch.zeros(E, dtype=torch.int32, device=z.device)
    load.index_add_(0, index.reshape(-1), torch.ones(T * k, dtype=torch.int32, device=z.device))
    return dict(index=index.to(torch.int32), weight=weight, load=load)


def _plain_route_grad(case, s):
    z, index = s["logits"].float(), s["index"].long()
    dw = torch.zeros_like(z).scatter_(1, index, s["dweight"])
    chosen = torch.zeros_like(z).scatter_(1, index, 1.0)
    if case["score"] == "sigmoid":
        p = 1 / (1 + torch.exp(-z))
        slope = p * (1 / (1 + torch.exp(z)))
        if case["renorm"]:
            total = (p * chosen).sum(1, keepdim=True)
            d = slope / total * (dw - chosen * (dw * p).sum(1, keepdim=True) / total)
        else:
            d = slope * dw
    else:
        e = torch.exp(z - z.amax(1, keepdim=True))
        e = e * chosen if case["renorm"] else e
        p = e / e.sum(1, keepdim=True)
        d = p * (dw - (p * dw).sum(1, keepdim=True))
    return d.to(s["logits"].dtype)


def _plain_norm(s):
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    return squares.sum().sqrt().reshape(1), squares.sqrt()


def _plain_clip(s):
    norm, each = _plain_norm(s)
    coef = (MAX_NORM / (norm + EPS)).clamp(max=1.0)
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * coef)
    return dict(norm=norm, tensor_norm=each, coef=coef, out=s["flat"])


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        return _own(case, kind, state)
    if kind in ("score", "loss"):
        return _plain_loss(case, state, kind == "loss")
    if kind == "route":
        return _plain_route(case, state)
    if kind == "route_grad":
        return _plain_route_grad(case, state)
    if kind == "norm":
        norm, each = _plain_norm(state)
        return dict(norm=norm, tensor_norm=each)
    return _plain_clip(state)


# ---------------------------------------------------------------- the framework's operators


def _own(case, kind, s):
    from paper_2606_06751_gb300 import stagefrontier as sf
    if kind in ("score", "loss"):
        r = sf.sf_policy_loss(s["logits"], s["target"], s["old_logp"], s["advantage"], ref_logp=s["ref_logp"],
                              weight=s["weight"], clip=CLIP, kl_coef=KL, inv_temperature=TAU, grad=kind == "loss",
                              status=s["status"])
        out = dict(logp=r.logp, token_loss=r.token_loss, stats=r.stats)
        if kind == "loss":
            out["dlogits"] = r.dlogits
        return out
    if kind == "route":
        r = sf.sf_route_experts(s["logits"], case["k"], bias=s["bias"], score=case["score"], groups=case["groups"],
                                top_groups=case["top_groups"], renorm=case["renorm"], status=s["status"])
        return dict(index=r.index, weight=r.weight, load=r.load)
    if kind == "route_grad":
        return sf.sf_route_experts_grad(s["logits"], s["index"], s["dweight"], score=case["score"],
                                        renorm=case["renorm"], status=s["status"])
    if kind == "norm":
        r = sf.sf_grad_norm(s["grads"], per_tensor=True, status=s["status"])
        return dict(norm=r.norm, tensor_norm=r.tensor_norm)
    r = sf.sf_grad_clip(s["grads"], MAX_NORM, out=s["out"], eps=EPS, per_tensor=True, status=s["status"])
    return dict(norm=r.norm, tensor_norm=r.tensor_norm, coef=r.coef, out=s["flat"])


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    kind = case["kind"]
    if kind in ("score", "loss"):
        N, V, b = case["N"], case["V"], BYTES[case["dtype"]]
        active = sum(_active(case))
        rows = active * 20 + N * 4 + N * 8 + 16  # token, three numbers, weight; log-probability, loss; sums
        return {"bytes": active * V * b + rows + (N * V * b if kind == "loss" else 0),
                "flops": active * V * (6 if kind == "loss" else 4)}
    if kind in ("route", "route_grad"):
        T, E, k, b = case["T"], case["E"], case["k"], BYTES[case["dtype"]]
        if kind == "route":
            return {"bytes": T * E * b + E * 4 + T * k * 8 + E * 4, "flops": T * E * (5 + k)}
        dense = case["score"] == "softmax" and not case["renorm"]
        read = T * E * b if dense else T * k * b
        return {"bytes": read + T * k * 8 + T * E * b, "flops": T * (E * 5 if dense else k * 10)}
    sizes, types = _sizes(case)
    data = sum(n * BYTES[t] for n, t in zip(sizes, types))
    if kind == "norm":
        return {"bytes": data + 4 * case["n"] + 4, "flops": 2 * sum(sizes)}
    return {"bytes": 2 * data + 4 * case["n"] + 8, "flops": 3 * sum(sizes)}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_loss(case, s, grad):
    N, V = case["N"], case["V"]
    lo, hi = CLIP
    logp, loss, terms, grads = [], [], [], []
    step = max(1, CELLS // V)
    for a in range(0, N, step):
        b = min(N, a + step)
        w, A = s["weight"][a:b].double(), s["advantage"][a:b].double()
        y = s["target"][a:b, None]
        x = s["logits"][a:b].double() * TAU
        p = torch.log_softmax(x, 1)
        lp = p.gather(1, y)[:, 0]
        r = (lp - s["old_logp"][a:b].double()).exp()
        up = torch.where(A >= 0, r.clamp(max=1 + hi), r.clamp(min=1 - lo))  # the bound that can hold a ratio back
        clipped = up != r
        u = (s["ref_logp"][a:b].double() - lp)
        kl = torch.expm1(u) - u
        l = -up * A + KL * kl
        on = w != 0
        logp.append(torch.where(on, lp, 0.0))
        loss.append(torch.where(on, l, 0.0))
        terms.append((torch.stack([l, -up * A, kl, clipped.double()]) * w).sum(1))
        if grad:
            c = torch.where(clipped, 0.0, -A * r) - KL * torch.expm1(u)
            d = -p.exp_()
            d.scatter_add_(1, y, torch.ones_like(y, dtype=torch.float64))
            grads.append(d * (c * w * TAU)[:, None])
    out = dict(logp=torch.cat(logp), token_loss=torch.cat(loss), stats=torch.stack(terms).sum(0))
    if grad:
        out["dlogits"] = torch.cat(grads)
    return out


def _exact_route(case, s):
    """The choice as it is made in 32 bits, its weights in 64."""
    index = _plain_route(case, s)["index"].long()
    z = s["logits"].double()
    p = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, 1)
    p = p.gather(1, index)
    return dict(index=None, weight=p / p.sum(1, keepdim=True) if case["renorm"] else p, load=None)


def _exact_route_grad(case, s):
    """By the chain rule through the weights' Jacobian, slot by slot."""
    z, index, dw = s["logits"].double(), s["index"].long(), s["dweight"].double()
    d = torch.zeros_like(z)
    if case["score"] == "sigmoid":
        p = torch.sigmoid(z.gather(1, index))
        inner = dw
        if case["renorm"]:
            t = p.sum(1, keepdim=True)
            inner = dw / t - (dw * p).sum(1, keepdim=True) / t ** 2
        return d.scatter_(1, index, inner * p * torch.sigmoid(-z.gather(1, index)))
    if case["renorm"]:
        p = torch.softmax(z.gather(1, index), 1)
        return d.scatter_(1, index, p * dw - p * (p * dw).sum(1, keepdim=True))
    p = torch.softmax(z, 1)
    q = p.gather(1, index)
    return d.scatter_(1, index, q * dw) - p * (q * dw).sum(1, keepdim=True)


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind in ("score", "loss"):
        return _exact_loss(case, s, kind == "loss")
    if kind == "route":
        return _exact_route(case, s)
    if kind == "route_grad":
        return _exact_route_grad(case, s)
    squares = torch.stack([sum(c.double().square().sum() for c in g.split(1 << 27)) for g in s["grads"]])
    norm, each = squares.sum().sqrt().reshape(1), squares.sqrt()
    if kind == "norm":
        return dict(norm=norm, tensor_norm=each)
    coef = (MAX_NORM / (norm + EPS)).clamp(max=1.0)
    out = {t: torch.zeros(f.shape, dtype=torch.float64, device=f.device) for t, f in s["flat"].items()}
    for g, (t, at, n) in zip(s["grads"], _views(case)[0]):
        out[t][at:at + n] = g.double() * coef
    return dict(norm=norm, tensor_norm=each, coef=coef, out=out)
