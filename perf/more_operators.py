"""Performance cases of the operators around a policy's layers: what a training
job runs between the router and the loss, and what a rollout runs to have tokens.

A case names an operator and its sizes.

  ffn       sf_gated_ffn: act(x Wg^T) * (x Wu^T), x [T][H], weights [F][H]
  ffn_grad  sf_gated_ffn_grad: the gradients of x and of both weights from that of the product
  dropout   sf_dropout: residual + x kept with probability 1 - p and scaled, the mask from counters;
            without residual it is the backward pass
  verify    sf_verify_draft: L drafted tokens for each of B sequences against the target's rows over V entries
"""
import math
import random

import torch

own = False

CELLS = 1 << 25  # logits made, or computed in 64 bits, at a time
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
TAU = 0.9  # inverse temperature of the rollout


def listed():
    return [
        # one token of a running generation: the weights are read for it alone
        dict(name="ffn_one_token", kind="ffn", T=1, H=4096, F=12288, act="silu", dtype="bf16"),
        # a step of a batch of generations
        dict(name="ffn_decode_batch", kind="ffn", T=48, H=2048, F=8192, act="silu", dtype="bf16"),
        # sizes that fill no tile and rows that are not aligned
        dict(name="ffn_ragged", kind="ffn", T=1357, H=1001, F=2731, act="gelu_tanh", dtype="f16"),
        # a rank's micro-batch through a large layer
        dict(name="ffn_micro_batch", kind="ffn", T=8192, H=4096, F=12288, act="silu", dtype="bf16"),
        # its backward pass
        dict(name="ffn_grad_micro_batch", kind="ffn_grad", T=8192, H=4096, F=12288, act="silu", dtype="bf16"),
        # the backward pass of a small layer and a token count that fills no tile
        dict(name="ffn_grad_ragged", kind="ffn_grad", T=1111, H=1016, F=2728, act="gelu", dtype="bf16"),
        # a few sequences' residual stream
        dict(name="dropout_small", kind="dropout", N=8, D=4096, p=0.1, residual=True, dtype="bf16"),
        # the residual stream of a micro-batch
        dict(name="dropout_stream", kind="dropout", N=16384, D=8192, p=0.1, residual=True, dtype="bf16"),
        # the backward pass over rows of an odd length
        dict(name="dropout_backward_odd", kind="dropout", N=4099, D=5001, p=0.25, residual=False, dtype="f32"),
        # one running generation, four drafted tokens
        dict(name="verify_one", kind="verify", B=1, L=4, V=32768, draft=True, greedy=False, ragged=False, dtype="bf16"),
        # a batch of them over a large vocabulary
        dict(name="verify_batch", kind="verify", B=64, L=4, V=131072, draft=True, greedy=False, ragged=False,
             dtype="bf16"),
        # drafts that were looked up in the text (no probabilities), of different lengths; rows of an odd length
        dict(name="verify_lookup_odd", kind="verify", B=24, L=7, V=50001, draft=False, greedy=False, ragged=True,
             dtype="f32"),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "ffn_grad", "ffn_grad", "dropout", "verify", "verify"])
    if kind in ("ffn", "ffn_grad"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        T, H, F = _between(rng, 1, 8192), _between(rng, 64, 4096), _between(rng, 64, 12288)
        if rng.random() < 0.6:  # most layers' widths are multiples of 64, some are not
            H, F = max(64, H // 64 * 64), max(64, F // 64 * 64)
        return dict(kind=kind, T=T, H=H, F=F, act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), dtype=dtype)
    if kind == "dropout":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        D = _between(rng, 64, 16384)
        if rng.random() < 0.5:
            D = max(64, D // 64 * 64)
        return dict(kind=kind, N=_between(rng, 1, min(65536, (1 << (26 if dtype == "f32" else 27)) // D)), D=D,
                    p=rng.choice([0.05, 0.1, 0.25, 0.5]), residual=rng.random() < 0.5, dtype=dtype)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    V, L = _between(rng, 4096, 131072), rng.randint(0, 8)
    if rng.random() < 0.5:
        V = V // 64 * 64
    draft = rng.random() < 0.7
    most = (1 << (26 if dtype != "f32" else 25)) // (V * (2 * L + 2))
    return dict(kind=kind, B=_between(rng, 1, max(1, min(256, most))), L=L, V=V, draft=draft,
                greedy=rng.random() < 0.2, ragged=rng.random() < 0.5, dtype=dtype)


# ---------------------------------------------------------------- inputs


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _normal(gen, rows, columns, dtype, scale):
    out = torch.empty((rows, columns), dtype=TYPES[dtype], device=gen.device)
    step = max(1, CELLS // columns)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        out[a:b] = torch.randn((b - a, columns), generator=gen, device=gen.device).mul_(scale)
    return out


def _ffn_inputs(case, gen):
    T, H, F, dtype = case["T"], case["H"], case["F"], case["dtype"]
    s = dict(x=_normal(gen, T, H, dtype, 1.0), w_gate=_normal(gen, F, H, dtype, H ** -0.5),
             w_up=_normal(gen, F, H, dtype, H ** -0.5))
    if case["kind"] == "ffn_grad":
        s["dh"] = _normal(gen, T, F, dtype, 0.0625)  # gradients times a loss scale
    return s


def _lengths(case, seed):
    """Drafted tokens of each sequence."""
    rng = random.Random(seed * 31 + case["B"])
    return [rng.randint(0, case["L"]) if case["ragged"] else case["L"] for _ in range(case["B"])]


def _softmax64(rows):
    x = rows.double() * TAU
    return torch.softmax(x, -1)


def _verify_inputs(case, seed, gen):
    """Target rows with a few likely tokens each; the draft's rows lie around
    them and its tokens are drawn from them.  No uniform number is within 1e-4
    of the ratio that it is compared with, and no sampled token's value within
    1e-4 of the next one, where the last bit of a sum in 32 bits would decide."""
    dev, B, L, V, dtype = gen.device, case["B"], case["L"], case["V"], case["dtype"]
    target = torch.empty((B, L + 1, V), dtype=TYPES[dtype], device=dev)
    draft = torch.empty((B, L, V), dtype=TYPES[dtype], device=dev) if case["draft"] else None
    token = torch.zeros((B, L), dtype=torch.int64, device=dev)
    uniform = torch.rand((B, L), generator=gen, device=dev)
    noise = torch.empty((B, V), device=dev)
    lengths = _lengths(case, seed)
    for b in range(B):
        z = torch.randn((L + 1, V), generator=gen, device=dev).mul_(1.5)
        likely = torch.randint(0, V, (L + 1, 8), generator=gen, device=dev)
        z.scatter_add_(1, likely, torch.rand((L + 1, 8), generator=gen, device=dev) * 6 + 9)
        target[b] = z
        noise[b].exponential_(generator=gen).clamp_(min=1e-30)
        if L == 0:
            continue
        if case["draft"]:
            draft[b] = z[:L] + torch.randn((L, V), generator=gen, device=dev).mul_(0.7)
            race = torch.empty((L, V), device=dev).exponential_(generator=gen).clamp_(min=1e-30)
            token[b] = (_softmax64(draft[b]) / race).argmax(1)
        else:  # looked up: often the likeliest one
            token[b] = torch.where(torch.rand(L, generator=gen, device=dev) < 0.8, z[:L].argmax(1), likely[:L, 1])
    for b in range(B):
        p = _softmax64(target[b])
        n = lengths[b]
        if L:
            at = token[b][:, None]
            ratio = p[:L].gather(1, at)[:, 0]
            if case["draft"]:
                ratio = ratio / _softmax64(draft[b]).gather(1, at)[:, 0]
            u = uniform[b].double()
            off = u - ratio
            u = torch.where(off.abs() < 1e-4, torch.where(ratio > 0.5, ratio - 1e-3, ratio + 1e-3), u)
            uniform[b] = u.clamp(0.0, 1.0 - 2.0 ** -24).float()
            went = (uniform[b].double() < ratio).tolist()
            k = 0
            while k < n and went[k]:
                k += 1
        else:
            k = 0
        r = p[k]
        if k < n:
            r = r.clone()
            if case["draft"]:
                r = (r - _softmax64(draft[b, k])).clamp(min=0.0)
            else:
                r[token[b, k]] = 0.0
        best = (r / noise[b].double()).topk(2)
        first = best.indices[0]
        close = best.values[1] > best.values[0] * (1 - 1e-4)
        noise[b, first] = torch.where(close, noise[b, first] * 0.99, noise[b, first])
    s = dict(target=target, draft=draft, token=token)
    if not case["greedy"]:
        s["uniform"], s["noise"] = uniform, noise
    if case["ragged"]:
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=_device()).manual_seed(seed)
    if case["kind"] in ("ffn", "ffn_grad"):
        s = _ffn_inputs(case, gen)
    elif case["kind"] == "dropout":
        s = dict(x=_normal(gen, case["N"], case["D"], case["dtype"], 1.0),
                 key=torch.tensor([seed * 0x9E3779B97F4A7C15 % (1 << 63), seed % 1000], dtype=torch.int64,
                                  device=_device()))
        if case["residual"]:
            s["residual"] = _normal(gen, case["N"], case["D"], case["dtype"], 2.0)
    else:
        s = _verify_inputs(case, seed, gen)
    s["case"] = case
    s["status"] = torch.zeros(1, dtype=torch.int32, device=_device())
    return s


# ---------------------------------------------------------------- the plain forms


def _activation(g, act):
    """act(g) and its derivative, by elementary operations in g's type."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    return torch.where(g > 0, g, 0.0), (g > 0).to(g.dtype)


def _plain_ffn(case, s):
    x = s["x"].float()
    a, _ = _activation(x @ s["w_gate"].float().t(), case["act"])
    return (a * (x @ s["w_up"].float().t())).to(s["x"].dtype)


def _plain_ffn_grad(case, s):
    x, wg, wu, dh = (s[n].float() for n in ("x", "w_gate", "w_up", "dh"))
    a, slope = _activation(x @ wg.t(), case["act"])
    du = dh * a
    dg = dh * (x @ wu.t()) * slope
    t = s["x"].dtype
    return dict(dx=(dg @ wg + du @ wu).to(t), dw_gate=(dg.t() @ x).to(t), dw_up=(du.t() @ x).to(t))


def _kept(N, D, p, key):
    """Philox4x32-10 of (pack of 8 columns, row, offset) under the seed: 16 bits for each column."""
    seed, offset = key[0], key[1]
    low = 0xFFFFFFFF
    packs = -(-D // 8)
    dev = key.device
    c0 = torch.arange(packs, device=dev)[None, :].expand(N, packs)
    c1 = torch.arange(N, device=dev)[:, None].expand(N, packs)
    c2, c3 = (offset & low).expand(N, packs), ((offset >> 32) & low).expand(N, packs)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], -1)
    bits = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(N, packs * 8)[:, :D]
    return bits >= int(math.floor(p * 65536 + 0.5))


def _scale(p):
    return 65536 / (65536 - int(math.floor(p * 65536 + 0.5)))


def _plain_dropout(case, s):
    x = torch.where(_kept(case["N"], case["D"], case["p"], s["key"]), s["x"].float() * _scale(case["p"]), 0.0)
    if case["residual"]:
        x = x + s["residual"].float()
    return x.to(s["x"].dtype)


def _plain_softmax(z):
    x = z.float() * TAU
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    return e / total, x - m - torch.log(total)


def _plain_verify(case, s):
    B, L, V = case["B"], case["L"], case["V"]
    dev = s["target"].device
    lengths = s["lengths"].long() if case["ragged"] else torch.full((B,), L, device=dev)
    token = s["token"]
    p, logp = _plain_softmax(s["target"])
    slots = torch.arange(L, device=dev)[None, :]
    if case["greedy"]:
        best = s["target"].float().argmax(-1)
        taken = token == best[:, :L]
    else:
        py = p[:, :L].gather(2, token[:, :, None])[:, :, 0]
        if case["draft"]:
            q, _ = _plain_softmax(s["draft"])
            taken = s["uniform"] * q.gather(2, token[:, :, None])[:, :, 0] < py
        else:
            taken = s["uniform"] < py
    taken = taken & (slots < lengths[:, None])
    accepted = taken.long().cumprod(1).sum(1)
    every = torch.arange(B, device=dev)
    if case["greedy"]:
        last = best[every, accepted]
    else:
        r = p[every, accepted]
        if L:
            stopped = accepted < lengths
            at = accepted.clamp(max=L - 1)
            if case["draft"]:
                left = (r - q[every, at]).clamp(min=0.0)
                left = torch.where((left > 0).any(1, keepdim=True), left, r)
            else:
                left = r.scatter(1, token[every, at][:, None], 0.0)
            r = torch.where(stopped[:, None], left, r)
        last = (r / s["noise"]).argmax(1)
    out = torch.cat([token, torch.zeros((B, 1), dtype=torch.int64, device=dev)], 1)
    out.scatter_(1, accepted[:, None], last[:, None])
    used = torch.arange(L + 1, device=dev)[None, :] <= accepted[:, None]
    lp = logp.gather(2, out[:, :, None])[:, :, 0]
    return dict(token=torch.where(used, out, -1), accepted=accepted.to(torch.int32), logp=torch.where(used, lp, 0.0))


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        return _own(case, kind, state)
    if kind == "ffn":
        return _plain_ffn(case, state)
    if kind == "ffn_grad":
        return _plain_ffn_grad(case, state)
    if kind == "dropout":
        return _plain_dropout(case, state)
    return _plain_verify(case, state)


# ---------------------------------------------------------------- the framework's operators


def _own(case, kind, s):
    from paper_2606_06751_gb300 import stagefrontier as sf
    if kind == "ffn":
        return sf.sf_gated_ffn(s["x"], s["w_gate"], s["w_up"], act=case["act"], status=s["status"])
    if kind == "ffn_grad":
        r = sf.sf_gated_ffn_grad(s["x"], s["w_gate"], s["w_up"], s["dh"], act=case["act"], status=s["status"])
        return dict(dx=r.dx, dw_gate=r.dw_gate, dw_up=r.dw_up)
    if kind == "dropout":
        return sf.sf_dropout(s["x"], case["p"], s["key"], residual=s.get("residual"))
    r = sf.sf_verify_draft(s["target"], s["token"], draft=s["draft"], lengths=s.get("lengths"),
                           uniform=s.get("uniform"), noise=s.get("noise"), inv_temperature=TAU, status=s["status"])
    return dict(token=r.token, accepted=r.accepted, logp=r.logp)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    kind = case["kind"]
    b = BYTES[case["dtype"]]
    if kind in ("ffn", "ffn_grad"):
        T, H, F = case["T"], case["H"], case["F"]
        if kind == "ffn":
            return {"bytes": b * (T * H + 2 * F * H + T * F), "flops": 4 * T * H * F}
        return {"bytes": b * (2 * T * H + 4 * F * H + T * F), "flops": 12 * T * H * F}
    if kind == "dropout":
        return {"bytes": b * case["N"] * case["D"] * (3 if case["residual"] else 2) + 16,
                "flops": case["N"] * case["D"] * (2 if case["residual"] else 1)}
    B, L, V = case["B"], case["L"], case["V"]
    n = B * L // 2 if case["ragged"] else B * L  # drafted tokens
    rows = n + B + (n if case["draft"] and not case["greedy"] else 0)
    values = rows * V
    return {"bytes": values * b + (0 if case["greedy"] else B * V * 4 + n * 4) + n * 8 + B * (L + 1) * 12 + B * 4,
            "flops": 4 * values}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_activation(g, act):
    """act(g) and its derivative by other formulas than the plain form's."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    if act == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":  # (1 + tanh y) / 2 = sigmoid(2 y)
        k = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(k * (g + 0.044715 * g ** 3))
        return g * s, s + g * s * (1 - s) * k * (1 + 0.134145 * g ** 2)
    return g.clamp(min=0.0), torch.heaviside(g, torch.zeros_like(g))


def _exact_ffn(case, s, grad):
    x, wg, wu = (s[n].double() for n in ("x", "w_gate", "w_up"))
    g, u = torch.einsum("th,fh->tf", x, wg), torch.einsum("th,fh->tf", x, wu)
    a, slope = _exact_activation(g, case["act"])
    if not grad:
        return a * u
    dh = s["dh"].double()
    dg, du = slope * u * dh, a * dh
    return dict(dx=torch.einsum("tf,fh->th", dg, wg) + torch.einsum("tf,fh->th", du, wu),
                dw_gate=torch.einsum("tf,th->fh", dg, x), dw_up=torch.einsum("tf,th->fh", du, x))


def _exact_dropout(case, s):
    out = s["residual"].double() if case["residual"] else torch.zeros_like(s["x"], dtype=torch.float64)
    step = max(1, CELLS // case["D"])
    kept = _kept(case["N"], case["D"], case["p"], s["key"])
    for a in range(0, case["N"], step):
        k = kept[a:a + step]
        out[a:a + step][k] += s["x"][a:a + step].double()[k] * _scale(case["p"])
    return out


def _exact_verify(case, s):
    """Sequence by sequence, token by token; the whole numbers have no value in 64 bits."""
    B, L = case["B"], case["L"]
    logp = torch.zeros((B, L + 1), dtype=torch.float64, device=s["target"].device)
    lengths = s["lengths"].tolist() if case["ragged"] else [L] * B
    for b in range(B):
        z = s["target"][b].double() * TAU
        lp = z - torch.logsumexp(z, 1, keepdim=True)
        ys, k = s["token"][b].tolist(), 0
        lq = None
        if case["draft"] and L and not case["greedy"]:
            q = s["draft"][b].double() * TAU
            lq = q - torch.logsumexp(q, 1, keepdim=True)
        while k < lengths[b]:
            y = ys[k]
            if case["greedy"]:
                if int(z[k].argmax()) != y:
                    break
            else:
                ratio = math.exp(float(lp[k, y]) - (float(lq[k, y]) if lq is not None else 0.0))
                if not float(s["uniform"][b, k]) < ratio:
                    break
            logp[b, k] = lp[k, y]
            k += 1
        if case["greedy"]:
            y = int(z[k].argmax())
        else:
            r = lp[k].exp()
            if k < lengths[b]:
                if lq is not None:
                    r = (r - lq[k].exp()).clamp(min=0.0)
                else:
                    r[ys[k]] = 0.0
            y = int((r / s["noise"][b].double()).argmax())
        logp[b, k] = lp[k, y]
    return dict(token=None, accepted=None, logp=logp)


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind in ("ffn", "ffn_grad"):
        return _exact_ffn(case, s, kind == "ffn_grad")
    if kind == "dropout":
        return _exact_dropout(case, s)
    return _exact_verify(case, s)
