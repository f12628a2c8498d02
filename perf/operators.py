"""Timed cases of the operators that a policy update takes beside the model's own passes, through the package's public
entry points and in plain torch.

Both ends of an update are here: what it reads of the output head, and how it moves the weight matrices.  Kinds:

  stats   token_stats: log-probabilities of given tokens, entropies and the most likely alternatives of every row, from
          hidden rows [t, d] and the output matrix [v, d]; no logits are given or returned
  grad    token_stats_backward: from the gradients of the log-probabilities and entropies to those of both operands
  orth    orthogonalize: Newton-Schulz iteration on a batch of matrices [batch, rows, cols]
  muon    muon_step: momentum, orthogonalised update and weights of all matrices of "layers" decoder layers of width d

`own` False computes the plain forms: products, sums, exp, comparisons and indexing in 32 bits.

Sizes are those of the benchmark's model shapes (widths 512, 768, 2048 and 2560, a vocabulary of 50,304, responses of 53 tokens)
or odd ones between them.
"""
import math

import torch

own = False  # set from outside: True makes run() call the package

DEVICE = "cuda:0"
TEMPERATURE = 0.7
VOCAB = 50304
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
COEFFS = (3.4445, -4.7750, 2.0315)  # of the quintic Newton-Schulz step
STEPS, EPS = 5, 1e-7
LR, MOMENTUM, DECAY, RMS = 3e-6, 0.95, 0.01, 0.2  # the paper's learning rate


def _head(name, kind, t, d, v, dtype, top=0):
    return dict(name=name, kind=kind, t=t, d=d, v=v, dtype=dtype, top=top)


def _orth(name, batch, rows, cols, dtype):
    return dict(name=name, kind="orth", batch=batch, rows=rows, cols=cols, dtype=dtype)


def _muon(name, layers, d):
    return dict(name=name, kind="muon", layers=layers, d=d)


def listed():
    return [
        # one token of one sequence at the 2.8B width, with its alternatives: latency while looking at samples
        _head("stats-2.8b-one", "stats", 1, 2560, VOCAB, "bf16", 8),
        # one decode step of the 160M shape's batch of 64: entropies only
        _head("stats-160m-b64", "stats", 64, 768, VOCAB, "fp16"),
        # an evaluation batch of odd size on a head without its padding entries, a width that no vector load divides
        _head("stats-odd", "stats", 1003, 1037, 50277, "fp16", 5),
        # the fp32 check mode's shape: the responses of a few sequences
        _head("stats-70m-fp32", "stats", 565, 512, VOCAB, "fp32", 4),
        # every response token of the headline rollout batch (256 of 53)
        _head("stats-2.8b-b256", "stats", 13568, 2560, VOCAB, "bf16", 8),
        # the smallest training batch, fp32
        _head("grad-70m-fp32", "grad", 106, 512, VOCAB, "fp32"),
        # the 160M shape's update batch, one token short: a loss-scaled fp16 head
        _head("grad-160m-b64", "grad", 3391, 768, VOCAB, "fp16"),
        # the headline batch
        _head("grad-2.8b-b256", "grad", 13568, 2560, VOCAB, "bf16"),
        # one matrix of odd sizes, on its own
        _orth("orth-odd", 1, 1025, 333, "fp32"),
        # the out-projections of the 1B shape's sixteen layers
        _orth("orth-1b", 16, 2048, 2048, "bf16"),
        # one optimizer step of the 70M shape's matrices (24 of them)
        _muon("muon-70m", 6, 512),
        # one optimizer step of two layers at the 2.8B width
        _muon("muon-2.8b", 2, 2560),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["stats", "stats", "grad", "orth", "muon"])
    if kind == "muon":
        return dict(kind=kind, layers=rng.randint(1, 4), d=_log_int(rng, 64, 1536))
    if kind == "orth":
        return dict(kind=kind, batch=rng.randint(1, 6), rows=_log_int(rng, 64, 2560), cols=_log_int(rng, 64, 2560),
                    dtype=rng.choice(["fp32", "bf16"]))
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
    t = _log_int(rng, 1, 1024 if dtype == "fp32" else 4096)
    d = _log_int(rng, 64, 4096)
    if rng.random() < 0.5:
        d = max(64, d // 64 * 64)  # widths of real models divide well
    return dict(kind=kind, t=t, d=d, v=rng.choice([VOCAB, _log_int(rng, 1000, 65536)]), dtype=dtype,
                top=rng.choice([0, rng.randint(1, 20)]) if kind == "stats" else 0)


# ------------------------------------------------------------------------------------------------ inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _on_grid(x, steps_per_one, most):
    return (x * steps_per_one).round().clamp_(-most, most) / steps_per_one


def _head_inputs(case, seed):
    """Rows like a final LayerNorm's, which lean towards the output row of a token by an amount of their own, so that some
    distributions are flat and some have nearly everything in one token; an output matrix N(0, 0.02).  All values lie on a
    grid that every type holds, coarse enough that the logits have one value in 32 bits whatever the order of the sums:
    the alternatives' ids are whole numbers, and equal logits, of which there are many, go to the lower one.  One target in
    ten is absent."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    t, d, v, dt = case["t"], case["d"], case["v"], TYPES[case["dtype"]]
    fine = 4 if case["dtype"] == "fp32" else 1
    weight = _on_grid(0.02 * _randn(gen, v, d), 1024 * fine, 127 * fine)
    lean = torch.randint(0, v, (t,), generator=gen, device=DEVICE)
    much = 19.0 * torch.rand((t, 1), generator=gen, device=DEVICE) / (4e-4 * d)
    hidden = _on_grid(_randn(gen, t, d) + much * weight[lean], 16 * fine, 127 * fine)
    targets = torch.where(torch.rand(t, generator=gen, device=DEVICE) < 0.7, lean,
                          torch.randint(0, v, (t,), generator=gen, device=DEVICE))
    targets = torch.where(torch.rand(t, generator=gen, device=DEVICE) < 0.1, -1, targets).int()
    s = dict(case=case, hidden=hidden.to(dt), weight=weight.to(dt), targets=targets)
    if case["kind"] == "grad":
        z = (hidden @ weight.T) / TEMPERATURE  # what the forward call has left
        s["lse"] = torch.logsumexp(z, 1)
        s["entropy"] = s["lse"] - (torch.softmax(z, 1) * z).sum(1)
        # advantages over the tokens and an entropy bonus of 0.05; a fp16 head's loss is scaled as the update scales it
        scale = 64.0 if case["dtype"] == "fp16" else 1.0 / t
        s["d_logprobs"] = torch.where(targets >= 0, scale * _randn(gen, t), 0.0)
        s["d_entropy"] = torch.full((t,), -0.05 * scale, device=DEVICE)
    return s


def _gradients(gen, batch, rows, cols):
    """A gradient's spectrum: few strong directions over a floor of weak ones."""
    rank = min(rows, cols) // 8 + 1
    g = torch.bmm(_randn(gen, batch, rows, rank), _randn(gen, batch, rank, cols)) / math.sqrt(rank)
    return 1e-4 * (g + 0.1 * _randn(gen, batch, rows, cols))


def _muon_shapes(case):
    """Stacks [layers, rows, cols]: QKV, out-projection and the two of the MLP."""
    n, d = case["layers"], case["d"]
    return [(n, 3 * d, d), (n, d, d), (n, 4 * d, d), (n, d, 4 * d)]


def prepare(case, seed):
    if case["kind"] in ("stats", "grad"):
        return _head_inputs(case, seed)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    if case["kind"] == "orth":
        return dict(case=case, x=_gradients(gen, case["batch"], case["rows"], case["cols"]).to(TYPES[case["dtype"]]))
    # the optimizer's arrays are views of one buffer each (what a trainer that reduces or saves them whole keeps)
    shapes = _muon_shapes(case)
    total = sum(math.prod(x) for x in shapes)
    flat = {k: torch.empty(total, device=DEVICE) for k in ("param", "grad", "moment")}
    flat["bf16"] = torch.empty(total, dtype=torch.bfloat16, device=DEVICE)
    stacks = {k: [] for k in flat}
    at = 0
    for shape in shapes:
        for k in flat:
            stacks[k].append(flat[k][at:at + math.prod(shape)].view(shape))
        at += math.prod(shape)
        stacks["param"][-1].copy_(0.02 * _randn(gen, *shape))
        stacks["grad"][-1].copy_(_gradients(gen, *shape))
        stacks["moment"][-1].copy_(0.5 * _gradients(gen, *shape))
        stacks["bf16"][-1].copy_(stacks["param"][-1])
    lists = {k: [m for stack in v for m in stack] for k, v in stacks.items()}
    return dict(case=case, flat=flat, stacks=stacks, lists=lists)


# ------------------------------------------------------------------------------------------------ the operators, plain
def _plain_stats(s):
    case = s["case"]
    logits = s["hidden"].float() @ s["weight"].float().T
    z = logits / TEMPERATURE
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    entropy = torch.log(total) - (e * (z - top)).sum(1) / total
    at = s["targets"].long()
    picked = torch.gather(z, 1, at.clamp(min=0)[:, None])[:, 0] - lse
    out = dict(logprobs=torch.where(at >= 0, picked, 0.0), entropy=entropy, lse=lse)
    if case["top"]:
        # one whole number per entry that orders by logit, then by lower id
        bits = (logits + 0.0).view(torch.int32)
        bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
        ids = torch.arange(case["v"], device=DEVICE)
        key = bits.long() * (1 << 32) + (case["v"] - 1 - ids)
        best = torch.topk(key, case["top"], dim=1).values
        out["top_ids"] = (case["v"] - 1 - (best & 0xFFFFFFFF)).int()
        out["top_logprobs"] = torch.gather(z, 1, out["top_ids"].long()) - lse[:, None]
    return out


def _plain_grad(s):
    hidden, weight = s["hidden"].float(), s["weight"].float()
    logp = (hidden @ weight.T) / TEMPERATURE - s["lse"][:, None]
    p = torch.exp(logp)
    at = s["targets"].long()
    g = torch.where(at >= 0, s["d_logprobs"], 0.0)
    dz = -p * (g[:, None] + s["d_entropy"][:, None] * (logp + s["entropy"][:, None]))
    dz.scatter_add_(1, at.clamp(min=0)[:, None], g[:, None])
    dz /= TEMPERATURE
    return dict(d_hidden=(dz @ weight).to(s["hidden"].dtype), d_weight=(dz.T @ hidden).to(s["weight"].dtype))


def _newton_schulz(x):
    """[batch, rows, cols] in the type of the arithmetic."""
    a, b, c = COEFFS
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.mT.contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + EPS)
    for _ in range(STEPS):
        g = torch.bmm(x, x.mT.contiguous())
        x = a * x + torch.bmm(b * g + c * torch.bmm(g, g), x)
    return x.mT if tall else x


def _plain_muon(s):
    for p, g, m, b in zip(*(s["stacks"][k] for k in ("param", "grad", "moment", "bf16"))):
        m.mul_(MOMENTUM).add_((1.0 - MOMENTUM) * g)
        update = _newton_schulz((1.0 - MOMENTUM) * g + MOMENTUM * m)
        p.mul_(1.0 - LR * DECAY).sub_(LR * RMS * math.sqrt(max(p.shape[1:])) * update)
        b.copy_(p)
    return {k: s["flat"][k] for k in ("param", "moment", "bf16")}


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2403_17031_amd import muon_step, orthogonalize, token_stats, token_stats_backward
        if kind == "stats":
            return token_stats(s["hidden"], s["weight"], s["targets"], TEMPERATURE, top_k=s["case"]["top"])
        if kind == "grad":
            return token_stats_backward(s["hidden"], s["weight"], s["targets"], s["lse"], s["entropy"], s["d_logprobs"],
                                        s["d_entropy"], TEMPERATURE)
        if kind == "orth":
            return orthogonalize(s["x"], ns_steps=STEPS, eps=EPS)
        x = s["lists"]
        muon_step(x["param"], x["grad"], x["moment"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, rms=RMS, ns_steps=STEPS,
                  eps=EPS, params_bf16=x["bf16"])
        return {k: s["flat"][k] for k in ("param", "moment", "bf16")}
    if kind == "stats":
        return _plain_stats(s)
    if kind == "grad":
        return _plain_grad(s)
    if kind == "orth":
        return _newton_schulz(s["x"].float()).bfloat16()
    return _plain_muon(s)


# ------------------------------------------------------------------------------------------------ work, 64-bit results
def _ns_flops(rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    return STEPS * (3.0 * m * m * n + 1.0 * m * m * m)  # of the two symmetric products one half each


def work(case):
    kind = case["kind"]
    if kind in ("stats", "grad"):
        t, d, v = case["t"], case["d"], case["v"]
        operands = (t + v) * d * (4.0 if case["dtype"] == "fp32" else 2.0)
        if kind == "stats":
            return {"bytes": operands + t * (16.0 + 8.0 * case["top"]), "flops": 2.0 * t * d * v}
        return {"bytes": 2 * operands + 20.0 * t, "flops": 6.0 * t * d * v}
    if kind == "orth":
        b, m, n = case["batch"], case["rows"], case["cols"]
        return {"bytes": b * m * n * ((4.0 if case["dtype"] == "fp32" else 2.0) + 2.0), "flops": b * _ns_flops(m, n)}
    shapes = _muon_shapes(case)
    return {"bytes": 22.0 * sum(math.prod(x) for x in shapes), "flops": sum(x[0] * _ns_flops(*x[1:]) for x in shapes)}


def _exact_head(s):
    h, w = s["hidden"].double(), s["weight"].double()
    z = torch.mm(h, w.t()).div_(TEMPERATURE)
    has = s["targets"] >= 0
    pick = s["targets"].long().clamp(min=0)
    if s["case"]["kind"] == "grad":
        z.sub_(s["lse"].double()[:, None])
        prob = z.exp()
        gl = s["d_logprobs"].double() * has
        z.add_(s["entropy"].double()[:, None]).mul_(s["d_entropy"].double()[:, None]).add_(gl[:, None]).mul_(prob).neg_()
        z[torch.arange(z.shape[0], device=DEVICE), pick] += gl
        z.div_(TEMPERATURE)
        return dict(d_hidden=torch.mm(z, w), d_weight=torch.mm(z.t(), h))
    lse = torch.logsumexp(z, 1)
    at = z[torch.arange(z.shape[0], device=DEVICE), pick]
    out = dict(logprobs=(at - lse) * has, lse=lse)
    logp = z - lse[:, None]
    out["entropy"] = -(logp.exp() * logp).sum(1)
    if s["case"]["top"]:
        out["top_ids"] = None
        out["top_logprobs"] = torch.topk(logp, s["case"]["top"], dim=1).values
    return out


def _exact_orth(x):
    """One matrix, products on whichever side is the smaller."""
    a, b, c = COEFFS
    y = x / (torch.linalg.matrix_norm(x) + EPS)
    if y.shape[0] > y.shape[1]:
        for _ in range(STEPS):
            g = y.t() @ y
            y = a * y + b * (y @ g) + c * ((y @ g) @ g)
    else:
        for _ in range(STEPS):
            g = y @ y.t()
            y = a * y + b * (g @ y) + c * (g @ (g @ y))
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("stats", "grad"):
        return _exact_head(s)
    if case["kind"] == "orth":
        return torch.stack([_exact_orth(x) for x in s["x"].double()])
    out = {k: [] for k in ("param", "moment", "bf16")}
    for p, g, m in zip(s["lists"]["param"], s["lists"]["grad"], s["lists"]["moment"]):
        m1 = MOMENTUM * m.double() + (1 - MOMENTUM) * g.double()
        o = _exact_orth((1 - MOMENTUM) * g.double() + MOMENTUM * m1)
        p1 = p.double() * (1 - LR * DECAY) - LR * RMS * max(p.shape) ** 0.5 * o
        out["param"].append(p1.reshape(-1))
        out["moment"].append(m1.reshape(-1))
        out["bf16"].append(p1.reshape(-1))
    return {k: torch.cat(v) for k, v in out.items()}
