"""The policy update that follows a likelihood pass and its rewards, as cases that can be timed and compared.

A trainer of a schedule policy holds logits over the actions, the actions taken, their advantages and, after its own network's
backward pass, gradients. It calls three operators: the clipped policy loss with a KL term and an entropy bonus, forward and
gradient in one call (`Sol.policy_loss`); the global norm of many gradients with clipping (`Sol.grad_clip`); the AdamW update
that takes the clip's coefficient on the device (`Sol.adamw_step`). `run` makes these calls, or computes the same in
elementary torch operations; `exact` gives the definitions in 64 bits.
"""
import math

import torch

own = False

CLIP = (0.2, 0.28)      # the ratio's bounds below and above 1
ADAM = dict(lr=1e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
CLIP_EPS = 1e-6         # added to the norm before the division
_CTX = []


def _ctx():
    """The program's library context (the operators take their sizes from their arguments, not from its model)."""
    if not _CTX:
        from paper_2605_10875_amd import sol, synth
        _CTX.append(sol.Sol(synth.TINY, synth.TABLE_C1, dtype=sol.F32, max_positions=16))
    return _CTX[0]


# ---- cases --------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one minibatch of the update: 512 steps under a table of 64 actions; latency and launches
        dict(name="loss_minibatch", op="loss", B=2, G=16, T=16, A=64, dtype="fp32", pad=0, kl="none", mean="steps",
             temperature=1.0, forbid=0, ragged=False),
        # all schedules of a batch of short episodes, ragged, 80 actions of which every eighth is not allowed, sampled at
        # the temperature of the rollouts, KL estimated from the reference's log-probability of the action
        dict(name="loss_rollout", op="loss", B=8, G=32, T=16, A=80, dtype="fp32", pad=0, kl="logp", mean="schedules",
             temperature=1.3, forbid=8, ragged=True),
        # the schedules of a whole likelihood pass, bf16 logits, exact KL against the reference's logits
        dict(name="loss_schedules", op="loss", B=2, G=8, T=2048, A=64, dtype="bf16", pad=0, kl="logits", mean="steps",
             temperature=1.3, forbid=0, ragged=False),
        # a fine table of 4001 actions in rows padded to 4096, odd length, exact KL
        dict(name="loss_fine_table", op="loss", B=4, G=8, T=509, A=4001, dtype="fp32", pad=95, kl="logits", mean="schedules",
             temperature=1.0, forbid=0, ragged=True),
        # the token policy of a language model: the vocabulary of the larger shapes as actions, KL estimate
        dict(name="loss_vocabulary", op="loss", B=1, G=8, T=333, A=128256, dtype="bf16", pad=0, kl="logp", mean="steps",
             temperature=1.0, forbid=0, ragged=False),
        # the gradients of a policy network (one layer of width 512 on the 8B shape's hidden states), clipped in place
        dict(name="clip_policy", op="clip", layout="policy", tensors=0, total=0, dtype="fp32"),
        # low-rank adapters of all linear maps of the 1B shape: many small tensors
        dict(name="clip_adapters", op="clip", layout="adapters", tensors=0, total=0, dtype="bf16"),
        # the gradients of a whole 1B model
        dict(name="clip_model", op="clip", layout="model", tensors=0, total=0, dtype="bf16"),
        # norm, coefficient and update of the policy network
        dict(name="update_policy", op="update", layout="policy", tensors=0, total=0, dtype="fp32", copy=False),
        # the same of the adapters, whose forward pass reads a bf16 copy
        dict(name="update_adapters", op="update", layout="adapters", tensors=0, total=0, dtype="bf16", copy=True),
        # four layers of the 1B shape with fp32 states, bf16 gradients and a bf16 copy
        dict(name="update_layers", op="update", layout="layers", tensors=0, total=0, dtype="bf16", copy=True),
    ]


def _size(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("loss", "loss", "loss", "clip", "update"))
    dtype = rng.choice(("fp32", "bf16"))
    if op == "loss":
        A = _size(rng, 2, 152064)
        rows = _size(rng, 1, max(1, min(40000, 160_000_000 // A)))
        T = _size(rng, 1, rows)
        G = _size(rng, 1, max(1, rows // T))
        return dict(op=op, B=max(1, rows // (T * G)), G=G, T=T, A=A, dtype=dtype, pad=rng.choice((0, 0, rng.randint(1, 64))),
                    kl=rng.choice(("none", "logp", "logits")), mean=rng.choice(("steps", "schedules")),
                    temperature=rng.choice((1.0, 1.3)), forbid=rng.choice((0, 0, 5)), ragged=rng.random() < 0.5)
    tensors = _size(rng, 1, 400)
    total = _size(rng, max(1000, 4 * tensors), 200_000_000)
    if op == "clip":
        return dict(op=op, layout="drawn", tensors=tensors, total=total, dtype=dtype)
    return dict(op=op, layout="drawn", tensors=tensors, total=total, dtype=dtype, copy=rng.random() < 0.5)


def _sizes(case):
    """Elements of the case's tensors."""
    d, kv, ff = 2048, 512, 8192                                  # the 1B shape
    maps = [(d, d), (kv, d), (kv, d), (d, d), (ff, d), (ff, d), (d, ff)]
    layer = [d, d] + [o * i for o, i in maps]
    if case["layout"] == "policy":                               # hidden state and embedding 4096, 8 features, 64 actions
        w = 512
        return [w * 4096, w, w * 4096, w, w * 8, w, 64 * 32, w * 32, w, w, w, w * w, w * w, w * w, w * w, w, 4 * w * w, 4 * w,
                4 * w * w, w, w, 64 * w, 64]
    if case["layout"] == "adapters":
        return [r for _ in range(16) for o, i in maps for r in (8 * i, 8 * o)]
    if case["layout"] == "layers":
        return layer * 4
    if case["layout"] == "model":
        return [128256 * d] + layer * 16 + [d]
    share = [((37 * k + 11) % 101 + 1) ** 2 for k in range(case["tensors"])]      # ragged: from one part in ten thousand up
    n = [max(1, case["total"] * x // sum(share)) for x in share]
    return n


# ---- inputs -------------------------------------------------------------------------------------------------------
def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _lengths(case):
    """Effective steps of each input: all, or a ragged batch whose inputs end between a third of T and T."""
    B, T = case["B"], case["T"]
    return [T if not case["ragged"] else T - (2 * T // 3) * ((5 * b + 3) % 8) // 8 for b in range(B)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 31)

    def rnd(*sz):
        return torch.randn(*sz, generator=gen, device="cuda")

    if case["op"] == "loss":
        return _prepare_loss(case, rnd, gen)
    sizes = _sizes(case)
    total = sum(sizes)
    s = {"case": case, "grad": rnd(total).mul_(0.02).to(_dt(case))}
    s["grads"] = list(torch.split(s["grad"], sizes))
    # a bound that clips: a third of the norm that such values have
    s["max_norm"] = 0.02 * math.sqrt(total) / 3
    if case["op"] == "update":
        s["param"] = rnd(total).mul_(0.02)
        s["m"] = rnd(total).mul_(0.005)
        s["v"] = rnd(total).mul_(0.01).square_().add_(1e-6)
        s["step"] = torch.full((1,), 100, dtype=torch.int32, device="cuda")
        s["copy"] = s["param"].to(torch.bfloat16) if case["copy"] else None
        for k in ("param", "m", "v", "copy"):
            s[k + "s"] = list(torch.split(s[k], sizes)) if s[k] is not None else None
    return s


def _prepare_loss(case, rnd, gen):
    B, G, T, A = case["B"], case["G"], case["T"], case["A"]
    buf = rnd(B, G, T, A + case["pad"]).mul_(2.0)
    if case["forbid"]:
        buf[..., case["forbid"] - 1:A:case["forbid"]] = -math.inf
    logits = buf.to(_dt(case))[..., :A]
    del buf
    t = case["temperature"]
    # actions drawn from the policy of the rollouts, a few updates ago
    ids = torch.empty((B, G, T), dtype=torch.int32, device="cuda")
    old = torch.empty((B, G, T), dtype=torch.float32, device="cuda")
    for b in range(B):
        for g in range(G):
            z = logits[b, g].float().div_(t)
            noise = torch.empty(z.shape, device="cuda").exponential_(generator=gen).log_().neg_()
            pick = (z + noise).argmax(-1)
            ids[b, g] = pick.int()
            old[b, g] = z.gather(-1, pick[:, None])[:, 0] - z.logsumexp(-1)
    s = {"case": case, "logits": logits, "ids": ids, "adv": rnd(B, G, T), "old": old + 0.15 * rnd(B, G, T), "ref_logp": None,
         "ref_logits": None, "eff": None}
    if case["kl"] == "logp":
        s["ref_logp"] = old + 0.1 * rnd(B, G, T)
    if case["kl"] == "logits":
        ref = torch.empty((B, G, T, A + case["pad"]), dtype=_dt(case), device="cuda")
        for b in range(B):
            ref[b, ..., :A] = logits[b].float() + 0.1 * rnd(G, T, A)
        s["ref_logits"] = ref[..., :A]
    if case["ragged"]:
        n = torch.tensor(_lengths(case), device="cuda")
        s["eff"] = (torch.arange(T, device="cuda")[None, :] < n[:, None]).int()
    return s


# ---- the operators ------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if case["op"] == "loss":
        if not own:
            return _loss(state)
        return _ctx().policy_loss(state["logits"], state["ids"], state["adv"], old_logp=state["old"], ref_logp=state["ref_logp"],
                                  ref_logits=state["ref_logits"], eff=state["eff"], clip=CLIP, kl_coef=_kl_coef(case),
                                  entropy_coef=0.05, temperature=case["temperature"], scale=0.125, mean=case["mean"])
    if case["op"] == "clip":
        if own:
            norm, coef = _ctx().grad_clip(state["grads"], state["max_norm"], eps=CLIP_EPS)
        else:
            norm, coef = _norm(state)
            state["grad"].copy_(state["grad"].float() * coef)
        return {"norm": norm, "coef": coef, "grad": state["grad"]}
    if own:
        norm, coef = _ctx().grad_clip(state["grads"], state["max_norm"], eps=CLIP_EPS, scale=False)
        _ctx().adamw_step(state["params"], state["grads"], state["ms"], state["vs"], state["step"], coef=coef, copies=state["copys"],
                          **ADAM)
    else:
        norm, coef = _norm(state)
        _adamw(state, coef)
    out = {"norm": norm, "param": state["param"], "m": state["m"], "v": state["v"]}
    if case["copy"]:
        out["copy"] = state["copy"]
    return out


def _kl_coef(case):
    return 0.0 if case["kl"] == "none" else 0.04


def _weights(case, eff):
    """Every step's share in the mean, [B][1][T] in 64 bits."""
    e = torch.ones((case["B"], case["T"]), device="cuda", dtype=torch.float64) if eff is None else (eff != 0).double()
    if case["mean"] == "steps":
        w = e / (e.sum() * case["G"]).clamp(min=1)
    else:
        n = e.sum(1, keepdim=True)
        w = e / n.clamp(min=1) / ((n > 0).sum() * case["G"]).clamp(min=1)
    return w[:, None, :]


def _loss(s):
    """Rows in 32 bits, the numbers of one step (log-probability, ratio, its bounds) in 64."""
    case, t = s["case"], s["case"]["temperature"]
    w = _weights(case, s["eff"])
    live = w > 0
    z = s["logits"].float() / t
    top = z.amax(-1, keepdim=True)
    z = z - top
    p = z.exp()
    total = p.sum(-1, keepdim=True, dtype=torch.float64)
    p = p / total.float()
    lp = z - total.log().float()                                  # log-probabilities
    ids = s["ids"].long()[..., None]
    logp = (s["logits"].gather(-1, ids).double() / t - top.double() - total.log())[..., 0]
    plain = torch.where(p > 0, lp, 0.0)                           # 0 log 0 = 0
    entropy = -(p * plain).sum(-1, dtype=torch.float64)
    ratio = (logp - s["old"].double()).exp()
    adv = s["adv"].double()
    free, held = ratio * adv, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv
    clipped = held < free
    pg = -torch.minimum(free, held)
    by_logp = torch.where(clipped, 0.0, -free)                    # the loss by the action's log-probability
    beta, bonus = _kl_coef(case), 0.05
    kl = torch.zeros_like(pg)
    grad = p * (plain + entropy.float()[..., None]) * bonus
    if case["kl"] == "logp":
        u = s["ref_logp"].double() - logp
        kl = u.exp() - u - 1
        by_logp = by_logp + beta * (1 - u.exp())
    if case["kl"] == "logits":
        y = s["ref_logits"].float() / t
        y = y - y.amax(-1, keepdim=True)
        far = torch.where(p > 0, lp - (y - y.exp().sum(-1, keepdim=True, dtype=torch.float64).log().float()), 0.0)
        kl = (p * far).sum(-1, dtype=torch.float64)
        grad = grad + p * (far - kl.float()[..., None]) * beta
    grad = grad - p * by_logp.float()[..., None]
    grad.scatter_add_(-1, ids, by_logp.float()[..., None])
    grad = grad * (w * (0.125 / t)).float()[..., None]
    grad = torch.where(live[..., None], grad, 0.0).to(s["logits"].dtype)

    def mean(x):
        return torch.where(live, x * w, 0.0).sum()

    parts = [mean(pg), mean(kl), mean(entropy), mean(clipped.double())]
    loss = 0.125 * (parts[0] + beta * parts[1] - bonus * parts[2])
    return {"loss": loss.float().reshape(1), "stats": torch.stack(parts).float(), "logp": torch.where(live, logp, 0.0).float(), "grad": grad}


def _norm(s):
    norm = s["grad"].float().square().sum(dtype=torch.float64).sqrt()
    coef = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    return norm.float().reshape(1), coef.float().reshape(1)


def _adamw(s, coef):
    b1, b2 = ADAM["betas"]
    step = s["step"].double()
    g = s["grad"].float() * coef
    s["m"].copy_(b1 * s["m"] + (1 - b1) * g)
    s["v"].copy_(b2 * s["v"] + (1 - b2) * g * g)
    denom = (s["v"] / (1 - b2 ** step).float()).sqrt() + ADAM["eps"]
    s["param"].copy_(s["param"] * (1 - ADAM["lr"] * ADAM["weight_decay"]) - (ADAM["lr"] / (1 - b1 ** step)).float() * s["m"] / denom)
    if s["copy"] is not None:
        s["copy"].copy_(s["param"])


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "loss":
        rows, A = case["B"] * case["G"] * case["T"], case["A"]
        live = case["G"] * sum(_lengths(case))
        reads = live * (A * size * (2 if case["kl"] == "logits" else 1) + 12 + (4 if case["kl"] == "logp" else 0))
        return {"bytes": reads + rows * (A * size + 4) + (4 * case["B"] * case["T"] if case["ragged"] else 0),
                "flops": live * A * (20 if case["kl"] == "logits" else 12)}
    n = sum(_sizes(case))
    if case["op"] == "clip":
        return {"bytes": 2 * n * size + 8, "flops": 3 * n}
    return {"bytes": n * (size + 24 + (2 if case["copy"] else 0)) + 8, "flops": 16 * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "loss":
        return _exact_loss(s)
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g)
    coef = min(1.0, s["max_norm"] / (float(norm) + CLIP_EPS))
    if case["op"] == "clip":
        return {"norm": norm.reshape(1), "coef": torch.tensor([coef], dtype=torch.float64), "grad": g * coef}
    (b1, b2), t = ADAM["betas"], int(s["step"])
    g *= coef
    m = torch.lerp(g, s["m"].double(), b1)
    v = torch.lerp(g * g, s["v"].double(), b2)
    p = s["param"].double()
    p -= ADAM["lr"] * (ADAM["weight_decay"] * p + m / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + ADAM["eps"]))
    return {"norm": norm.reshape(1), "param": p, "m": m, "v": v, **({"copy": p} if case["copy"] else {})}


def _exact_loss(s):
    """The loss as written, its gradient by differentiation."""
    case = s["case"]
    B, G, T = case["B"], case["G"], case["T"]
    x = s["logits"].double().requires_grad_(True)
    with torch.enable_grad():
        lp = torch.log_softmax(x / case["temperature"], -1)
        logp = lp.gather(-1, s["ids"].long()[..., None]).squeeze(-1)
        finite = lp.masked_fill(lp == -math.inf, 0.0)
        entropy = -(lp.exp() * finite).sum(-1)
        ratio = torch.exp(logp - s["old"].double())
        a = s["adv"].double()
        pg = -torch.min(ratio * a, torch.clamp(ratio, 1 - CLIP[0], 1 + CLIP[1]) * a)
        kl = torch.zeros_like(pg)
        if case["kl"] == "logp":
            u = s["ref_logp"].double() - logp
            kl = torch.expm1(u) - u
        elif case["kl"] == "logits":
            lq = torch.log_softmax(s["ref_logits"].double() / case["temperature"], -1)
            kl = (lp.exp() * (finite - lq.masked_fill(lq == -math.inf, 0.0))).sum(-1)
        # the mean, counted input by input
        n = _lengths(case)
        weight = torch.zeros((B, 1, T), dtype=torch.float64, device="cuda")
        for b in range(B):
            weight[b, 0, :n[b]] = 1.0 / (G * sum(n)) if case["mean"] == "steps" else 1.0 / (G * B * n[b])
        parts = [(weight * v).sum() for v in (pg, kl, entropy)]
        loss = 0.125 * (parts[0] + _kl_coef(case) * parts[1] - 0.05 * parts[2])
        grad = torch.autograd.grad(loss, x)[0]
    with torch.no_grad():
        clipped = torch.where(a > 0, ratio > 1 + CLIP[1], ratio < 1 - CLIP[0]) & (a != 0)
        stats = torch.stack([*parts, (weight * clipped.double()).sum()])
        return {"loss": loss.reshape(1), "stats": stats, "logp": logp * (weight > 0), "grad": grad}
