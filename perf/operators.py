"""The operators of wide policies as they are measured: an int8 dense layer whose activations are quantised with a scale for each
token, the log-probabilities of the actions taken, and the clipped policy loss with its KL term and its gradient.

`run` computes them in elementary torch operations, or with `own` set makes the calls a user makes of the package.  `exact` is the
definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token through a square layer: the latency of a single decision
        dict(name="dense one token", op="dense", m=1, k=4096, n=4096, x="bf16", out="bf16", bias=True, relu=False),
        # a handful of environments stepping together, behaviour logits over a wide action set
        dict(name="dense few tokens", op="dense", m=24, k=2048, n=8192, x="bf16", out="f32", bias=False, relu=False),
        # the flat convolution output of the paper's network into its dense layer, a ragged batch of fp32 activations
        dict(name="dense flat image", op="dense", m=301, k=3136, n=512, x="f32", out="f32", bias=True, relu=True),
        # odd sizes all over: no extent is a multiple of a tile
        dict(name="dense odd", op="dense", m=999, k=1777, n=2501, x="f16", out="f16", bias=True, relu=False),
        # a learner's batch through a wide layer
        dict(name="dense batch", op="dense", m=8192, k=4096, n=16384, x="bf16", out="bf16", bias=True, relu=False),
        # one step of a few environments, 18 actions: the smallest call of the loss
        dict(name="loss one step", op="loss", b=32, a=18, dtype="f32", kl="forward", mask="none", pad=0.0, ld=0),
        # a whole unroll's states with 18 actions, of which each state allows some; KL to the original policy
        dict(name="loss unroll", op="loss", b=262144, a=18, dtype="f32", kl="forward", mask="rows", pad=0.1, ld=0),
        # token actions: packed rows of different lengths' padding, the reference's log-probability of the sampled token only
        dict(name="loss sampled KL", op="loss", b=8192, a=32000, dtype="bf16", kl="sampled", mask="none", pad=0.2, ld=0),
        # odd width, rows with a stride of their own, the KL of whole distributions the other way round
        dict(name="loss odd rows", op="loss", b=777, a=50001, dtype="f16", kl="reverse", mask="shared", pad=0.05, ld=7),
        # the widest action set with the distillation-like KL of both whole distributions
        dict(name="loss widest", op="loss", b=2048, a=150000, dtype="bf16", kl="forward", mask="none", pad=0.0, ld=0),
        # the behaviour's log-probabilities of one decoding step of a few environments
        dict(name="logprob one step", op="logprob", b=16, a=100000, dtype="bf16", mask="none", ld=0),
        # the same over a learner's batch, fp32 logits
        dict(name="logprob batch", op="logprob", b=4096, a=32768, dtype="f32", mask="none", ld=0),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["dense", "dense", "loss", "loss", "logprob"])
    if op == "dense":
        while True:
            m, k, n = _log_uniform(rng, 1, 8192), _log_uniform(rng, 64, 8192), _log_uniform(rng, 64, 32768)
            if m * k * n <= 1 << 37:
                break
        return dict(op=op, m=m, k=k, n=n, x=rng.choice(["bf16", "bf16", "f16", "f32"]), out=rng.choice(["bf16", "f16", "f32"]),
                    bias=rng.random() < 0.5, relu=rng.random() < 0.3)
    while True:
        b, a = _log_uniform(rng, 1, 262144), _log_uniform(rng, 2, 160000)
        if b * a <= 1 << 27:
            break
    case = dict(op=op, b=b, a=a, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), mask=rng.choice(["none", "none", "shared", "rows"]),
                ld=rng.choice([0, 0, rng.randint(1, 64)]))
    if op == "loss":
        case.update(kl=rng.choice(["none", "sampled", "forward", "reverse"]), pad=rng.choice([0.0, 0.1, 0.3]))
    return case


def work(case):
    if case["op"] == "dense":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": m * k * BYTES[case["x"]] + n * k + 4 * n * (2 if case["bias"] else 1) + m * n * BYTES[case["out"]], "flops": 2 * m * k * n}
    b, a, e = case["b"], case["a"], BYTES[case["dtype"]]
    masked = {"none": 0, "shared": a, "rows": b * a}[case["mask"]]
    if case["op"] == "logprob":
        return {"bytes": b * a * e + masked + 12 * b, "flops": 5 * b * a}
    live = b - int(b * case["pad"])                     # rows that are padding are written, not read
    tables = 2 if case["kl"] in ("forward", "reverse") else 1
    masked = live * a if case["mask"] == "rows" else masked
    return {"bytes": live * a * e * tables + b * a * e + masked + (36 if case["kl"] == "sampled" else 32) * b, "flops": (12 * tables) * live * a}


def _table(g, b, a, ld, dtype, scale):
    """[b, a] logits whose rows lie a + ld apart."""
    t = torch.empty((b, a + ld), dtype=DTYPES[dtype], device="cuda")
    rows = max(1, (1 << 28) // (a + ld))
    for i in range(0, b, rows):
        n = min(rows, b - i)
        t[i:i + n] = torch.randn((n, a + ld), generator=g, device="cuda") * scale
    return t[:, :a]


def _mask(g, kind, b, a):
    if kind == "none":
        return None
    m = (torch.rand((1 if kind == "shared" else b, a), generator=g, device="cuda") < 0.7).to(torch.uint8)
    if kind == "rows":
        m[torch.rand(b, generator=g, device="cuda") < 0.01] = 0       # states without an allowed action
    else:
        m[0, torch.randint(0, a, (1,), generator=g, device="cuda")] = 1
    return m


def _sample(g, logits, mask):
    """Actions as an actor draws them, among the allowed ones: the largest of logit + Gumbel noise."""
    b, a = logits.shape
    out = torch.empty(b, dtype=torch.int32, device="cuda")
    rows = max(1, (1 << 27) // a)
    for i in range(0, b, rows):
        z = logits[i:i + rows].float()
        z = z - torch.log(-torch.log(torch.rand(z.shape, generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)))
        if mask is not None:
            z = z.masked_fill((mask if mask.shape[0] == 1 else mask[i:i + rows]) == 0, -math.inf)
        out[i:i + rows] = z.argmax(dim=1).to(torch.int32)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = dict(case=case)
    if case["op"] == "dense":
        m, k, n = case["m"], case["k"], case["n"]
        # activations with a few large channels, weights of different magnitude for each output
        x = torch.randn((m, k), generator=g, device="cuda") * (1 + 15 * (torch.rand(k, generator=g, device="cuda") < 0.01))
        w = torch.randn((n, k), generator=g, device="cuda") * (0.5 + torch.rand((n, 1), generator=g, device="cuda")) / math.sqrt(k)
        w_scale = w.abs().amax(dim=1) / 127
        state.update(x=x.to(DTYPES[case["x"]]), w_scale=w_scale, wq=torch.round(w / w_scale[:, None]).clamp(-127, 127).to(torch.int8),
                     bias=torch.randn(n, generator=g, device="cuda") if case["bias"] else None)
        if own:
            import paper_2211_15023_amd as A
            state["layer"] = A.DenseInt8(state["wq"], w_scale, state["bias"], relu=case["relu"])
        return state
    b, a = case["b"], case["a"]
    state["logits"] = _table(g, b, a, case["ld"], case["dtype"], 2.0)
    state["mask"] = _mask(g, case["mask"], b, a)
    state["actions"] = _sample(g, state["logits"], state["mask"])
    if case["op"] == "logprob":
        if own:
            import paper_2211_15023_amd as A
            state["loss"] = A.PolicyLoss()
        return state
    lp = _logprob(state["logits"], state["mask"], state["actions"])[0].float()
    lp = torch.where(torch.isfinite(lp), lp, torch.zeros_like(lp))
    # the behaviour's policy lags behind: ratios on both sides of the clipping borders
    state["old_logp"] = lp + 0.2 * torch.randn(b, generator=g, device="cuda")
    state["advantages"] = torch.randn(b, generator=g, device="cuda")
    live = torch.ones(b, device="cuda")
    live[torch.randperm(b, generator=g, device="cuda")[:int(b * case["pad"])]] = 0
    state["weights"] = live
    state["scale"] = 1.0 / max(1, b - int(b * case["pad"]))
    if case["kl"] == "sampled":
        state["ref_logp"] = lp + 0.3 * torch.randn(b, generator=g, device="cuda")
    elif case["kl"] != "none":
        ref = _table(g, b, a, case["ld"], case["dtype"], 0.5)
        rows = max(1, (1 << 28) // a)
        for i in range(0, b, rows):
            ref[i:i + rows] += state["logits"][i:i + rows]
        state["ref"] = ref
    if own:
        import paper_2211_15023_amd as A
        state["loss"] = A.PolicyLoss(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl=case["kl"], kl_coef=KL_COEF, entropy_coef=ENTROPY_COEF)
    return state


CLIP_LOW, CLIP_HIGH, KL_COEF, ENTROPY_COEF = 0.2, 0.25, 0.05, 0.01


def run(state):
    case = state["case"]
    if case["op"] == "dense":
        if own:
            return state["layer"].forward(state["x"], dtype=DTYPES[case["out"]])
        return _dense(state)
    if case["op"] == "logprob":
        if own:
            return state["loss"].logprob(state["logits"], state["actions"], mask=state["mask"])
        lp, ent = _logprob(state["logits"], state["mask"], state["actions"])
        return lp.float(), ent.float()
    if own:
        r = state["loss"].forward(state["logits"], state["actions"], state["old_logp"], state["advantages"], mask=state["mask"],
                                  weights=state["weights"], scale=state["scale"], ref_logits=state.get("ref"), ref_logp=state.get("ref_logp"))
        return dict(loss=r.loss, logp=r.logp, kl=r.kl, entropy=r.entropy, stats=r.stats, grad=r.grad)
    return _loss(state)


# ------------------------------------------------------------------ the plain forms
def _dense(state):
    x = state["x"].float()
    amax = x.abs().amax(dim=1, keepdim=True)
    # in 64 bits: what lies next to the middle of two steps
    q = torch.where(amax > 0, torch.round(x.double() * 127 / amax.double()), 0.0).float()
    y = (q @ state["wq"].float().t()) * (amax / 127) * state["w_scale"]
    if state["bias"] is not None:
        y = y + state["bias"]
    if state["case"]["relu"]:
        y = y.clamp_min(0)
    return y.to(DTYPES[state["case"]["out"]])


def _allowed(logits, mask):
    z = logits.float()
    return z if mask is None else torch.where(mask != 0, z, -math.inf)


def _soft(z):
    """exp(z - max), its sum and log-sum-exp (in 64 bits: ratios next to a clipping border); an empty row gives zeros and -inf."""
    m = z.amax(dim=1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    s = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    return e, s, m.double() + torch.log(s)


def _dot(p, v):
    """sum_j p_j v_j over the places where p is not 0."""
    return torch.where(p > 0, p * v, 0.0).sum(dim=1, keepdim=True, dtype=torch.float64)


def _logprob(logits, mask, actions):
    z = _allowed(logits, mask)
    e, s, l = _soft(z)
    lp = z.gather(1, actions.long()[:, None]).double() - l
    lp = torch.where(s > 0, lp, -math.inf)
    ent = torch.where(s > 0, l - _dot(e, z) / s, 0.0)
    return lp[:, 0], ent[:, 0]


def _loss(state):
    case, mask, old, adv = state["case"], state["mask"], state["old_logp"].double()[:, None], state["advantages"].double()[:, None]
    z = _allowed(state["logits"], mask)
    a = state["actions"].long()[:, None]
    e, s, l = _soft(z)
    some = s > 0
    one = torch.where(some, s, 1.0)
    p = e * (1 / one).float()
    logp = torch.where(some, z - l.float(), -math.inf)
    lp = torch.where(some, z.gather(1, a).double() - l, -math.inf)
    ent = torch.where(some, l - _dot(e, z) / one, 0.0)
    ratio = torch.exp(lp - old)
    cut = ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    use = ratio * adv <= cut * adv
    loss = -torch.where(use, ratio * adv, cut * adv)
    at = torch.where(use, -ratio * adv, 0.0)                 # the derivative by log pi(a)
    grad = ENTROPY_COEF * torch.where(p > 0, p * (logp + ent.float()), 0.0)
    if case["kl"] == "sampled":
        d = state["ref_logp"].double()[:, None] - lp
        kl = torch.where(some, torch.exp(d) - d - 1, 0.0)
        at = at + KL_COEF * torch.where(some, 1 - torch.exp(d), 0.0)
    elif case["kl"] == "none":
        kl = torch.zeros_like(lp)
    else:
        zr = _allowed(state["ref"], mask)
        er, sr, lr = _soft(zr)
        pr = er * torch.where(sr > 0, 1 / sr, 0.0).float()
        apart = torch.where(some, z - zr, 0.0)
        if case["kl"] == "forward":
            kl = torch.where(some, l - lr - _dot(pr, apart), 0.0)
            grad = grad + KL_COEF * (p - pr)
        else:
            kl = torch.where(some, lr - l + _dot(p, apart), 0.0)
            grad = grad + KL_COEF * torch.where(p > 0, p * (apart - (l - lr + kl).float()), 0.0)
    grad = grad - at.float() * p
    grad.scatter_add_(1, a, at.float())
    w = state["weights"].double()[:, None]
    live = (w != 0) & some
    seen = (w != 0).double()
    loss = torch.where(live, loss + KL_COEF * kl - ENTROPY_COEF * ent, 0.0)
    kl, ent = torch.where(live, kl, 0.0), torch.where(live, ent, 0.0)
    lp = torch.where(seen > 0, lp, 0.0)
    wide = (live & ((ratio < 1 - CLIP_LOW) | (ratio > 1 + CLIP_HIGH))).double()
    grad = torch.where(live, grad * (w * state["scale"]).float(), 0.0)
    stats = (state["scale"] * torch.cat([(w * v).sum(dim=0) for v in (loss, kl, ent, wide)])).float()
    return dict(loss=loss[:, 0].float(), logp=lp[:, 0].float(), kl=kl[:, 0].float(), entropy=ent[:, 0].float(), stats=stats,
                grad=grad.to(DTYPES[case["dtype"]]))


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "dense":
        return _exact_dense(state)
    if case["op"] == "logprob":
        parts = [_exact_rows(state, i, j)[:2] for i, j in _blocks(case)]
        return tuple(torch.cat(t) for t in zip(*parts))
    parts = [_exact_loss(state, i, j) for i, j in _blocks(case)]
    out = {k: torch.cat([p[k] for p in parts]) for k in ("loss", "logp", "kl", "entropy", "grad")}
    out["stats"] = torch.stack([p["stats"] for p in parts]).sum(dim=0)
    return {k: out[k] for k in ("loss", "logp", "kl", "entropy", "stats", "grad")}


def _blocks(case):
    rows = max(1, (1 << 26) // case["a"])
    return [(i, min(case["b"], i + rows)) for i in range(0, case["b"], rows)]


def _exact_dense(state):
    x, w = state["x"].double(), state["wq"].double()
    top = x.abs().max(dim=1).values
    out = []
    for i in range(0, x.shape[0], 2048):
        d = top[i:i + 2048, None]
        # rounded once: x * 127 has no rounding here, so the middle of two steps is met exactly
        q = torch.div(x[i:i + 2048] * 127, torch.where(d > 0, d, 1.0)).round()
        y = torch.matmul(q, w.t()) * (d / 127) * state["w_scale"].double()[None, :]
        if state["bias"] is not None:
            y += state["bias"].double()
        out.append(torch.relu(y) if state["case"]["relu"] else y)
    return torch.cat(out)


def _exact_rows(state, i, j):
    """log pi(a), entropy, log pi and pi of rows i to j."""
    z = state["logits"][i:j].double()
    ok = torch.ones_like(z, dtype=torch.bool)
    if state["mask"] is not None:
        ok = (state["mask"] if state["mask"].shape[0] == 1 else state["mask"][i:j]).bool().expand_as(z)
        z = z.masked_fill(~ok, -math.inf)
    lg = z - torch.logsumexp(z, dim=1, keepdim=True)
    empty = ~ok.any(dim=1, keepdim=True)
    lg = lg.masked_fill(empty, -math.inf)
    pi = lg.exp()
    lp = lg[torch.arange(j - i, device=z.device), state["actions"][i:j].long()]
    return lp, -torch.special.xlogy(pi, pi).sum(dim=1), lg, pi, ok, empty[:, 0]


def _exact_loss(state, i, j):
    case, ids = state["case"], torch.arange(j - i, device="cuda")
    lp, ent, lg, pi, ok, empty = _exact_rows(state, i, j)
    act, old, adv = state["actions"][i:j].long(), state["old_logp"][i:j].double(), state["advantages"][i:j].double()
    w = state["weights"][i:j].double()
    rho = (lp - old).exp()
    inside = torch.where(adv >= 0, rho <= 1 + CLIP_HIGH, rho >= 1 - CLIP_LOW)
    pg = -torch.minimum(rho * adv, rho.clamp(min=1 - CLIP_LOW, max=1 + CLIP_HIGH) * adv)
    by_lp = -rho * adv * inside
    kl = torch.zeros_like(lp)
    grad = ENTROPY_COEF * (torch.special.xlogy(pi, pi) + pi * ent[:, None])
    if case["kl"] == "sampled":
        u = (state["ref_logp"][i:j].double() - lp).masked_fill(empty, 0.0)
        kl = torch.expm1(u) - u
        by_lp = by_lp - KL_COEF * torch.expm1(u)
    elif case["kl"] != "none":
        lr = torch.log_softmax(state["ref"][i:j].double().masked_fill(~ok, -math.inf), dim=1)
        diff = (lg - lr).masked_fill(~ok, 0.0)
        pr = lr.exp().masked_fill(~ok, 0.0)
        if case["kl"] == "forward":
            kl = -(pr * diff).sum(dim=1)
            grad += KL_COEF * (pi - pr)
        else:
            kl = (pi * diff).sum(dim=1)
            grad += KL_COEF * pi * (diff - kl[:, None])
    grad -= pi * by_lp[:, None]
    grad[ids, act] += by_lp
    dead = (w == 0) | empty
    loss = (pg + KL_COEF * kl - ENTROPY_COEF * ent).masked_fill(dead, 0.0)
    kl, ent = kl.masked_fill(dead, 0.0), ent.masked_fill(dead, 0.0)
    far = ((rho - 1 > CLIP_HIGH) | (1 - rho > CLIP_LOW)).double().masked_fill(dead, 0.0)
    grad = (grad * (w * state["scale"])[:, None]).masked_fill(dead[:, None], 0.0)
    stats = torch.stack([(w * v).sum() for v in (loss, kl, ent, far)]) * state["scale"]
    return dict(loss=loss, logp=lp.masked_fill(w == 0, 0.0), kl=kl, entropy=ent, grad=grad, stats=stats)
