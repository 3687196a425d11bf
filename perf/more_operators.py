"""The operators of policies with a memory as they are measured: linear attention with a decay for each head (an unroll, its gradients, the
step of single tokens) and the norms around a block, fused with its gate and its residual (values and gradients).

`run` computes them in elementary torch operations, or with `own` set makes the calls a user makes of the package.  `exact` is the
definition in 64 bits.

Linear attention, for a head of decay g:  S_t = g S_{t-1} + k_t v_t^T  (S_{t-1} = 0 where the token begins an episode),  o_t = scale q_t S_t.
Norms:  u = skip x + branch act(gate) after(y),  h = before(u),  after and before being norms with a weight for each channel.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
SKIP, BRANCH = 1.0, 0.5


def listed():
    return [
        # one environment's next token: the latency of a single decision
        dict(name="step one environment", op="step", b=1, h=8, hk=8, dk=64, dv=64, dtype="bf16", resets=0.0),
        # all environments of a large actor at once, some of them beginning an episode
        dict(name="step many environments", op="step", b=512, h=16, hk=16, dk=128, dv=128, dtype="bf16", resets=0.02),
        # a learner's short unrolls of 20 steps, fp32
        dict(name="unroll short", op="unroll", b=32, t=20, h=8, hk=8, dk=64, dv=64, dtype="f32", resets=0.02, ragged=False, state=True),
        # a learner's batch of unrolls with episode borders, from the actors' states on
        dict(name="unroll batch", op="unroll", b=64, t=512, h=16, hk=16, dk=128, dv=128, dtype="bf16", resets=0.005, ragged=False, state=True),
        # one long history read in
        dict(name="unroll long", op="unroll", b=1, t=65536, h=16, hk=16, dk=128, dv=128, dtype="bf16", resets=0.0, ragged=False, state=False),
        # odd sizes, heads that share keys and values, histories of different lengths
        dict(name="unroll odd", op="unroll", b=3, t=1777, h=6, hk=2, dk=80, dv=100, dtype="f16", resets=0.003, ragged=True, state=False),
        # the learner's step through the batch
        dict(name="gradient batch", op="gradient", b=32, t=512, h=16, hk=16, dk=128, dv=128, dtype="bf16", resets=0.005, ragged=False, state=True),
        # the same for odd sizes and shared keys, fp32
        dict(name="gradient odd", op="gradient", b=5, t=333, h=4, hk=2, dk=48, dv=72, dtype="f32", resets=0.01, ragged=True, state=True),
        # the tokens of one actor step through a block's end and the next one's beginning
        dict(name="norm few rows", op="norm", n=16, d=1024, groups=1, kind="rms", gate="sigmoid", after=True, before=True, skip=True, dtype="bf16", stream="f32"),
        # a learner's batch through the same
        dict(name="norm batch", op="norm", n=65536, d=2048, groups=1, kind="rms", gate="sigmoid", after=True, before=True, skip=True, dtype="bf16", stream="f32"),
        # the heads' outputs of an attention, normed each by itself and gated, odd number of rows: gradients
        dict(name="norm heads gradient", op="norm_gradient", n=9999, d=2048, groups=16, kind="layer", gate="silu", after=True, before=False, skip=False,
             dtype="f16", stream="f16"),
        # the learner's gradients through a wide block's end
        dict(name="norm gradient batch", op="norm_gradient", n=32768, d=4096, groups=1, kind="rms", gate="sigmoid", after=True, before=True, skip=True,
             dtype="bf16", stream="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["step", "unroll", "unroll", "gradient", "norm", "norm_gradient"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_gradient"):
        while True:
            n, d = _log_uniform(rng, 1, 262144), _log_uniform(rng, 16, 16384)
            if n * d <= 1 << 27:
                break
        groups = rng.choice([1, 1, 1, 4, 16])
        d = max(1, d // groups) * groups
        return dict(op=op, n=n, d=d, groups=groups, kind=rng.choice(["rms", "rms", "layer"]), gate=rng.choice(["none", "sigmoid", "silu"]),
                    after=groups > 1 or rng.random() < 0.8, before=groups == 1 and rng.random() < 0.7, skip=rng.random() < 0.7, dtype=dtype,
                    stream=rng.choice([dtype, "f32"]))
    while True:
        hk, share = _log_uniform(rng, 1, 16), rng.choice([1, 1, 1, 2, 4])
        dk, dv = (rng.choice([32, 64, 96, 128, 256, rng.randint(8, 256)]) for _ in range(2))
        b, t = _log_uniform(rng, 1, 512), _log_uniform(rng, 1, 65536)
        if op == "step" and b * hk * share * dk * dv <= 1 << 27:
            return dict(op=op, b=b, h=hk * share, hk=hk, dk=dk, dv=dv, dtype=dtype, resets=rng.choice([0.0, 0.05]))
        if op != "step" and b * t * hk * share * (dk + dv) <= (1 << 28 if op == "unroll" else 1 << 26):
            return dict(op=op, b=b, t=t, h=hk * share, hk=hk, dk=dk, dv=dv, dtype=dtype, resets=rng.choice([0.0, 0.003, 0.03]),
                        ragged=rng.random() < 0.4, state=rng.random() < 0.5)


def work(case):
    op = case["op"]
    if op in ("norm", "norm_gradient"):
        n, d, e, s = case["n"], case["d"], BYTES[case["dtype"]], BYTES[case["stream"]] if case["skip"] else BYTES[case["dtype"]]
        gated, weights = case["gate"] != "none", 4 * d * (case["after"] + case["before"])
        if op == "norm":          # y, gate and x read, u and h written
            return {"bytes": n * d * (e * (1 + gated + case["before"]) + s * (1 + case["skip"])) + weights, "flops": 20 * n * d}
        # y, gate, x and the gradients of u and h read, those of y, gate and x written (x only shapes the norm before the next block)
        return {"bytes": n * d * (e * (2 + 2 * gated + case["before"]) + s * (1 + case["skip"] + (case["skip"] and case["before"]))) + 2 * weights,
                "flops": 40 * n * d}
    b, h, hk, dk, dv, e = case["b"], case["h"], case["hk"], case["dk"], case["dv"], BYTES[case["dtype"]]
    state = 4 * b * h * dk * dv
    token = e * (h * (dk + dv) + hk * (dk + dv))                      # q and o, k and v
    if op == "step":
        return {"bytes": 2 * state + b * token, "flops": 5 * b * h * dk * dv}
    t = case["t"] if not case["ragged"] else (case["t"] + 1) // 2
    if op == "unroll":
        return {"bytes": b * t * token + state * (1 + case["state"]), "flops": 4 * b * t * h * dk * dv}
    # q, k, v and the output's gradient read, the gradients of q, k and v written; the state and its gradients
    return {"bytes": b * t * e * (2 * h * dk + h * dv + 2 * hk * (dk + dv)) + 3 * state * case["state"], "flops": 10 * b * t * h * dk * dv}


def _decay(h):
    """Memories of 16 to 1024 tokens."""
    return [1.0 - 2.0 ** -(4 + 6 * (i + 0.5) / h) for i in range(h)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    dtype = DTYPES[case["dtype"]]
    state = dict(case=case)
    if case["op"] in ("norm", "norm_gradient"):
        n, d, stream = case["n"], case["d"], DTYPES[case["stream"]] if case["skip"] else dtype
        # block outputs whose rows differ in size, a residual stream that has grown
        state["y"] = (normal(n, d) * torch.exp(normal(n, 1))).to(dtype)
        state["x"] = (3 * normal(n, d)).to(stream) if case["skip"] else None
        state["gate"] = (1.5 * normal(n, d)).to(dtype) if case["gate"] != "none" else None
        state["after"] = 1 + 0.2 * normal(d) if case["after"] else None
        state["before"] = 1 + 0.2 * normal(d) if case["before"] else None
        if case["op"] == "norm_gradient":
            state["grad_u"] = normal(n, d).to(stream)
            state["grad_h"] = normal(n, d).to(dtype) if case["before"] else None
        if own:
            import paper_2211_15023_amd as A
            state["norm"] = A.BlockNorm(d, after=state["after"], before=state["before"], kind=case["kind"], groups=case["groups"], eps=EPS,
                                        gate=None if case["gate"] == "none" else case["gate"], skip=SKIP, branch=BRANCH)
        return state
    b, h, hk, dk, dv = case["b"], case["h"], case["hk"], case["dk"], case["dv"]
    lead = (b,) if case["op"] == "step" else (b, case["t"])
    # queries, keys and values are parts of one projection's rows; keys of about unit length
    rows = normal(*lead, h * dk + hk * (dk + dv))
    rows[..., h * dk:(h + hk) * dk] /= math.sqrt(dk)
    rows = rows.to(dtype)
    q, k, v = rows.split([h * dk, hk * dk, hk * dv], dim=-1)
    state["q"], state["k"], state["v"] = q.unflatten(-1, (h, dk)), k.unflatten(-1, (hk, dk)), v.unflatten(-1, (hk, dv))
    state["decay"] = _decay(h)
    state["scale"] = 1 / math.sqrt(dk)
    state["reset"] = (torch.rand(lead, generator=g, device="cuda") < case["resets"]).to(torch.uint8) if case["resets"] else None
    if case["op"] == "step":
        state["memory"] = normal(b, h, dk, dv)
        state["next"] = torch.empty_like(state["memory"])
    else:
        state["memory"] = normal(b, h, dk, dv) if case["state"] else None
        state["lengths"] = None
        if case["ragged"]:
            state["lengths"] = torch.randint(0, case["t"] + 1, (b,), generator=g, device="cuda").to(torch.int32)
        if case["op"] == "gradient":
            state["grad"] = normal(*lead, h, dv).to(dtype)
            state["grad_memory"] = 0.1 * normal(b, h, dk, dv) if case["state"] else None
    if own:
        import paper_2211_15023_amd as A
        state["attention"] = A.LinearAttention(state["decay"], scale=state["scale"])
    return state


def run(state):
    op = state["case"]["op"]
    if op == "step":
        if own:
            # the new memory goes beside the old one, from which a learner's unroll may begin
            return state["attention"].step(state["q"], state["k"], state["v"], state["memory"], reset=state["reset"], out_state=state["next"]), state["next"]
        return _step(state)
    if op == "unroll":
        if own:
            return state["attention"].forward(state["q"], state["k"], state["v"], state=state["memory"], reset=state["reset"], lengths=state["lengths"])
        return _unroll(state)
    if op == "gradient":
        if own:
            r = state["attention"].backward(state["grad"], state["q"], state["k"], state["v"], state=state["memory"], reset=state["reset"],
                                            lengths=state["lengths"], grad_state=state["grad_memory"])
            return dict(q=r.q, k=r.k, v=r.v, state=r.state)
        return _unroll_gradient(state)
    if op == "norm":
        if own:
            return state["norm"].forward(state["y"], x=state["x"], gate=state["gate"])
        return _norm(state)
    if own:
        r = state["norm"].backward(state["y"], x=state["x"], gate=state["gate"], grad_u=state["grad_u"], grad_h=state["grad_h"])
        return dict(y=r.y, x=r.x, gate=r.gate, after=r.after, before=r.before)
    return _norm_gradient(state)


# ------------------------------------------------------------------ the plain forms
def _heads(x, h):
    """fp32, a copy for each head that shares it."""
    return x.float().repeat_interleave(h // x.shape[-2], dim=-2)


def _step(state):
    case = state["case"]
    q, k, v = (_heads(state[n], case["h"]) for n in "qkv")
    decay = torch.tensor(state["decay"], device="cuda")[None, :, None, None]
    s = state["memory"]
    if state["reset"] is not None:
        s = torch.where(state["reset"][:, None, None, None] != 0, 0.0, s)
    s = decay * s + k[..., :, None] * v[..., None, :]
    o = state["scale"] * (q[..., :, None] * s).sum(dim=-2)
    return o.to(DTYPES[case["dtype"]]), s


CHUNK = 64


def _mix(a, b, c, enter, log_decay, cut):
    """out_i = a_i E_i with E_i = d_i E_{i-1} + b_i c_i^T, d_i = exp(log_decay_i) or 0 where cut, from E_{-1} = enter on: within pieces
    of CHUNK tokens by products of all pairs, between pieces by their states.  a, b [B, T, H, X], c [B, T, H, Y]; returns out and the last E."""
    B, T, H, X = a.shape
    n = max(1, -(-T // CHUNK))
    pad = n * CHUNK - T

    def pieces(x):
        return torch.nn.functional.pad(x, (0, 0, 0, 0, 0, pad)).view(B, n, CHUNK, H, -1).permute(0, 3, 1, 2, 4)

    a, b, c = pieces(a), pieces(b), pieces(c)
    total = pieces(log_decay[..., None])[..., 0].cumsum(dim=-1)                     # [B, H, n, CHUNK], 64 bits
    part = torch.nn.functional.pad(cut, (0, pad)).view(B, 1, n, CHUNK).long().cumsum(dim=-1)
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=a.device).tril()
    apart = (total[..., :, None] - total[..., None, :]).float()
    near = lower & (part[..., :, None] == part[..., None, :])
    out = (torch.matmul(a, b.transpose(-1, -2).contiguous()) * torch.where(near, torch.exp(apart), 0.0)) @ c
    first = torch.where(part == 0, torch.exp(total), 0.0).float()
    last = torch.where(part == part[..., -1:], torch.exp(total[..., -1:] - total), 0.0).float()
    local = torch.matmul((b * last[..., None]).transpose(-1, -2).contiguous(), c)
    # the state that enters piece i (n: the last one) from what each piece before it adds
    passed = torch.nn.functional.pad(total[..., -1].cumsum(dim=-1), (1, 0))         # [B, H, n + 1]
    parts = torch.nn.functional.pad(part[..., -1].cumsum(dim=-1), (1, 0))
    before = torch.ones((n + 1, n), dtype=torch.bool, device=a.device).tril(-1)
    weight = torch.where(before & (parts[..., :, None] == parts[..., None, 1:]), passed[..., :, None] - passed[..., None, 1:], -math.inf)
    states = torch.matmul(torch.exp(weight).float(), local.flatten(-2)).unflatten(-1, local.shape[-2:])
    states += torch.where(parts == 0, torch.exp(passed), 0.0).float()[..., None, None] * enter[:, :, None]
    out = out + first[..., None] * torch.matmul(a, states[:, :, :n])
    return out.permute(0, 2, 3, 1, 4).reshape(B, n * CHUNK, H, -1)[:, :T], states[:, :, n]


def _unroll_parts(state):
    case = state["case"]
    b, t, h = case["b"], case["t"], case["h"]
    q, k, v = (_heads(state[n], h) for n in "qkv")
    live = torch.ones((b, t), dtype=torch.bool, device="cuda")
    if state["lengths"] is not None:
        live = torch.arange(t, device="cuda")[None] < state["lengths"][:, None]
        q, k, v = (torch.where(live[..., None, None], x, 0.0) for x in (q, k, v))
    cut = (state["reset"] != 0) & live if state["reset"] is not None else torch.zeros((b, t), dtype=torch.bool, device="cuda")
    log_decay = torch.log(torch.tensor(state["decay"], dtype=torch.float64, device="cuda"))
    return q, k, v, live, cut, log_decay


def _unroll(state):
    case = state["case"]
    q, k, v, live, cut, log_decay = _unroll_parts(state)
    enter = state["memory"] if state["memory"] is not None else torch.zeros((case["b"], case["h"], case["dk"], case["dv"]), device="cuda")
    out, last = _mix(q, k, v, enter, torch.where(live[..., None], log_decay, 0.0), cut)
    return (state["scale"] * out).to(DTYPES[case["dtype"]]), last


def _unroll_gradient(state):
    case, scale, dtype = state["case"], state["scale"], DTYPES[state["case"]["dtype"]]
    q, k, v, live, cut, log_decay = _unroll_parts(state)
    go = torch.where(live[..., None, None], state["grad"].float(), 0.0)
    zeros = torch.zeros((case["b"], case["h"], case["dk"], case["dv"]), device="cuda")
    enter = state["memory"] if state["memory"] is not None else zeros
    gq, _ = _mix(go, v, k, enter.transpose(-1, -2), torch.where(live[..., None], log_decay, 0.0), cut)
    # from the last token to the first; what a token's state hands back is cut where the next token begins an episode, and not decayed after the last
    flip = lambda x: x.flip(1)
    behind = torch.zeros_like(live)
    behind[:, :-1] = live[:, 1:]
    cut_behind = torch.zeros_like(cut)
    cut_behind[:, :-1] = cut[:, 1:]
    logs, cuts = flip(torch.where(behind[..., None], log_decay, 0.0)), flip(cut_behind)
    last = state["grad_memory"] if state["grad_memory"] is not None else zeros
    gv, back = _mix(flip(k), flip(q) * scale, flip(go), last, logs, cuts)
    gk, _ = _mix(flip(v), flip(go) * scale, flip(q), last.transpose(-1, -2), logs, cuts)
    if state["memory"] is not None:
        through = torch.where(cut[:, 0, None], 0.0, torch.where(live[:, 0, None], torch.exp(log_decay), 1.0)).float()
        back = through[..., None, None] * back
    shared = lambda x: x.unflatten(2, (case["hk"], case["h"] // case["hk"])).sum(dim=3)
    return dict(q=(scale * gq).to(dtype), k=shared(flip(gk)).to(dtype), v=shared(flip(gv)).to(dtype), state=back if state["memory"] is not None else None)


def _rows_norm(x, kind, groups):
    """x centred (layer) and divided by its root mean square, by groups; and the reciprocal roots."""
    x = x.unflatten(1, (groups, -1))
    if kind == "layer":
        x = x - x.mean(dim=2, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=2, keepdim=True) + EPS)
    return (x * r).flatten(1), r


def _rows_norm_gradient(g, n, r, kind, groups):
    g, n = g.unflatten(1, (groups, -1)), n.unflatten(1, (groups, -1))
    d = g - n * (g * n).mean(dim=2, keepdim=True)
    if kind == "layer":
        d = d - g.mean(dim=2, keepdim=True)
    return (r * d).flatten(1)


def _norm_parts(state):
    case = state["case"]
    y = state["y"].float()
    n, r = _rows_norm(y, case["kind"], case["groups"]) if case["after"] else (y, None)
    m = n * state["after"] if case["after"] else n
    gate = state["gate"].float() if state["gate"] is not None else None
    sig = torch.sigmoid(gate) if gate is not None else None
    s = None if gate is None else sig if case["gate"] == "sigmoid" else gate * sig
    u = BRANCH * (m if s is None else s * m)
    if state["x"] is not None:
        u = SKIP * state["x"].float() + u
    return y, n, r, m, gate, sig, s, u


def _norm(state):
    case = state["case"]
    u = _norm_parts(state)[-1]
    h = (_rows_norm(u, case["kind"], 1)[0] * state["before"]).to(DTYPES[case["dtype"]]) if case["before"] else None
    return u.to(state["x"].dtype if state["x"] is not None else DTYPES[case["dtype"]]), h


def _norm_gradient(state):
    case, dtype = state["case"], DTYPES[state["case"]["dtype"]]
    y, n, r, m, gate, sig, s, u = _norm_parts(state)
    g = state["grad_u"].float()
    out = dict(y=None, x=None, gate=None, after=None, before=None)
    if case["before"]:
        gh = state["grad_h"].float()
        un, ur = _rows_norm(u, case["kind"], 1)
        out["before"] = (gh * un).sum(dim=0, dtype=torch.float64).float()
        g = g + _rows_norm_gradient(gh * state["before"], un, ur, case["kind"], 1)
    if state["x"] is not None:
        out["x"] = (SKIP * g).to(state["x"].dtype)
    g = BRANCH * g
    if gate is not None:
        slope = sig * (1 - sig) if case["gate"] == "sigmoid" else sig * (1 + gate * (1 - sig))
        out["gate"] = (g * m * slope).to(dtype)
        g = g * s
    if case["after"]:
        out["after"] = (g * n).sum(dim=0, dtype=torch.float64).float()
        g = _rows_norm_gradient(g * state["after"], n, r, case["kind"], case["groups"])
    out["y"] = g.to(dtype)
    return out


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] in ("norm", "norm_gradient"):
        return _exact_norm(state)
    return {"step": _exact_step, "unroll": _exact_unroll, "gradient": _exact_gradient}[case["op"]](state)


def _wide(x, h):
    """[..., shared heads, D] in 64 bits as [..., h, D]."""
    x = x.double()
    return x[..., None, :].expand(*x.shape[:-1], h // x.shape[-2], x.shape[-1]).flatten(-3, -2)


def _exact_step(state):
    h = state["case"]["h"]
    g = torch.tensor(state["decay"], dtype=torch.float64, device="cuda").view(1, h, 1, 1).expand(state["case"]["b"], h, 1, 1)
    if state["reset"] is not None:
        g = g * (state["reset"] == 0).double().view(-1, 1, 1, 1)
    new = state["memory"].double() * g + torch.einsum("bhi,bhj->bhij", _wide(state["k"], h), _wide(state["v"], h))
    return torch.einsum("bhi,bhij->bhj", _wide(state["q"], h), new) * state["scale"], new


def _steps(state):
    """For every token: which sequences have it, and the decay of each head's state before it (0 where an episode begins)."""
    case = state["case"]
    n = torch.full((case["b"],), case["t"], device="cuda") if state["lengths"] is None else state["lengths"].long()
    g = torch.tensor(state["decay"], dtype=torch.float64, device="cuda")
    for t in range(case["t"]):
        has = (t < n).double().view(-1, 1)
        keep = torch.ones_like(has) if state["reset"] is None else (state["reset"][:, t] == 0).double().view(-1, 1)
        yield t, has[..., None], (has * keep * g + (1 - has))[..., None, None]


def _start(state, name):
    case = state["case"]
    s = state[name]
    return torch.zeros((case["b"], case["h"], case["dk"], case["dv"]), dtype=torch.float64, device="cuda") if s is None else s.double()


def _exact_unroll(state):
    h, s, out = state["case"]["h"], _start(state, "memory"), []
    for t, has, d in _steps(state):
        s = s * d + (has * _wide(state["k"][:, t], h))[..., :, None] * _wide(state["v"][:, t], h)[..., None, :]
        out.append(state["scale"] * ((has * _wide(state["q"][:, t], h))[..., :, None] * s).sum(dim=-2))
    return torch.stack(out, dim=1), s


def _exact_gradient(state):
    case, h, scale = state["case"], state["case"]["h"], state["scale"]
    s, gq, gk, gv = _start(state, "memory"), [], [], []
    steps = list(_steps(state))
    for t, has, d in steps:
        s = s * d + (has * _wide(state["k"][:, t], h))[..., :, None] * _wide(state["v"][:, t], h)[..., None, :]
        gq.append(scale * (s * (has * state["grad"][:, t].double())[..., None, :]).sum(dim=-1))
    gs = _start(state, "grad_memory")                                 # the gradient of the state behind token t
    for t, has, d in reversed(steps):
        gs = gs + scale * (has * _wide(state["q"][:, t], h))[..., :, None] * state["grad"][:, t].double()[..., None, :]
        gv.append((gs * (has * _wide(state["k"][:, t], h))[..., :, None]).sum(dim=-2))
        gk.append((gs * (has * _wide(state["v"][:, t], h))[..., None, :]).sum(dim=-1))
        gs = gs * d
    fold = lambda x: torch.stack(x[::-1], dim=1).view(case["b"], case["t"], case["hk"], -1, x[0].shape[-1]).sum(dim=3)
    return dict(q=torch.stack(gq, dim=1), k=fold(gk), v=fold(gv), state=gs if state["memory"] is not None else None)


def _exact_norm(state):
    """Values by the definition, gradients by differentiating it, in blocks of rows."""
    case = state["case"]
    rows = max(1, (1 << 25) // case["d"])
    weights = {k: state[k].double().requires_grad_() for k in ("after", "before") if state[k] is not None}
    parts = [_exact_rows(state, weights, slice(i, i + rows)) for i in range(0, case["n"], rows)]
    cat = lambda k: torch.cat([p[k] for p in parts]) if parts[0][k] is not None else None
    if case["op"] == "norm":
        return cat("u"), cat("h")
    return dict(y=cat("y"), x=cat("x"), gate=cat("gate"), **{k: weights[k].grad if k in weights else None for k in ("after", "before")})


def _exact_rows(state, weights, at):
    case = state["case"]
    leaf = {k: state[k][at].double().requires_grad_() if state[k] is not None else None for k in ("y", "x", "gate")}

    def norm(z, groups, weight):
        z = z.reshape(len(z), groups, -1)
        if case["kind"] == "layer":
            z = z - z.sum(dim=-1, keepdim=True) / z.shape[-1]
        return (z / (z.pow(2).sum(dim=-1, keepdim=True) / z.shape[-1] + EPS).sqrt()).reshape(len(z), -1) * weight

    gradient = case["op"] == "norm_gradient"
    with torch.set_grad_enabled(gradient):
        u = leaf["y"] if not case["after"] else norm(leaf["y"], case["groups"], weights["after"])
        if leaf["gate"] is not None:
            open_ = 1 / (1 + torch.exp(-leaf["gate"]))
            u = u * (open_ if case["gate"] == "sigmoid" else leaf["gate"] * open_)
        u = BRANCH * u
        if leaf["x"] is not None:
            u = u + SKIP * leaf["x"]
        h = norm(u, 1, weights["before"]) if case["before"] else None
    if not gradient:
        return dict(u=u, h=h)
    to = [u] + ([h] if h is not None else [])
    torch.autograd.backward(to, [state["grad_u"][at].double()] + ([state["grad_h"][at].double()] if h is not None else []))
    return {k: t.grad if t is not None else None for k, t in leaf.items()}
