"""The operators of policies with a memory in 64 bits, on the CPU, from their formulas (numpy only), and what fp32 and bf16 may lose of them."""
import numpy as np

U = 2.0 ** -24                                         # half a step of fp32, relative
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}   # results below the normal range (f16: half its last step)


# ------------------------------------------------------------------ linear attention
def _wide(x, H):
    return np.repeat(x, H // x.shape[-2], axis=-2)


def _has(b, t, lengths, T):
    return t < (T if lengths is None else min(max(int(lengths[b]), 0), T))


def unroll(q, k, v, decay, scale, reset=None, lengths=None, state=None):
    """Token by token, what a sequence does not have left out (it may hold anything) -> out [B, T, H, Dv], state [B, H, Dk, Dv]."""
    B, T, H, Dk = q.shape
    Dv = v.shape[3]
    out, S = np.zeros((B, T, H, Dv)), np.zeros((B, H, Dk, Dv))
    with np.errstate(all="ignore"):
        for b in range(B):
            s = np.zeros((H, Dk, Dv)) if state is None else state[b].astype(np.float64)
            for t in range(T):
                if not _has(b, t, lengths, T):
                    break
                if reset is not None and reset[b, t]:
                    s = np.zeros_like(s)
                s = decay[:, None, None] * s + _wide(k[b, t], H)[:, :, None] * _wide(v[b, t], H)[:, None, :]
                out[b, t] = scale * (q[b, t][:, :, None] * s).sum(axis=1)
            S[b] = s
    return out, S


def unroll_grad(go, q, k, v, decay, scale, reset=None, lengths=None, state=None, gs=None):
    """dict of q, k, v, state: the gradients of sum(go . out) + sum(gs . state behind the last token)."""
    B, T, H, Dk = q.shape
    Hk, Dv = v.shape[2], v.shape[3]
    g = dict(q=np.zeros(q.shape), k=np.zeros(k.shape), v=np.zeros(v.shape), state=np.zeros((B, H, Dk, Dv)))
    fold = lambda x: x.reshape(Hk, H // Hk, -1).sum(axis=1)
    with np.errstate(all="ignore"):
        for b in range(B):
            n = sum(_has(b, t, lengths, T) for t in range(T))
            s = np.zeros((H, Dk, Dv)) if state is None else state[b].astype(np.float64)
            for t in range(n):
                if reset is not None and reset[b, t]:
                    s = np.zeros_like(s)
                s = decay[:, None, None] * s + _wide(k[b, t], H)[:, :, None] * _wide(v[b, t], H)[:, None, :]
                g["q"][b, t] = scale * (s * go[b, t][:, None, :]).sum(axis=2)
            r = np.zeros((H, Dk, Dv)) if gs is None else gs[b].astype(np.float64)
            for t in range(n)[::-1]:
                r = r + scale * q[b, t][:, :, None] * go[b, t][:, None, :]
                g["v"][b, t] = fold((r * _wide(k[b, t], H)[:, :, None]).sum(axis=1))
                g["k"][b, t] = fold((r * _wide(v[b, t], H)[:, None, :]).sum(axis=2))
                r = np.zeros_like(r) if reset is not None and reset[b, t] else decay[:, None, None] * r
            g["state"][b] = r
    return g


def unroll_roundings(T, D, decay):
    """Roundings of fp32, each relative to the sum of the terms' magnitudes, that a result of the chunked form may have gone through: D of a product over
    a head, 64 of one over a chunk, and again 64 and the decay for each chunk that the state is carried on; the powers of the decay, whose exponent n log g
    is off by 3 parts (its logarithm, its base and the product; weights below e^-104 are nothing), 2 for the power itself; 8 for scales, splits and sums of heads."""
    chunks = T / 64 + 1
    slow = max([0.0] + [min(-T * np.log(d), 104.0) for d in decay if d > 0])
    return 2 * D + 64 + 66 * chunks + 3 * slow + 2 + 8


def unroll_tolerance(ref, size, dtype, T, D, decay, state=False):
    """size: the same result of magnitudes.  bf16: the weights of pairs and the state's copy are rounded once (half a step of the size); a state's terms may be
    held in two halves of which the second is rounded (half a step, squared).  Last the result's own rounding."""
    part = unroll_roundings(T, D, decay) * U
    if dtype == "bf16":
        part += HALF_STEP["bf16"] ** 2 if state else HALF_STEP["bf16"] * 1.01
    kind = "f32" if state else dtype
    return size * part + HALF_STEP[kind] * np.abs(ref) * 1.001 + TINY[kind]


# ------------------------------------------------------------------ norms around a block
def _norm(z, kind, groups, eps):
    z = z.reshape(len(z), groups, -1)
    m = z.mean(axis=2, keepdims=True) if kind == "layer" else 0.0
    r = 1.0 / np.sqrt(((z - m) ** 2).mean(axis=2, keepdims=True) + eps)
    flat = lambda x: np.broadcast_to(x, z.shape).reshape(len(z), -1)
    return flat((z - m) * r), flat(r)


def _through(t, n, r, kind, groups, sign=-1.0):
    """The gradient by a norm's input; sign = +1 adds magnitudes."""
    part = lambda x: x.reshape(len(x), groups, -1)
    mean = lambda x: np.broadcast_to(part(x).mean(axis=2, keepdims=True), part(x).shape).reshape(x.shape)
    return r * (t + sign * n * mean(t * n) + (sign * mean(t) if kind == "layer" else 0.0))


def block_norm(y, x=None, gate=None, after=None, before=None, kind="rms", gate_kind=None, groups=1, eps=1e-6, skip=1.0, branch=1.0, gu=None, gh=None):
    """Values and, with gu or gh, gradients; and by "size" the magnitudes that fp32's roundings are relative to.

    A normed value carries the error of its mean, which is a part of the mean magnitude: its size is r (|z| + mean |z|) with "layer".  The
    sizes of what is made of it are the same formulas with every term's size and all signs positive."""
    with np.errstate(all="ignore"):
        mean = lambda z, g: np.broadcast_to(z.reshape(len(z), g, -1).mean(axis=2, keepdims=True), (len(z), g, z.shape[1] // g)).reshape(z.shape)
        size_of = lambda z, r, g: r * (z + (mean(z, g) if kind == "layer" else 0.0))
        n, r = _norm(y, kind, groups, eps) if after is not None else (y, np.ones_like(y))
        ns = size_of(np.abs(y), r, groups) if after is not None else np.abs(y)
        m, ms = (n * after, ns * np.abs(after)) if after is not None else (n, ns)
        s, slope = np.ones_like(y), np.zeros_like(y)
        ss, slopes = s, slope
        if gate_kind is not None:
            e = 1 / (1 + np.exp(-gate))
            s, slope = (e, e * (1 - e)) if gate_kind == "sigmoid" else (gate * e, e * (1 + gate * (1 - e)))
            more = 1 + np.abs(gate)                              # an exponential's error is in proportion to its argument
            ss, slopes = more * np.abs(s), more * (e if gate_kind == "sigmoid" else e * (1 + np.abs(gate)))
        u, us = branch * s * m, abs(branch) * ss * ms
        if x is not None:
            u, us = u + skip * x, us + np.abs(skip * x)
        out, size = dict(u=u), dict(u=us)
        if before is not None:
            hn, hr = _norm(u, kind, 1, eps)
            # (an element's error moves the row's root mean square too)
            hs = size_of(us, hr, 1)
            hs = hs + np.abs(hn) * np.sqrt((hs ** 2).mean(axis=1, keepdims=True))
            out["h"], size["h"] = hn * before, hs * np.abs(before)
        if gu is None and gh is None:
            return out, size
        g = np.zeros_like(y) if gu is None else gu
        gs = np.abs(g)
        if before is not None and gh is not None:
            t = gh * before
            g = g + _through(t, hn, hr, kind, 1)
            gs = gs + _through(np.abs(t), hs, hr * np.sqrt(1 + (hs ** 2).mean(axis=1, keepdims=True)), kind, 1, 1.0)
            out["before"], size["before"] = (gh * hn).sum(axis=0), (np.abs(gh) * hs).sum(axis=0)
        elif before is not None:
            out["before"], size["before"] = np.zeros(y.shape[1]), np.zeros(y.shape[1])
        if x is not None:
            out["x"], size["x"] = skip * g, abs(skip) * gs
        g, gs = branch * g, abs(branch) * gs
        if gate_kind is not None:
            out["gate"], size["gate"] = g * m * slope, gs * ms * slopes
            g, gs = g * s, gs * ss
        if after is not None:
            out["after"], size["after"] = (g * n).sum(axis=0), (gs * ns).sum(axis=0)
            g = _through(g * after, n, r, kind, groups)
            gs = _through(gs * np.abs(after), ns, r, kind, groups, 1.0)
        out["y"], size["y"] = g, gs
    return out, size


def norm_tolerance(ref, size, dtype, D, rows=1):
    """A row's sum goes through at most 16 roundings in a lane, 6 in a wavefront and 16 of a workgroup's wavefronts (half of them count in a root), and an
    element of a gradient sees at most six sums (two norms, each forwards and by two sums back) and 40 other roundings; a weight's gradient is summed over the rows of a slot in
    fp32 (at most `rows` of them) and joined in 64 bits."""
    part = (6 * 38 + 40 + rows) * U
    return size * part + HALF_STEP[dtype] * np.abs(ref) * 1.001 + TINY[dtype]
