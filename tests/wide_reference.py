"""The operators of wide policies in 64 bits, on the CPU, from their formulas (numpy only)."""
import numpy as np

U = 2.0 ** -24                                         # half a step of fp32, relative
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}   # results below the normal range (f16: half its last step)


def quantize(x):
    """x float64 [R, K] -> (q, scale in fp32 as stored, max)."""
    top = np.abs(x).max(axis=1, keepdims=True) if x.shape[1] else np.zeros((len(x), 1))
    with np.errstate(all="ignore"):
        q = np.where(np.isfinite(top) & (top > 0), np.rint(x * 127.0 / top), 0.0)
        scale = top[:, 0].astype(np.float32) / np.float32(127)
    return np.nan_to_num(q).astype(np.int64), scale


def dense(x, wq, w_scale, bias, relu):
    """(y, size of the product part) with the exact scale max / 127."""
    q, _ = quantize(x)
    top = np.abs(x).max(axis=1, keepdims=True)
    prod = (q.astype(np.float64) @ wq.astype(np.float64).T) * (top / 127.0) * w_scale.astype(np.float64)
    y = prod + (0.0 if bias is None else bias.astype(np.float64))
    return (np.where(y < 0, 0.0, y) if relu else y), np.abs(prod)


def softmax_rows(z, mask):
    """(log pi, pi, empty) of float64 logits; masked places -inf."""
    z = np.where(mask, z, -np.inf)
    m = z.max(axis=1, keepdims=True)
    empty = m[:, 0] == -np.inf
    m = np.where(m == -np.inf, 0.0, m)
    with np.errstate(all="ignore"):
        logp = z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))
    logp = np.where(empty[:, None], -np.inf, logp)
    return logp, np.exp(logp), empty


def dot0(p, v):
    with np.errstate(invalid="ignore"):
        return np.where(p > 0, p * v, 0.0)


def policy_loss(z, act, old, adv, mask=None, w=None, kl="none", zr=None, ref_lp=None, clip_low=0.2, clip_high=0.2, ck=0.0, ch=0.0, scale=1.0):
    """dict of loss, logp, kl, entropy [B], stats [4], grad [B, A], and what the tolerances need."""
    B, A = z.shape
    mask = np.ones((B, A), bool) if mask is None else np.broadcast_to(mask, (B, A)).astype(bool)
    w = np.ones(B) if w is None else w.astype(np.float64)
    ids = np.arange(B)
    out_of_range = (act < 0) | (act >= A)
    a = np.where(out_of_range, 0, act)
    with np.errstate(all="ignore"):
        logp, p, empty = softmax_rows(z, mask)
        lp = logp[ids, a]
        H = -dot0(p, logp).sum(axis=1)
        r = np.where(lp == -np.inf, 0.0, np.exp(lp - old))
        lo, hi = 1.0 - clip_low, 1.0 + clip_high
        clipped = np.where(adv >= 0, np.minimum(r, hi), np.maximum(r, lo))
        pg = -clipped * adv
        at = np.where(clipped == r, -r * adv, 0.0)
        D, pr = np.zeros(B), np.zeros((B, A))
        g = ch * dot0(p, logp + H[:, None])
        k = np.zeros(B)
        if kl == "sampled":
            d = ref_lp - lp
            k = np.where(d == np.inf, d, np.exp(d) - d - 1)
            at = at + ck * (1 - np.exp(d))
        elif kl != "none":
            lr, pr, none = softmax_rows(zr, mask)
            diff = logp - lr
            D = np.abs(np.where((p > 0) & (pr > 0), z - zr, 0.0)).max(axis=1) if A else D
            if kl == "forward":
                k = np.where(none, 0.0, dot0(pr, -diff).sum(axis=1))
                g = g + np.where(none, 0.0, ck)[:, None] * (p - pr)
            else:
                k = np.where(none, np.inf, dot0(p, diff).sum(axis=1))
                g = g + ck * dot0(p, diff - k[:, None])
        g = g - at[:, None] * p
        g[ids, a] += at
        dead = out_of_range | (w == 0)
        gone = dead | empty
        loss = np.where(gone, 0.0, pg + ck * k - ch * H)
        k, H = np.where(gone, 0.0, k), np.where(gone, 0.0, H)
        outside = np.where(gone, 0.0, (r < lo) | (r > hi))
        g = np.where(gone[:, None], 0.0, g * (w * scale)[:, None])
        stats = scale * np.array([(w * v)[~dead].sum() for v in (loss, k, H, outside)])
        lp = np.where(dead, 0.0, np.where(empty, -np.inf, lp))
    weight = np.nan_to_num(p) + np.nan_to_num(pr)          # an element's gradient is in proportion to its probabilities
    weight[ids, a] += 1
    return dict(loss=loss, logp=lp, kl=k, entropy=H, stats=stats, grad=g, weight=weight, D=D, at=at, ratio=r, gone=gone, w=w)


def sum_error(A):
    """Relative error of the sums under the maximum.  A term is off by 3 u |d| + 2 u (difference, product and exponential; d = z - max), in
    the mean over the distribution at most 3 u (ln A + 1) + 2 u; a lane adds at most A / 256 + 32 terms, and 16 joins follow that each
    correct a sum by two roundings and an exponential of its own (6 u)."""
    return U * (3 * (np.log(A) + 1) + 2 + A / 256 + 32 + 16 * 6)


def tolerances(ref, z, mask, dtype, kl, adv, ck, ch, scale):
    """Absolute tolerances of the outputs: the sums' error carried through the formulas."""
    B, A = z.shape
    e = sum_error(A)
    lnA = np.log(A) + 1
    with np.errstate(all="ignore"):
        lp = np.where(np.isfinite(ref["logp"]), np.abs(ref["logp"]), 0.0)
        t_lp = e + 4 * U * (lp + 1)
        t_H = 2 * e * (1 + lnA) + 0 * t_lp
        if kl == "sampled":
            x = 1 + ref["kl"]                                # d/d lp of exp(d) - d - 1 is at most 1 + kl + |d|, |d| <= 1 + kl + 1
            t_kl = 3 * x * t_lp + 8 * U * (x + 3)
        else:
            t_kl = 2 * e * (1 + ref["D"] + lnA) + 0 * t_lp
        r = ref["ratio"]
        t_loss = np.abs(adv) * r * (t_lp + 4 * U) + ck * t_kl + ch * t_H + 4 * U * (np.abs(ref["loss"]) + np.abs(adv) * r + ck * ref["kl"] + ch * ref["entropy"])
        size = np.abs(ref["at"]) + np.abs(adv) * r + ck * (2 + ref["D"] + ref["kl"] + lnA) + ch * (1 + 2 * lnA)
        if kl == "sampled":
            size = size + ck * 3 * (1 + ref["kl"])
        t_g = np.where(ref["gone"], 0.0, ref["w"] * scale * size * (4 * e + 16 * U))[:, None] * ref["weight"]
    return dict(logp=t_lp, entropy=t_H, kl=t_kl, loss=t_loss, grad=t_g + HALF_STEP[dtype] * np.abs(ref["grad"]) * 1.001 + TINY[dtype])
