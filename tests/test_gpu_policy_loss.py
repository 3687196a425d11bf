"""The clipped policy loss, its gradient and the log-probabilities of actions against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from tests import wide_reference as ref

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KLS = ["none", "sampled", "forward", "reverse"]
# one lane to a whole row's lanes; rows of a workgroup; rows in pieces; rows enough that none is split
SIZES = [(1, 1), (1, 2), (5, 3), (33, 18), (70, 33), (64, 64), (7, 65), (300, 130), (9, 511), (4, 512), (3, 513), (2, 4097), (5, 9001), (1, 70001), (513, 1000), (530, 5003)]


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def as64(t):
    return t.cpu().double().numpy()


class Inputs:
    def __init__(self, B, A, dtype, kl, mask, seed, ld=0, spread=2.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.A, self.dtype, self.kl = B, A, dtype, kl

        def table(t):
            full = torch.full((B, A + ld), float("nan"), dtype=TORCH[dtype], device="cuda")
            full[:, :A] = t.to(TORCH[dtype]).cuda()
            return full[:, :A]

        z = torch.randn((B, A), generator=g) * spread
        self.z, self.zr = table(z), table(z + 0.5 * torch.randn((B, A), generator=g))
        self.mask = None
        if mask != "none":
            self.mask = (torch.rand((B if mask == "rows" else 1, A), generator=g) < 0.6).to(torch.uint8)
            if mask == "rows":
                self.mask[B // 2] = 0                                         # a row that allows nothing
        act = torch.randint(0, A, (B,), generator=g, dtype=torch.int32)
        if kl == "sampled" and self.mask is not None:                         # (an action of probability 0 has an infinite KL)
            act = torch.argmax(self.mask.expand(B, A) * torch.rand((B, A), generator=g), dim=1).to(torch.int32)
        if B > 4:
            act[1], act[2] = -1, A                                            # rows without an action
        self.act = act
        m = np.ones((B, A), bool) if self.mask is None else np.broadcast_to(self.mask.numpy() != 0, (B, A))
        lp = ref.softmax_rows(as64(self.z), m)[0][np.arange(B), np.clip(act.numpy(), 0, A - 1)]
        lp = np.where(np.isfinite(lp), lp, -1.0)
        # ratios that are clear of the clipping borders by more than any rounding
        self.old = (torch.from_numpy(lp) + torch.tensor([-0.4, -0.1, 0.0, 0.1, 0.4])[torch.randint(0, 5, (B,), generator=g)]).float()
        self.ref_lp = (torch.from_numpy(lp) + 0.3 * torch.randn(B, generator=g)).float()
        self.adv = torch.randn(B, generator=g)
        self.w = (torch.rand(B, generator=g) + 0.5) * (torch.rand(B, generator=g) < 0.8)
        self.scale = 1.0
        self.ck, self.ch, self.lo, self.hi = 0.3, 0.05, 0.2, 0.25

    def run(self, A, grad=True, stream=None):
        self.how = A.PolicyLoss(self.lo, self.hi, self.kl, self.ck, self.ch)
        c = lambda t: None if t is None else t.cuda()
        wide = self.kl in ("forward", "reverse")
        return self.how.forward(self.z, c(self.act), c(self.old), c(self.adv), mask=c(self.mask), weights=c(self.w), scale=self.scale,
                                ref_logits=self.zr if wide else None, ref_logp=c(self.ref_lp) if self.kl == "sampled" else None, grad=grad, stream=stream)

    def want(self):
        mask = None if self.mask is None else self.mask.numpy()
        r = ref.policy_loss(as64(self.z), self.act.numpy(), as64(self.old), as64(self.adv), mask, as64(self.w), self.kl, as64(self.zr), as64(self.ref_lp),
                            self.lo, self.hi, self.ck, self.ch, self.scale)
        t = ref.tolerances(r, as64(self.z), mask, self.dtype, self.kl, as64(self.adv), self.ck, self.ch, self.scale)
        return r, t

    def check(self, got, grad=True):
        r, t = self.want()
        for name in ("loss", "logp", "kl", "entropy"):
            y, x = as64(getattr(got, name)), r[name]
            assert np.array_equal(np.isfinite(y), np.isfinite(x)), name
            ok = np.isfinite(x)
            assert np.array_equal(y[~ok], x[~ok]), name
            off = np.abs(y[ok] - x[ok])
            assert (off <= t[name][ok]).all(), (name, np.max(off / t[name][ok]))
        w = as64(self.w)
        fp = 2 * ref.U
        for k, name in enumerate(("loss", "kl", "entropy")):
            tol = np.nansum(w * np.where(np.isfinite(t[name]), t[name], 0)) * self.scale + fp * np.abs(r["stats"][k]) + 1e-30
            assert abs(float(got.stats[k]) - r["stats"][k]) <= tol, name
        assert abs(float(got.stats[3]) - r["stats"][3]) <= fp * abs(r["stats"][3])
        if grad:
            off = np.abs(as64(got.grad) - r["grad"])
            worst = np.unravel_index(np.argmax(off / t["grad"]), off.shape)
            assert (off <= t["grad"]).all(), (worst, off[worst], t["grad"][worst])


@pytest.mark.parametrize("B,n", SIZES)
@pytest.mark.parametrize("kl", KLS)
def test_loss_sizes(A, B, n, kl):
    x = Inputs(B, n, "f32", kl, "none", seed=B * 7 + n)
    x.check(x.run(A))


@pytest.mark.parametrize("B,n", [(33, 18), (300, 130), (3, 513), (5, 9001), (513, 1000)])
@pytest.mark.parametrize("mask", ["shared", "rows"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kl", KLS)
def test_loss_masks_and_types(A, B, n, mask, dtype, kl):
    x = Inputs(B, n, dtype, kl, mask, seed=B + n)
    x.check(x.run(A))


@pytest.mark.parametrize("B,n,ld", [(9, 18, 3), (70, 65, 1), (4, 1001, 7), (520, 1001, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kl", ["none", "forward"])
def test_loss_strides(A, B, n, ld, dtype, kl):
    """Rows of a stride of their own, the gradient's another one; nothing behind a row is read (NaN) or written."""
    x = Inputs(B, n, dtype, kl, "none", seed=ld, ld=ld)
    g = torch.full((B, n + 5), 9.0, dtype=TORCH[dtype], device="cuda")
    x.check(x.run(A, grad=g[:, :n]))
    assert torch.all(g[:, n:] == 9.0)


class Sparse(Inputs):
    """Many rows, of which few count: the others are not read, and only those few are worked out in 64 bits."""

    def __init__(self, B, A, dtype, kl, mask, seed, live=5):
        super().__init__(live, A, dtype, kl, mask, seed)
        self.live = torch.randperm(B, generator=torch.Generator().manual_seed(seed))[:live]
        few = {k: getattr(self, k) for k in ("z", "zr", "mask", "act", "old", "ref_lp", "adv", "w")}
        few["w"] = few["w"] + 0.25
        self.few, self.B = few, B

        def spread(t, fill):
            out = torch.full((B, *t.shape[1:]), fill, dtype=t.dtype, device=t.device)
            out[self.live.to(t.device)] = t
            return out

        self.z, self.zr = spread(few["z"], float("nan")), spread(few["zr"], float("nan"))
        if mask == "rows":
            self.mask = spread(few["mask"], 1)
        self.act, self.old, self.ref_lp, self.adv = (spread(few[k], 0) for k in ("act", "old", "ref_lp", "adv"))
        self.w = spread(few["w"], 0)

    def check(self, got):
        where = self.live.cuda()
        dead = torch.ones(self.B, dtype=torch.bool, device="cuda")
        dead[where] = False
        assert not got.grad[dead].any() and not got.loss[dead].any() and not got.logp[dead].any()
        part = type(got)()
        part.stats = got.stats
        for k in ("loss", "logp", "kl", "entropy", "grad"):
            setattr(part, k, getattr(got, k)[where])
        for k, v in self.few.items():
            setattr(self, k, v)
        super().check(part)


@pytest.mark.parametrize("n", [5003, 9000, 17001, 33333, 60001, 130001, 190003])
@pytest.mark.parametrize("dtype,kl,mask", [("f32", "forward", "none"), ("bf16", "reverse", "rows"), ("f16", "none", "shared"), ("bf16", "forward", "none"), ("f32", "sampled", "none")])
def test_loss_long_rows(A, n, dtype, kl, mask):
    """Every number of vectors that stay in registers, what LDS holds behind them, and what is read twice."""
    x = Sparse(300, n, dtype, kl, mask, seed=n)
    x.check(x.run(A))


@pytest.mark.parametrize("vectors", [4, 8, 15, 17, 20, 28, 30, 36, 44, 48, 56, 96, 112])
@pytest.mark.parametrize("more", [-1, 0, 1, 1027])
@pytest.mark.parametrize("dtype,kl", [("bf16", "forward"), ("f16", "sampled"), ("f32", "reverse"), ("bf16", "none")])
def test_loss_long_rows_at_whole_vectors(A, vectors, more, dtype, kl):
    """Rows of a whole number of vectors for 256 threads, and a little less or more, where one form takes over from another and where what
    registers and LDS hold just ends."""
    x = Sparse(257, vectors * 256 * (4 if dtype == "f32" else 8) + more, dtype, kl, "shared" if vectors % 8 else "none", seed=vectors)
    x.check(x.run(A))


@pytest.mark.parametrize("vectors", [8, 15, 20, 27, 28, 44])
@pytest.mark.parametrize("dtype,kl", [("bf16", "forward"), ("f16", "reverse"), ("f32", "none")])
def test_loss_long_rows_with_masks_of_their_own(A, vectors, dtype, kl):
    x = Sparse(257, vectors * 256 * (4 if dtype == "f32" else 8) + 5, dtype, kl, "rows", seed=vectors)
    x.check(x.run(A))


@pytest.mark.parametrize("n", [40001, 130001])
@pytest.mark.parametrize("dtype,kl", [("f32", "forward"), ("bf16", "reverse"), ("f16", "sampled"), ("bf16", "none")])
@pytest.mark.parametrize("B", [1, 3, 40])
def test_loss_long_rows_in_pieces(A, B, n, dtype, kl):
    x = Sparse(B, n, dtype, kl, "none", seed=n, live=min(B, 4))
    x.check(x.run(A))


@pytest.mark.parametrize("n", [9000, 130001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kl", KLS)
def test_loss_long_rows_with_infinities(A, n, dtype, kl):
    """Logits of -inf and of the type's lowest value in long rows, which are then summed the careful way."""
    x = Sparse(300, n, dtype, kl, "none", seed=n)
    for t, k in ((x.z, "z"), (x.zr, "zr")):
        t[:, 1::3] = float("-inf")
        t[:, 2::3] = torch.finfo(TORCH[dtype]).min
        x.few[k] = t[x.live.cuda()]
    x.act[x.live] = 0
    x.few["act"] = x.act[x.live]
    x.check(x.run(A))


@pytest.mark.parametrize("B,n", [(40, 18), (3, 9001), (513, 1000)])
@pytest.mark.parametrize("kl", ["sampled", "reverse"])
def test_loss_gradient_in_place_and_without(A, B, n, kl):
    x = Inputs(B, n, "bf16", kl, "rows", seed=1)
    got = x.run(A)
    alone = x.run(A, grad=False)
    assert alone.grad is None
    for name in ("loss", "logp", "kl", "entropy", "stats"):
        assert torch.equal(getattr(alone, name), getattr(got, name)), name
    kept = x.z.clone()
    again = x.run(A, grad=x.z)
    assert torch.equal(again.grad, got.grad) and torch.equal(again.loss, got.loss) and torch.equal(again.stats, got.stats)
    assert again.grad.data_ptr() == x.z.data_ptr() and not torch.equal(x.z, kept)


@pytest.mark.parametrize("B,n", [(6, 18), (6, 300), (6, 5000), (600, 1000)])
@pytest.mark.parametrize("kl", KLS)
def test_loss_repeats(A, B, n, kl):
    x = Inputs(B, n, "f32", kl, "none", seed=11)
    a, b = x.run(A), x.run(A)
    for name in ("loss", "logp", "kl", "entropy", "stats", "grad"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("B,n", [(8, 18), (8, 200), (8, 3000), (520, 1000)])
@pytest.mark.parametrize("kl", KLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_loss_masked_places_hold_anything(A, B, n, kl, dtype):
    """NaN, infinities and the type's lowest value where the mask has a zero; the lowest value and -inf where it has not."""
    x = Inputs(B, n, dtype, kl, "rows", seed=21)
    clean = x.run(A)
    hole = x.mask.cuda() == 0
    for v in (float("nan"), float("inf"), float("-inf"), torch.finfo(TORCH[dtype]).min):
        x.z[hole] = v
        x.zr[hole] = v
        got = x.run(A)
        for name in ("loss", "logp", "kl", "entropy", "stats", "grad"):
            assert torch.equal(getattr(got, name), getattr(clean, name)), (v, name)
    low = torch.finfo(TORCH[dtype]).min
    y = Inputs(B, n, dtype, kl, "none", seed=21)
    y.act = torch.zeros(B, dtype=torch.int32)
    y.z[:, 1::3] = low
    y.zr[:, 1::3] = low
    lowest = y.run(A)
    y.z[:, 1::3] = float("-inf")
    y.zr[:, 1::3] = float("-inf")
    minus = y.run(A)
    for name in ("loss", "logp", "kl", "entropy", "stats", "grad"):
        assert torch.equal(getattr(lowest, name), getattr(minus, name)), name
    y.check(minus)


@pytest.mark.parametrize("n", [18, 200, 3000])
def test_loss_rows_of_lowest_values_are_uniform(A, n):
    for low in (torch.finfo(torch.float32).min, -1e30, 1e30):
        z = torch.full((600 if n == 3000 else 4, n), low, device="cuda")
        lp, ent = A.PolicyLoss().logprob(z, torch.zeros(len(z), dtype=torch.int32, device="cuda"))
        tol = ref.sum_error(n) * 2 * (1 + np.log(n))
        assert (lp + np.log(n)).abs().max() <= tol and (ent - np.log(n)).abs().max() <= tol
    z = torch.full((4, n), float("-inf"), device="cuda")
    lp, ent = A.PolicyLoss().logprob(z, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert torch.all(lp == float("-inf")) and torch.all(ent == 0)


@pytest.mark.parametrize("n", [18, 300, 5000])
@pytest.mark.parametrize("kl", KLS)
def test_loss_not_a_number_stays_in_its_row(A, n, kl):
    for rows in (6, 600) if n == 5000 else (6,):
        x = Inputs(rows, n, "f32", kl, "none", seed=31)
        x.w[:] = 1.0
        x.act[:] = 0
        x.z[3, n // 2], x.z[4, n - 1] = float("nan"), float("inf")
        r = x.run(A)
        assert torch.isnan(r.loss[3:5]).all() and torch.isnan(r.grad[3:5]).all() and torch.isnan(r.logp[3:5]).all()
        keep = [i for i in range(rows) if i not in (3, 4)]
        assert torch.isfinite(r.loss[keep]).all() and torch.isfinite(r.grad[keep]).all()
        assert torch.isnan(r.stats[0])
        # of no weight: neither read nor counted
        x.w[3:5] = 0.0
        r = x.run(A)
        assert torch.isfinite(r.stats).all() and torch.all(r.grad[3:5] == 0) and torch.all(r.loss[3:5] == 0) and torch.all(r.logp[3:5] == 0)


@pytest.mark.parametrize("B,n", [(5, 18), (5, 400), (5, 3000), (515, 1100)])
def test_loss_probability_zero(A, B, n):
    """An action that the mask forbids has ratio 0; a reference without an allowed action gives the forward KL 0."""
    x = Inputs(B, n, "f32", "forward", "none", seed=41)
    x.w[:] = 1.0
    x.mask = torch.ones((1, n), dtype=torch.uint8)
    x.mask[0, 0] = 0
    x.act[:] = 0
    x.zr[:] = float("-inf")
    r = x.run(A)
    x.check(r)
    assert torch.all(r.logp == float("-inf")) and torch.all(r.kl == 0)
    x.kl = "reverse"
    assert torch.all(x.run(A).kl == float("inf"))
    kept, x.ck = x.ck, 0.0
    zero = x.run(A)
    assert torch.isfinite(zero.loss).all() and torch.isfinite(zero.grad).all()
    x.ck, x.kl = kept, "sampled"
    x.ref_lp[:] = -3.0
    r = x.run(A)
    assert torch.all(r.kl == float("inf")) and torch.all(r.loss == float("inf"))
    x.ck = 0.0                                                                # a term of coefficient 0 is no part of the loss
    zero = x.run(A)
    x.kl = "none"
    plain = x.run(A)
    assert torch.equal(zero.loss, plain.loss) and torch.equal(zero.grad, plain.grad) and torch.isfinite(zero.grad).all()


@pytest.mark.parametrize("B,n", [(2000, 18), (64, 400)])
def test_loss_next_to_the_clipping_border(A, B, n):
    """Ratios within a few parts in 2^24 of a border: the side is the one that 64 bits give."""
    x = Inputs(B, n, "f32", "none", "none", seed=51)
    x.w[:] = 1.0
    x.act = torch.randint(0, n, (B,), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    lp = ref.softmax_rows(as64(x.z), np.ones((B, n), bool))[0][np.arange(B), x.act.numpy()]
    border = np.where(np.arange(B) % 2 == 0, np.log(1.25), np.log(0.8))
    x.adv = torch.from_numpy(np.where(np.arange(B) % 4 < 2, 1.0, -1.0)).float()
    x.old = torch.from_numpy(lp - border).float()                              # the ratio is off the border by the rounding of `old`
    x.check(x.run(A))


def test_loss_gradient_against_differences(A):
    """The kernel's gradient is the slope of the 64-bit loss."""
    x = Inputs(6, 30, "f32", "reverse", "rows", seed=61)
    x.act = torch.from_numpy(np.array([np.flatnonzero(m)[0] if m.any() else 0 for m in x.mask.numpy()], np.int32))
    g = as64(x.run(A).grad)
    r, t = x.want()
    z, h = as64(x.z), 1e-5
    f = lambda z: ref.policy_loss(z, x.act.numpy(), as64(x.old), as64(x.adv), x.mask.numpy(), as64(x.w), x.kl, as64(x.zr), as64(x.ref_lp), x.lo, x.hi, x.ck,
                                  x.ch, x.scale)["stats"][0]
    for b in range(6):
        for j in range(30):
            up, down = z.copy(), z.copy()
            up[b, j] += h
            down[b, j] -= h
            assert abs((f(up) - f(down)) / (2 * h) - g[b, j]) <= t["grad"][b, j] + 50 * h * h + 1e-14 / h


@pytest.mark.parametrize("B,n", SIZES)
@pytest.mark.parametrize("dtype,mask", [("f32", "none"), ("bf16", "rows"), ("f16", "shared")])
def test_logprob(A, B, n, dtype, mask):
    x = Inputs(B, n, dtype, "none", mask, seed=n)
    lp, ent = A.PolicyLoss().logprob(x.z, x.act.cuda(), mask=None if x.mask is None else x.mask.cuda())
    x.w[:] = 1.0
    r, t = x.want()
    for got, name in ((lp, "logp"), (ent, "entropy")):
        y = as64(got)
        assert np.array_equal(np.isfinite(y), np.isfinite(r[name])) and np.array_equal(y[~np.isfinite(y)], r[name][~np.isfinite(y)])
        ok = np.isfinite(y)
        assert np.all(np.abs(y - r[name])[ok] <= t[name][ok]), name


def test_logprob_is_the_losss(A):
    """What the actor stored is what the learner finds: ratio 1 on the same logits, to the last bit of the log-probability."""
    for B, n in ((200, 18), (4, 5000), (600, 1000)):
        x = Inputs(B, n, "bf16", "none", "rows", seed=3)
        x.w[:] = 1.0
        lp, _ = A.PolicyLoss().logprob(x.z, x.act.cuda(), mask=x.mask.cuda())
        assert torch.equal(x.run(A).logp, lp)


def test_loss_long_rows_past_32_bits(A):
    """A table of more than 2^32 bytes: the last rows are where they should be."""
    B, n = 2049, 1 << 20
    z = torch.zeros((B, n), dtype=torch.bfloat16, device="cuda")
    act = torch.full((B,), n - 1, dtype=torch.int32, device="cuda")
    z[B - 1, n - 1] = 3.0
    lp, ent = A.PolicyLoss().logprob(z, act)
    r = A.PolicyLoss().forward(z, act, lp, torch.ones(B, device="cuda"), scale=1.0)
    want = 3.0 - np.log(np.exp(3.0) + n - 1)
    tol = ref.sum_error(n) + 4 * ref.U * 15
    assert abs(float(lp[B - 1]) - want) <= tol and abs(float(lp[0]) + np.log(n)) <= tol
    assert abs(float(r.grad[B - 1, n - 1]) + 1 - np.exp(want)) <= 2 ** -8 and abs(float(r.grad[B - 2, n - 1]) + 1 - 1 / n) <= 2 ** -8
    assert float(r.grad[B - 1, 0]) > 0


def test_loss_refuses_tensors(A):
    x = Inputs(4, 10, "f32", "forward", "none", seed=1)
    how = A.PolicyLoss(kl="forward", kl_coef=0.1)
    act, v = x.act.clamp(0, 9).cuda(), x.adv.cuda()
    good = dict(ref_logits=x.zr)
    how.forward(x.z, act, v, v, **good)
    for bad in (dict(ref_logits=x.zr[:, :9]), dict(ref_logits=x.zr.half()), dict(ref_logits=None), dict(good, mask=torch.ones(4, 10, device="cuda")),
                dict(good, mask=torch.ones((3, 10), dtype=torch.uint8, device="cuda")), dict(good, weights=v[:3]), dict(good, weights=v.double()),
                dict(good, grad=torch.empty((4, 9), device="cuda"))):
        with pytest.raises((ValueError, A.AccerlError)):
            how.forward(x.z, act, v, v, **bad)
    for z, a, o in ((x.z.double(), act, v), (x.z.t(), act, v), (x.z, act.long(), v), (x.z, act[:3], v), (x.z, act, v.cpu()), (x.z[:, ::2], act, v)):
        with pytest.raises((ValueError, A.AccerlError)):
            how.forward(z, a, o, v, ref_logits=z)
    with pytest.raises(KeyError):
        A.PolicyLoss(kl="other")


def test_loss_empty_batch(A):
    e = torch.empty(0, device="cuda")
    r = A.PolicyLoss().forward(torch.empty((0, 5), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), e, e)
    assert r.grad.shape == (0, 5) and torch.all(r.stats == 0)


@pytest.mark.parametrize("B,n", [(50, 18), (3, 9001), (600, 1000)])
def test_loss_on_another_stream_and_in_a_graph(A, B, n):
    x = Inputs(B, n, "bf16", "forward", "none", seed=71)
    want = x.run(A)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    how, c = x.how, lambda t: t.cuda()
    act, old, adv, w = c(x.act), c(x.old), c(x.adv), c(x.w)
    torch.cuda.synchronize()
    got = [how.forward(x.z, act, old, adv, weights=w, scale=1.0, ref_logits=x.zr, stream=s) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(r.grad, want.grad) and torch.equal(r.stats, want.stats) for r in got)
    z = x.z.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = how.forward(z, act, old, adv, weights=w, scale=1.0, ref_logits=x.zr)
    for k in range(4):
        z.copy_(x.z * (1 + 0.1 * k))
        graph.replay()
        torch.cuda.synchronize()
        eager = how.forward(z, act, old, adv, weights=w, scale=1.0, ref_logits=x.zr)
        for name in ("loss", "logp", "kl", "entropy", "stats", "grad"):
            assert torch.equal(getattr(r, name), getattr(eager, name)), (k, name)


@pytest.mark.parametrize("B,n", [(300, 18), (300, 130), (40, 2000), (600, 5003)])
@pytest.mark.parametrize("apart", [0.3, 1e-2, 1e-3])
def test_loss_small_sampled_kl(A, B, n, apart):
    """A reference close to the policy: its KL is a small number, and keeps six digits of it."""
    x = Inputs(B, n, "f32", "sampled", "none", seed=81, spread=1.0)
    x.w[:] = 1.0
    x.act = torch.randint(0, n, (B,), dtype=torch.int32, generator=torch.Generator().manual_seed(2))
    lp = ref.softmax_rows(as64(x.z), np.ones((B, n), bool))[0][np.arange(B), x.act.numpy()]
    x.ref_lp = torch.from_numpy(lp + apart * np.random.default_rng(3).uniform(0.5, 1, B)).float()
    got = x.run(A)
    r, _ = x.want()
    d = as64(x.ref_lp) - r["logp"]
    # off by the slope exp(d) - 1 times the sum's error (terms within 2 u, exponents of at most 8: 8 u; the joins of a lane's terms), and by 8 u
    tol = np.expm1(d) * (16 * ref.U + 4 * ref.U * np.sqrt(n / 64 + 32)) + 16 * ref.U * r["kl"]
    off = np.abs(as64(got.kl) - r["kl"])
    assert (off <= tol).all(), np.max(off / tol)


@pytest.mark.parametrize("B,n", [(9, 18), (9, 400), (300, 5003), (3, 60001)])
@pytest.mark.parametrize("far", [float("-inf"), -1e9, -3e5])
def test_loss_sampled_kl_of_an_action_the_reference_forbids(A, B, n, far):
    """A reference's log-probability of -inf (which logprob gives for an action that its mask forbids), or far down: the KL is infinite or large, its slope
    1 - exp(d) is 1, and the gradient is a number."""
    x = Inputs(B, n, "f32", "sampled", "none", seed=91)
    x.w[:] = 1.0
    x.ref_lp[:] = far
    got = x.run(A)
    r, _ = x.want()
    live = (x.act.numpy() >= 0) & (x.act.numpy() < n)
    assert np.array_equal(np.isinf(as64(got.kl)), np.isinf(r["kl"])) and np.array_equal(np.isinf(as64(got.loss)), np.isinf(r["loss"]))
    assert np.isfinite(r["grad"]).all() and live.any()
    # a slope that does not depend on the sums: the tolerance is the one of a KL of 0
    t = ref.tolerances(dict(r, kl=np.zeros(B), loss=np.zeros(B)), as64(x.z), None, "f32", "sampled", as64(x.adv), x.ck, x.ch, x.scale)
    off = np.abs(as64(got.grad) - r["grad"])
    assert (off <= t["grad"]).all(), np.nanmax(off / t["grad"])


def _at_the_border(x):
    """Ratios within a few parts in 2^24 of a border, on both sides of it, for advantages of both signs."""
    B, n = len(x.act), x.z.shape[1]
    lp = ref.softmax_rows(as64(x.z), np.ones((B, n), bool))[0][np.arange(B), x.act.numpy()]
    border = np.where(np.arange(B) % 2 == 0, np.log(1.25), np.log(0.8))
    x.adv = torch.from_numpy(np.where(np.arange(B) % 4 < 2, 1.0, -1.0)).float()
    x.old = torch.from_numpy(lp - border).float()


@pytest.mark.parametrize("B,n", [(2000, 18), (2000, 400), (500, 2000)])
@pytest.mark.parametrize("kl", ["none", "forward"])
@pytest.mark.parametrize("down,up", [(0, 0), (40, 0), (85, 0), (3, 1000), (40, 20000)])
def test_loss_next_to_the_clipping_border_of_improbable_actions(A, B, n, kl, down, up):
    """What 32 bits leave of log pi(a) grows with it; where the logits lie makes no difference."""
    x = Inputs(B, n, "f32", kl, "none", seed=52)
    x.w[:] = 1.0
    x.act = torch.randint(0, n, (B,), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    x.z[torch.arange(B, device="cuda"), x.act.cuda().long()] -= down
    x.z += up
    x.zr += up
    _at_the_border(x)
    x.check(x.run(A))


@pytest.mark.parametrize("n,dtype,kl", [(5003, "f32", "none"), (5003, "f32", "forward"), (9001, "bf16", "reverse"), (33333, "bf16", "none"), (33333, "f16", "forward"),
                                        (70001, "f32", "sampled")])
@pytest.mark.parametrize("down,up,holes", [(0, 0, False), (30, 0, False), (3, 1000, False), (3, 0, True)])
def test_loss_next_to_the_clipping_border_of_long_rows(A, n, dtype, kl, down, up, holes):
    """Rows of a workgroup each; with holes of -inf they are summed the careful way."""
    B = 257
    x = Inputs(B, n, dtype, kl, "none", seed=53)
    x.w[:] = 1.0
    x.act = torch.randint(0, n // 4, (B,), dtype=torch.int32, generator=torch.Generator().manual_seed(1)) * 4
    if holes:
        x.z[:, 1::4] = float("-inf")
        x.zr[:, 1::4] = float("-inf")
    x.z[torch.arange(B, device="cuda"), x.act.cuda().long()] -= down
    x.z += up
    x.zr += up
    _at_the_border(x)
    x.ref_lp = x.old + 0.1
    x.check(x.run(A))
    kept = x.z.clone()
    got, again = x.run(A), x.run(A, grad=x.z)                                   # and in place
    assert torch.equal(got.grad, again.grad) and torch.equal(got.stats, again.stats) and not torch.equal(kept, x.z)


@pytest.mark.parametrize("B,n", [(1, 40001), (40, 40001), (3, 300001)])
@pytest.mark.parametrize("dtype,kl", [("f32", "none"), ("bf16", "forward"), ("f16", "reverse")])
@pytest.mark.parametrize("down,up", [(0, 0), (30, 0), (3, 1000)])
def test_loss_next_to_the_clipping_border_of_rows_in_pieces(A, B, n, dtype, kl, down, up):
    """With the gradient beside the logits and over them, and without one; the border is tried at several hundred distances."""
    x = Inputs(B, n, dtype, kl, "shared", seed=54)
    x.w[:] = 1.0
    x.act = torch.from_numpy(np.flatnonzero(x.mask[0].numpy())[np.random.default_rng(1).integers(0, n // 2, B)]).to(torch.int32)
    x.z[torch.arange(B, device="cuda"), x.act.cuda().long()] -= down
    x.z += up
    x.zr += up
    mask = x.mask.numpy() != 0
    lp = ref.softmax_rows(as64(x.z), np.broadcast_to(mask, (B, n)))[0][np.arange(B), x.act.numpy()]
    kept, rng = x.z.clone(), np.random.default_rng(2)
    how = A.PolicyLoss(x.lo, x.hi, kl, x.ck, x.ch)
    wide = dict(ref_logits=x.zr) if kl != "none" else {}
    outside = lambda old, adv, **k: how.forward(x.z, x.act.cuda(), old.cuda(), adv.cuda(), mask=x.mask.cuda(), scale=1.0, **wide, **k)
    for turn in range(max(4, 120 // B)):
        border = np.log(rng.choice([x.hi + 1, 1 - x.lo], B))
        old = torch.from_numpy(lp - border).float() + 0.0
        # whole steps of fp32 to either side of what is next to the border
        old = torch.from_numpy(old.numpy() + rng.integers(-3, 4, B).astype(np.float32) * np.spacing(np.abs(old.numpy())))
        adv = torch.from_numpy(rng.choice([1.0, -1.0], B)).float()
        r = np.exp(lp - as64(old))
        want = ((r < 1 - x.lo) | (r > 1 + x.hi)).sum()
        a, b = outside(old, adv), outside(old, adv, grad=False)
        assert float(a.stats[3]) == want == float(b.stats[3]), turn
        c = outside(old, adv, grad=x.z)
        assert torch.equal(a.grad, c.grad) and torch.equal(a.stats, c.stats) and torch.equal(a.loss, b.loss)
        x.z.copy_(kept)
    x.old, x.adv = old, adv
    x.check(a)


def _softmax_64(z):
    """(log p, p) of logits in 64 bits on the GPU, in elementary operations."""
    z = z.double()
    z = z - z.amax(dim=1, keepdim=True)
    e = z.exp()
    s = e.sum(dim=1, keepdim=True)
    return z - s.log(), e / s


@pytest.mark.parametrize("vectors", [2, 4, 8, 15, 20, 28, 30, 44, 48, 96, 112])
@pytest.mark.parametrize("more", [0, 1027])
@pytest.mark.parametrize("dtype,kl", [("bf16", "forward"), ("f16", "reverse"), ("f32", "none"), ("bf16", "none"), ("f32", "forward")])
@pytest.mark.parametrize("B", [300, 40])
def test_loss_long_rows_see_every_vector(A, B, vectors, more, dtype, kl):
    """Each row has most of its probability in one place, next to where a lane's vectors, registers, LDS, stream or pieces may end: the place tried moves on
    from row to row, the reference's backwards.  Whoever leaves a vector out, or takes one twice, is off by far more than 32-bit sums of 2^17 terms."""
    vec = 4 if dtype == "f32" else 8
    n = vectors * 256 * vec + more
    spots = sorted({min(max(k * 256 * vec + o, 1), n - 1) for k in range(vectors + 1) for o in (-1, 0)} | {n - 1, n - vec, n - vec - 1})
    g = torch.Generator(device="cuda").manual_seed(vectors)
    table = lambda: torch.randn((B, n), generator=g, device="cuda").to(TORCH[dtype])
    z, zr = table(), table()
    tried = [b % len(spots) if len(spots) <= B else b * len(spots) // B for b in range(B)]      # (all of them by 300 rows)
    at, at_ref = (torch.tensor([spots[i] for i in t], device="cuda") for t in (tried, [-1 - i for i in tried]))
    rows = torch.arange(B, device="cuda")
    z[rows, at] = 16.0
    zr[rows, at_ref] = 16.0
    act = torch.zeros(B, dtype=torch.int32, device="cuda")
    logp, p = _softmax_64(z)
    lp = logp[:, 0]
    old = (lp + 0.1).float()                                                    # a ratio of exp(-0.1), inside the borders
    adv = torch.where(rows % 2 == 0, 1.0, -1.0)
    out = torch.full((B, n), 9.0, dtype=TORCH[dtype], device="cuda")
    ck = 0.25 if kl != "none" else 0.0
    got = A.PolicyLoss(0.2, 0.2, kl, ck).forward(z, act, old, adv, scale=1.0, ref_logits=zr if ck else None, grad=out)
    at_grad = -(lp - old.double()).exp() * adv
    want = -at_grad[:, None] * p
    want[:, 0] += at_grad
    e, far = ref.sum_error(n), 40.0                                             # 16 + 16 and the spread of normal numbers between any two logits' differences
    size = at_grad.abs()[:, None] * p
    if ck:
        logr, pr = _softmax_64(zr)
        if kl == "forward":
            k = (pr * (logr - logp)).sum(dim=1)
            want += ck * (p - pr)
            size = size + ck * (p + pr)
        else:
            k = (p * (logp - logr)).sum(dim=1)
            want += ck * p * (logp - logr - k[:, None])
            size = size + ck * p * 2 * far
        assert ((got.kl.double() - k).abs() <= 2 * e * (1 + far + np.log(n))).all()
    size[:, 0] += at_grad.abs()
    assert ((got.logp.double() - lp).abs() <= e + 4 * ref.U * (lp.abs() + 1)).all()
    off = (got.grad.double() - want).abs()
    tol = size * (4 * e + 64 * ref.U) + ref.HALF_STEP[dtype] * want.abs() * 1.001 + ref.TINY[dtype]
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("B,n", [(300, 17), (300, 2000), (300, 5003), (300, 20001), (300, 60001), (300, 260001), (40, 60001), (3, 1 << 20)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["two", "one", "rising"])
def test_loss_next_to_the_clipping_border_whatever_the_roundings(A, B, n, dtype, shape):
    """Rows whose sums are off by roundings that all go one way: of two logits only, of one large logit and many equal small ones, of logits that
    rise.  The side is the one that a sum in 64 bits gives."""
    rng = np.random.default_rng(n)
    place = torch.arange(n, device="cuda")[None]
    column = lambda v: torch.from_numpy(v).cuda()[:, None]
    if shape == "two":
        z = torch.where(place < column(rng.integers(1, n, B)), 0.0, column(-rng.uniform(0.1, 6.0, B)))
    elif shape == "one":
        z = torch.where(place == column(rng.integers(0, n, B)), 0.0, column(-rng.uniform(0.5, 1.5, B) * np.log(n) - rng.uniform(0, 4, B)))
    else:
        z = (place / n - 0.5) * column(rng.uniform(0.01, 20.0, B))
    z = z.to(TORCH[dtype])
    act = torch.from_numpy(np.where(rng.random(B) < 0.5, 0, n - 1)).to(torch.int32)
    lp = np.array([float(_softmax_64(z[b:b + 1])[0][0, int(act[b])]) for b in range(B)])
    for turn in range(6):
        up = rng.random(B) < 0.5
        old = (lp - np.where(up, np.log(1.25), np.log(0.8))).astype(np.float32)
        old += rng.integers(-2, 3, B).astype(np.float32) * np.spacing(np.abs(old))
        adv = np.where(rng.random(B) < 0.5, 1.0, -1.0).astype(np.float32)
        r = np.exp(lp - old.astype(np.float64))
        assert (np.abs(r / np.where(up, 1.25, 0.8) - 1) > 1e-13).all()          # (the definition itself tells the sides apart)
        cut = np.where(adv > 0, r > 1.25, r < 0.8)
        got = A.PolicyLoss(0.2, 0.25).forward(z, act.cuda(), torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda(), scale=1.0)
        wrong = np.flatnonzero((got.grad == 0).all(dim=1).cpu().numpy() != cut)
        assert wrong.size == 0, (turn, wrong[:5], (r / np.where(up, 1.25, 0.8) - 1)[wrong[:5]])
        assert float(got.stats[3]) == ((r > 1.25) | (r < 0.8)).sum(), turn
