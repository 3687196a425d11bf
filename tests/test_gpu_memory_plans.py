"""LinearAttention and BlockNorm where sizes choose another way to the same result: segments, wide sums, launches that roles share, states past the caches, offsets past
32 bits."""
import numpy as np
import pytest
import torch

from tests import memory_reference as ref
from tests.test_gpu_linear_attention import DT, check, decays, make, run, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [(1, 600, 1, 1, 256, 256), (1, 513, 2, 1, 7, 5), (1, 577, 2, 2, 5, 200), (2, 640, 2, 1, 128, 64), (1, 1025, 1, 1, 65, 129), (3, 530, 1, 1, 100, 1)])
def test_segments_of_heads_of_all_sizes(A, dtype, B, T, H, Hk, Dk, Dv):
    run(A, make(B, T, H, Hk, Dk, Dv, dtype, resets=0.004, ragged=B > 1), decays(H), 0.2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Dk,Dv", [(6, 100, 8, 48, 72), (2, 100, 8, 48, 72), (3, 70, 4, 130, 20), (16, 70, 8, 130, 20)])
def test_gradients_of_two_widths(A, dtype, B, T, H, Dk, Dv):
    """Few of them in one launch, more in two."""
    run(A, make(B, T, H, H, Dk, Dv, dtype, resets=0.01), decays(H), 0.2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["plain", "rows"])
def test_segments_of_rows_of_a_table(A, dtype, layout):
    run(A, make(2, 700, 2, 1, 48, 40, dtype, resets=0.004, ragged=True, layout=layout), decays(2, "mixed"), 0.2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["q", "k", "v", "state"])
def test_what_is_not_finite_in_segments(A, dtype, what, which):
    """It stays with its episode, head and column, across the segments' borders and in the gradients."""
    B, T, H, Hk = 2, 700, 4, 2
    a = make(B, T, H, Hk, 48, 72, dtype)
    reset = torch.zeros((B, T), dtype=torch.uint8, device="cuda")
    reset[:, 500] = 1
    a["reset"] = reset
    if which == "state":
        a["state"][0, 1, 5, 3] = what
    else:
        a[which][0, 333, 1, 5] = what
    d = np.array(decays(H))
    at = A.LinearAttention(decays(H), scale=0.125)
    go = torch.ones((B, T, H, 72), dtype=DT[dtype], device="cuda")
    out, last = at.forward(a["q"], a["k"], a["v"], state=a["state"], reset=reset)
    r = at.backward(go, a["q"], a["k"], a["v"], state=a["state"], reset=reset)
    w = {n: wide(a[n]) for n in "qkv"}
    arg = dict(reset=wide(reset), state=wide(a["state"]))
    clean = lambda x: np.nan_to_num(np.abs(x), nan=0, posinf=0, neginf=0)
    with np.errstate(invalid="ignore"):
        o, s = ref.unroll(w["q"], w["k"], w["v"], d, 0.125, **arg)
        g = ref.unroll_grad(wide(go), w["q"], w["k"], w["v"], d, 0.125, **arg)
    sizes = dict(reset=wide(reset), state=clean(arg["state"]))
    oa, sa = ref.unroll(*(clean(w[n]) for n in "qkv"), d, 0.125, **sizes)
    ga = ref.unroll_grad(wide(go), *(clean(w[n]) for n in "qkv"), d, 0.125, **sizes)
    for name, got, want, mags, state in (("out", out, o, oa, False), ("state", last, s, sa, True), ("grad q", r.q, g["q"], ga["q"], False), ("grad k", r.k, g["k"], ga["k"], False),
                                         ("grad v", r.v, g["v"], ga["v"], False), ("grad state", r.state, g["state"], ga["state"], True)):
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(wide(got)), fine), name
        tol = ref.unroll_tolerance(np.where(fine, want, 0), mags, dtype, T, 72, decays(H), state=state)
        check(name, got[torch.from_numpy(fine).cuda()], want[fine], np.broadcast_to(tol, want.shape)[fine])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_sums_of_wide_columns(A, dtype):
    """16384 tokens of 16 heads: two of them against the recurrence in 64 bits."""
    T, H, Dk, Dv = 16384, 16, 100, 120
    a = make(1, T, H, H, Dk, Dv, dtype, resets=0.0005)
    decay = [0.9] + [0.99] * (H - 2) + [0.9995]
    out, last = A.LinearAttention(decay, scale=0.1).forward(a["q"], a["k"], a["v"], state=a["state"], reset=a["reset"])
    heads = [0, H - 1]
    d = torch.tensor([decay[h] for h in heads], dtype=torch.float64, device="cuda").view(1, 2, 1, 1)
    q, k, v = (a[n][0][:, heads].double() for n in "qkv")
    sides = torch.stack([a["state"][0, heads].double(), a["state"][0, heads].double().abs()])          # the state, and the sizes of what it sums
    qs, ks, vs = (torch.stack([t, t.abs()], dim=1) for t in (q, k, v))                             # [T, 2, heads, D]
    outs, cut = [], a["reset"][0].tolist()
    for t in range(T):
        if cut[t]:
            sides.zero_()
        sides = sides * d + ks[t][..., None] * vs[t][..., None, :]
        outs.append((qs[t][..., None] * sides).sum(-2) * 0.1)
    o = torch.stack(outs).cpu().numpy()
    s = sides.cpu().numpy()
    d = np.array([decay[h] for h in heads])
    check("out", out[0][:, heads], o[:, 0], ref.unroll_tolerance(o[:, 0][None], o[:, 1][None], dtype, T, 120, d)[0])
    check("state", last[0, heads], s[0], ref.unroll_tolerance(s[:1], s[1:], dtype, T, 120, d, state=True)[0])


@pytest.mark.parametrize("Dk,Dv", [(256, 256), (250, 250)])
def test_a_step_past_the_caches(A, Dk, Dv):
    """More states than the caches hold: the same bits as in parts."""
    H, B = 4, 300
    g = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, v, state = n(B, H, Dk).bfloat16(), n(B, H, Dk).bfloat16(), n(B, H, Dv).bfloat16(), n(B, H, Dk, Dv)
    assert state.numel() * 4 > 256 << 20
    at = A.LinearAttention(decays(H))
    beside = torch.empty_like(state)
    out = at.step(q, k, v, state, out_state=beside)
    for part in (slice(0, 100), slice(100, 300)):
        s = state[part].clone()
        assert torch.equal(at.step(q[part], k[part], v[part], s), out[part]) and torch.equal(s, beside[part])
    again = at.step(q, k, v, state)
    assert torch.equal(again, out) and torch.equal(state, beside)


def test_states_past_32_bits(A):
    B, H, D = 8200, 4, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v = (torch.randn((B, H, D), generator=g, device="cuda").bfloat16() for _ in range(3))
    state = torch.zeros((B, H, D, D), device="cuda")
    assert state.numel() > 1 << 31
    state[-2:].normal_(generator=g)
    tail = state[-2:].clone()
    at = A.LinearAttention(decays(H))
    x = lambda t: t[:, None]
    out, last = at.forward(x(q), x(k), x(v), state=state)
    o, s = at.forward(x(q)[-2:], x(k)[-2:], x(v)[-2:], state=tail)
    assert torch.equal(out[-2:], o) and torch.equal(last[-2:], s)
    del last
    out = at.step(q, k, v, state)
    want = at.step(q[-2:], k[-2:], v[-2:], tail)
    assert torch.equal(out[-2:], want) and torch.equal(state[-2:], tail)


@pytest.mark.parametrize("T", [40, 600])
def test_tokens_past_32_bits(A, T):
    """Tokens so far apart that their offsets need more than 32 bits."""
    far = (1 << 31) // (T - 1) + 64
    a = make(1, T, 2, 2, 48, 40, "bf16")
    at = A.LinearAttention(decays(2))
    go = torch.randn((1, T, 2, 40), device="cuda").bfloat16()
    want, ws = at.forward(a["q"], a["k"], a["v"], state=a["state"])
    wr = at.backward(go, a["q"], a["k"], a["v"], state=a["state"])
    table = torch.empty((T, far), dtype=torch.bfloat16, device="cuda")
    assert table.stride(0) * (T - 1) >= 1 << 31

    def spread(t, to):
        x = table[None, :, to:to + t.shape[2] * t.shape[3]].unflatten(-1, t.shape[2:])
        x.copy_(t)
        return x
    q, k, v, g = spread(a["q"], 0), spread(a["k"], 100), spread(a["v"], 200), spread(go, 300)
    out, last = at.forward(q, k, v, state=a["state"], out=spread(torch.zeros_like(go), 400))
    r = at.backward(g, q, k, v, state=a["state"])
    assert torch.equal(out, want) and torch.equal(last, ws) and all(torch.equal(getattr(r, n), getattr(wr, n)) for n in "qkv") and torch.equal(r.state, wr.state)


def test_rows_past_32_bits(A):
    R, D = 50, 300
    far = (1 << 31) // (R - 1) + 64
    norm = A.BlockNorm(D, after=torch.linspace(0.5, 1, D), before=torch.ones(D), gate="silu")
    y, x, gate, gu, gh = (torch.randn((R, D), device="cuda").bfloat16() for _ in range(5))
    want = norm.forward(y, x=x, gate=gate)
    wr = norm.backward(y, x=x, gate=gate, grad_u=gu, grad_h=gh)
    table = torch.empty((R, far), dtype=torch.bfloat16, device="cuda")

    def spread(t, to):
        z = table[:, to:to + D]
        z.copy_(t)
        return z
    y, x, gate, gu, gh = (spread(t, 1000 * i) for i, t in enumerate((y, x, gate, gu, gh)))
    got = norm.forward(y, x=x, gate=gate)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    r = norm.backward(y, x=x, gate=gate, grad_u=gu, grad_h=gh)
    assert all(torch.equal(getattr(r, n), getattr(wr, n)) for n in ("y", "x", "gate", "after", "before"))


@pytest.mark.parametrize("D", [9, 20, 300, 515, 1030, 2050, 3001, 9000])
@pytest.mark.parametrize("where", ["gate", "after"])
def test_an_infinity_near_a_rows_end(A, D, where):
    """As anywhere else in the row: the norm that follows makes zeros of the others and NaN of it, and the rows beside it are as they were."""
    R = 6
    y, gate = torch.rand((R, D), device="cuda") + 0.5, torch.rand((R, D), device="cuda") + 0.5
    after = torch.ones(D)
    clean = A.BlockNorm(D, after=after, before=torch.ones(D), gate="silu").forward(y, gate=gate)
    for back in range(1, 10):
        if where == "gate":
            g, a, rows = gate.clone(), after, slice(2, 3)
            g[2, D - back] = float("inf")
        else:
            g, a, rows = gate, after.clone(), slice(0, R)
            a[D - back] = float("inf")
        u, h = A.BlockNorm(D, after=a, before=torch.ones(D), gate="silu").forward(y, gate=g)
        there = torch.zeros((R, D), dtype=torch.bool, device="cuda")
        there[rows, D - back] = True
        beside = torch.zeros((R, D), dtype=torch.bool, device="cuda")
        beside[rows] = True
        assert torch.isinf(u[there]).all() and torch.equal(u[~there], clean[0][~there]), back
        assert torch.isnan(h[there]).all() and (h[beside & ~there] == 0).all() and torch.equal(h[~beside], clean[1][~beside]), back


@pytest.mark.parametrize("D,groups", [(600, 1), (1024, 1), (1201, 1), (2048, 1), (3000, 1), (3000, 5), (2048, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norms_of_few_and_many_rows(A, D, groups, dtype):
    """A row's result does not depend on how many there are: sums of up to 3000 terms in other orders, 3000 2^-24 apart before the root, and a rounding to the type."""
    R = 1100
    g = torch.Generator(device="cuda").manual_seed(D)
    y, gate, x = (torch.randn((R, D), generator=g, device="cuda").to(t) for t in (dtype, dtype, torch.float32))
    norm = A.BlockNorm(D, after=torch.linspace(0.5, 1.5, D), before=torch.ones(D) if groups == 1 else None, gate="silu", groups=groups, kind="layer")
    u, h = norm.forward(y, x=x, gate=gate)
    for rows in (slice(0, 1), slice(5, 70), slice(76, R)):
        us, hs = norm.forward(y[rows], x=x[rows], gate=gate[rows])
        assert torch.allclose(us, u[rows], rtol=2e-4, atol=2e-4)
        if groups == 1:
            step = 2e-4 + (0 if dtype == torch.float32 else 2.0 ** -7)
            assert torch.allclose(hs.float(), h[rows].float(), rtol=step, atol=2e-4)
    want = x.double() + torch.nn.functional.layer_norm(y.double().view(R, groups, -1), (D // groups,), eps=1e-6).view(R, D) * norm.after.double() * torch.nn.functional.silu(gate.double())
    assert torch.allclose(u.double(), want, rtol=2e-4, atol=2e-4)
