"""The operators of policies with a memory at sizes and in uses beyond the other tests': rows that a slot has several of, sums of wide columns, graphs replayed on other
inputs, no tokens of shared heads, and how far bf16 results are off on the whole."""
import numpy as np
import pytest
import torch

from tests import memory_reference as ref
from tests import test_gpu_block_norm as norms
from tests.test_gpu_linear_attention import DT, check, decays, make, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ragged", [False, True])
def test_no_tokens_of_shared_heads(A, dtype, ragged):
    """T = 0: the state and its gradient pass through."""
    a = make(2, 0, 4, 2, 33, 20, dtype)
    lengths = torch.tensor([0, 3], dtype=torch.int32, device="cuda") if ragged else None
    at = A.LinearAttention(decays(4))
    out, last = at.forward(a["q"], a["k"], a["v"], state=a["state"], lengths=lengths)
    assert out.shape == (2, 0, 4, 20) and torch.equal(last, a["state"])
    gs = torch.randn_like(last)
    r = at.backward(out, a["q"], a["k"], a["v"], state=a["state"], lengths=lengths, grad_state=gs)
    assert r.q.shape == a["q"].shape and r.k.shape == a["k"].shape and r.v.shape == a["v"].shape and torch.equal(r.state, gs)


# ------------------------------------------------------------------ norms
def _slots(A, N, D, groups):
    """Rows (of a group) that the gradients work on at a time: the workspace has two records of D floats for each workgroup that works on rows of its own, or for
    each group of it."""
    d = D // groups
    records = A.accerl_block_norm_workspace(N, D, groups) // (8 * d)
    lanes = 1
    while lanes * 8 < d:
        lanes *= 2
    rows = 256 // lanes if d <= 512 else 1                       # of a workgroup
    return records // groups * rows if rows % groups == 0 else records


@pytest.mark.parametrize("dtype,stream", norms.TYPES)
@pytest.mark.parametrize("N,D,groups", [(70001, 40, 1), (250001, 6, 1), (30011, 100, 5), (5000, 1300, 1), (3001, 600, 1), (1100, 2048, 1), (1101, 3000, 5), (700, 9000, 1), (600, 16384, 1),
                                        (4200, 1026, 1)])
def test_slots_of_several_rows(A, dtype, stream, N, D, groups):
    """A slot goes from row to row: pointers that move on, the next row's loads under way, sums of weights over several rows."""
    before = groups == 1
    assert N * groups > _slots(A, N, D, groups)
    if D in (40, 1300, 1026):                                   # and forwards: 256 compute units hold 2048 lanes each, and these rows have 8 or 128 lanes
        assert N > 256 * 2048 // (8 if D == 40 else 128)
    a, w, flow = norms.make(N, D, dtype, stream, ld=5, before=before)
    if groups > 1:
        a["x"], stream = None, dtype
        flow["grad_u"] = flow["grad_u"].to(DT[dtype])
    norm, u, h, r = norms.run(A, a, w, flow, "layer", "silu", dtype, stream, groups=groups)
    again = norm.backward(**a, **flow)
    assert all(getattr(r, n) is None or torch.equal(getattr(r, n), getattr(again, n)) for n in ("y", "x", "gate", "after", "before"))


# ------------------------------------------------------------------ linear attention
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", [(128, 128), (256, 128), (200, 100), (250, 70)])
def test_sums_of_wide_columns_of_all_depths(A, dtype, Dk, Dv):
    """16384 tokens of 16 heads, whose segments' sums take 128 columns a workgroup: two heads against the recurrence in 64 bits."""
    T, H = 16384, 16
    a = make(1, T, H, H, Dk, Dv, dtype, resets=0.0005)
    decay = [0.9] + [0.99] * (H - 2) + [0.9995]
    out, last = A.LinearAttention(decay, scale=0.1).forward(a["q"], a["k"], a["v"], state=a["state"], reset=a["reset"])
    heads = [0, H - 1]
    d = torch.tensor([decay[h] for h in heads], dtype=torch.float64, device="cuda").view(1, 2, 1, 1)
    q, k, v = (a[n][0][:, heads].double() for n in "qkv")
    sides = torch.stack([a["state"][0, heads].double(), a["state"][0, heads].double().abs()])
    qs, ks, vs = (torch.stack([t, t.abs()], dim=1) for t in (q, k, v))
    outs, cut = [], a["reset"][0].tolist()
    for t in range(T):
        if cut[t]:
            sides.zero_()
        sides = sides * d + ks[t][..., None] * vs[t][..., None, :]
        outs.append((qs[t][..., None] * sides).sum(-2) * 0.1)
    o, s = torch.stack(outs).cpu().numpy(), sides.cpu().numpy()
    d = np.array([decay[h] for h in heads])
    check("out", out[0][:, heads], o[:, 0], ref.unroll_tolerance(o[:, 0][None], o[:, 1][None], dtype, T, max(Dk, Dv), d)[0])
    check("state", last[0, heads], s[0], ref.unroll_tolerance(s[:1], s[1:], dtype, T, max(Dk, Dv), d, state=True)[0])


@pytest.mark.parametrize("wanted", [True, False])
@pytest.mark.parametrize("T", [512, 1024])
def test_how_far_bf16_outputs_are_off_on_the_whole(A, wanted, T):
    """Two roundings to bf16 lie between a term and the result: of the weight of a pair or of the state's copy, and of the output.  Each is uniform within its step, so
    2^-7 / sqrt(12) of the power of two below, whose mean square is at most 0.6 of the values' own (0.54 for values of any size alike); errors of terms add up as the
    terms do, at random.  Long memories: nearly all of an output comes from the state, and one more rounding there, of keys or values, would show (sqrt(3/2))."""
    B, H, D = 2, 4, 64
    a = make(B, T, H, H, D, D, "bf16")
    decay = [1 - 2.0 ** -(9 + i) for i in range(H)]
    out = torch.empty_like(a["v"])
    at = A.LinearAttention(decay)
    need = A.accerl_linear_attention_workspace(B, T, H, H, D, D)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    A.accerl_linear_attention(a["q"], a["k"], a["v"], at.log_decay, out, ws, scale=0.125, state=a["state"], out_state=torch.empty_like(a["state"]) if wanted else None)
    o, _ = ref.unroll(*(wide(a[n]) for n in "qkv"), np.array(decay), 0.125, state=wide(a["state"]))
    off = np.linalg.norm(wide(out) - o) / np.linalg.norm(o)
    assert off <= (2 * 0.6) ** 0.5 * 2.0 ** -7 / 12 ** 0.5, off


# ------------------------------------------------------------------ graphs
def _call(A, kind):
    """(the call, the tensors it reads)"""
    n = lambda *s: torch.randn(s, device="cuda")
    if kind.startswith("norm"):
        o = A.BlockNorm(300, after=torch.linspace(0.5, 1, 300), before=torch.linspace(0, 1, 300), gate="silu")
        t = [n(3000, 300) for _ in range(5)]
        if kind == "norm":
            return lambda: list(o.forward(t[0], x=t[1], gate=t[2])), t[:3]

        def back():
            r = o.backward(t[0], x=t[1], gate=t[2], grad_u=t[3], grad_h=t[4])
            return [r.y, r.x, r.gate, r.after, r.before]
        return back, t
    H, Hk, D, T = 4, 2, 64, 1000                                 # (in segments, heads shared: states and parts of gradients lie in the workspace)
    o = A.LinearAttention([0.9, 0.99, 0.5, 1.0], scale=0.1)
    if kind == "step":
        q, k, v, state, reset = n(2, H, D).bfloat16(), n(2, Hk, D).bfloat16(), n(2, Hk, D).bfloat16(), n(2, H, D, D), torch.zeros(2, dtype=torch.uint8, device="cuda")
        beside = torch.empty_like(state)
        return lambda: [o.step(q, k, v, state, reset=reset, out_state=beside), beside], [q, k, v, state, reset]
    q, k, v, state = n(2, T, H, D).bfloat16(), n(2, T, Hk, D).bfloat16(), n(2, T, Hk, D).bfloat16(), n(2, H, D, D)
    reset, lengths = torch.zeros((2, T), dtype=torch.uint8, device="cuda"), torch.full((2,), T, dtype=torch.int32, device="cuda")
    if kind == "unroll":
        return lambda: list(o.forward(q, k, v, state=state, reset=reset, lengths=lengths)), [q, k, v, state, reset, lengths]
    go, gs = n(2, T, H, D).bfloat16(), n(2, H, D, D)

    def back():
        r = o.backward(go, q, k, v, state=state, reset=reset, lengths=lengths, grad_state=gs)
        return [r.q, r.k, r.v, r.state]
    return back, [q, k, v, state, reset, lengths, go, gs]


@pytest.mark.parametrize("kind", ["unroll", "gradient", "step", "norm", "norm gradient"])
def test_a_replay_works_on_what_lies_in_the_tensors_then(A, kind):
    call, inputs = _call(A, kind)
    first = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for i in range(3):
        for t in inputs:
            if t.dtype == torch.uint8:
                t.copy_(torch.rand(t.shape, device="cuda") < 0.01 * (i + 1))
            elif t.dtype == torch.int32:
                t.copy_(torch.tensor([977 - 300 * i, 1000], device="cuda"))
            else:
                t.normal_()
        want = [t.clone() for t in call()]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)) and not torch.equal(want[0], first[0]), i
