"""LinearAttention and BlockNorm as owners: threads, streams, captured graphs, devices; and the two together, actor and learner."""
import pytest
import torch

from tests.test_gpu_wide_owners import _replays, _threads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def _attention(T, H=2, Dk=64, Dv=64, B=2, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    return dict(q=n(B, T, H, Dk), k=n(B, T, H, Dk), v=n(B, T, H, Dv)), n(B, T, H, Dv), torch.randn((B, H, Dk, Dv), generator=g, device="cuda")


# (of 1000 tokens: in segments, whose states lie in the workspace)
CALLS = ["unroll", "gradient", "step", "norm", "norm gradient"]


def _call(A, kind, seed=0, owner={}):
    """(owner's call, its inputs) of one kind; one owner for all."""
    if kind in ("norm", "norm gradient"):
        o = owner.setdefault("norm", A.BlockNorm(300, after=torch.ones(300), before=torch.linspace(0, 1, 300), gate="silu"))
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = [torch.randn((2000, 300), generator=g, device="cuda") for _ in range(5)]
        if kind == "norm":
            return lambda **k: list(o.forward(t[0], x=t[1], gate=t[2], **k))

        def back(**k):
            r = o.backward(t[0], x=t[1], gate=t[2], grad_u=t[3], grad_h=t[4], **k)
            return [r.y, r.x, r.gate, r.after, r.before]
        return back
    o = owner.setdefault("attention", A.LinearAttention([0.9, 0.99], scale=0.1))
    x, go, state = _attention(1000, seed=seed)
    if kind == "unroll":
        return lambda **k: list(o.forward(**x, state=state, **k))
    if kind == "step":
        beside = torch.empty_like(state)
        return lambda **k: [o.step(*(x[n][:, 0] for n in "qkv"), state, out_state=beside, **k)]

    def back(**k):
        r = o.backward(go, **x, state=state, grad_state=state, **k)
        return [r.q, r.k, r.v, r.state]
    return back


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("kind", CALLS)
def test_two_threads_share_an_owner(A, kind):
    calls = [_call(A, kind, seed=i) for i in range(2)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    got = _threads(lambda i: [calls[i]() for _ in range(50)])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(_same(r, want[i]) for r in got[i]), i


@pytest.mark.parametrize("kind", CALLS)
def test_streams(A, kind):
    """The current one, one handed in, one by its number: a call waits for what its stream has."""
    call = _call(A, kind)
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [call(stream=s), call(stream=s.cuda_stream)]
    with torch.cuda.stream(s):
        got.append(call())
    s.synchronize()
    assert all(_same(g, want) for g in got)


@pytest.mark.parametrize("kind", CALLS)
def test_two_graphs_of_one_owner(A, kind):
    """Captured one after the other, replayed on two streams at once, with eager calls between: no workspace is shared."""
    calls = [_call(A, kind, seed=i) for i in range(2)]
    want = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], [None, None]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            outs[i] = calls[i]()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for i in range(2):
            for o in outs[i]:
                o.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        calls[0]()
        torch.cuda.synchronize()
        for i in range(2):
            assert _same(outs[i], want[i]), i


@pytest.mark.parametrize("kind", CALLS)
def test_a_graph_replayed_on_new_inputs(A, kind):
    """What lies in the captured tensors then is what a replay works on."""
    call = _call(A, kind)
    call()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        want = [t.clone() for t in call()]
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = call()
        _replays([graph], out, want)


def test_what_is_given_in_autograd_is_taken_as_it_is(A):
    """Leaves that require gradients: values and gradients are the same, nothing is recorded, and the gradients continue into what made the tokens."""
    x, go, state = _attention(70, dtype=torch.float32)
    at = A.LinearAttention([0.9, 0.99])
    want, last = at.forward(**x, state=state)
    r = at.backward(go, **x, state=state)
    leaf = torch.randn((2, 70, 32), device="cuda", requires_grad=True)
    w = torch.randn((32, 2 * 64), device="cuda", requires_grad=True)
    q = (leaf @ w).unflatten(-1, (2, 64))
    out, _ = at.forward(q, x["k"], x["v"], state=state)
    assert not out.requires_grad
    g = at.backward(go, q, x["k"], x["v"], state=state)
    torch.autograd.backward([q], [g.q])
    assert torch.allclose(w.grad, leaf.detach().flatten(0, 1).t() @ g.q.flatten(0, 1).flatten(1), rtol=1e-4, atol=1e-3)
    y = {n: t.clone().requires_grad_() for n, t in x.items()}
    again, last2 = at.forward(**y, state=state)
    assert torch.equal(again, want) and torch.equal(last2, last) and torch.equal(at.backward(go, **y, state=state).q, r.q)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_outputs_lie_where_the_inputs_do(A):
    with torch.cuda.device(1):
        call = _call(A, "unroll", owner={})
        want = call()
    assert all(t.device.index == 1 for t in call()) and _same(call(), want)


def test_other_owners_tensors_are_refused(A):
    at = A.LinearAttention([0.9, 0.99])
    x, go, state = _attention(10)
    with pytest.raises(ValueError):
        at.forward(x["q"][:, :, :1], x["k"], x["v"])
    with pytest.raises(ValueError):
        at.forward(x["q"], x["k"].float(), x["v"])
    with pytest.raises(ValueError):
        at.forward(**x, state=state[:1])
    with pytest.raises(ValueError):
        at.forward(**x, reset=torch.zeros((2, 10), dtype=torch.bool, device="cuda"))
    with pytest.raises(ValueError):
        at.forward(**x, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises((ValueError, A.AccerlError)):
        at.step(*(x[n][:, 0] for n in "qkv"), None)
    with pytest.raises((ValueError, A.AccerlError)):
        at.forward(**x, out=x["v"])
    with pytest.raises((ValueError, A.AccerlError)):
        at.forward(x["q"].cpu(), x["k"].cpu(), x["v"].cpu())
    norm = A.BlockNorm(64, after=torch.ones(64), gate="silu")
    y = torch.randn((4, 64), device="cuda")
    for bad in (dict(y=y[:, :60]), dict(y=y), dict(y=y, gate=y[:2]), dict(y=y, gate=y.half()), dict(y=y, x=y.half(), gate=y)):
        with pytest.raises((ValueError, A.AccerlError)):
            norm.forward(**bad)
    with pytest.raises(ValueError):
        norm.backward(y, gate=y, grad_u=y, grad_h=y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_block_as_it_is_used(A, dtype):
    """Projections, memory, heads normed and gated, projection, end of the block: the actor step by step, the learner at once, and its gradients against autograd's
    of the same block in 64 bits."""
    B, T, H, D, W = 3, 50, 4, 32, 96
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    wide = dict(x=n(B, T, W), wqkv=n(W, 3 * H * D) / W ** 0.5, wg=n(W, H * D) / W ** 0.5, wo=n(H * D, W) / (H * D) ** 0.5, heads=1 + 0.1 * n(H * D), after=1 + 0.1 * n(W),
                before=1 + 0.1 * n(W), state=n(B, H, D, D))
    reset = (torch.rand((B, T), generator=g, device="cuda") < 0.05).to(torch.uint8)
    decay = [0.8, 0.9, 0.95, 0.99]
    low = {k: wide[k].to(dtype) for k in ("x", "wqkv", "wg", "wo")}
    at = A.LinearAttention(decay, scale=D ** -0.5)
    heads = A.BlockNorm(H * D, after=wide["heads"], gate="silu", groups=H)
    end = A.BlockNorm(W, after=wide["after"], before=wide["before"], branch=0.5)

    def project(x):
        q, k, v = (x @ low["wqkv"]).split(H * D, dim=-1)
        return [t.unflatten(-1, (H, D)) for t in (q, k, v)], x @ low["wg"]
    # the learner
    (q, k, v), gate = project(low["x"])
    o, last = at.forward(q, k, v, state=wide["state"], reset=reset)
    flat = lambda t: t.reshape(B * T, -1)
    m, _ = heads.forward(flat(o), gate=flat(gate))
    y = m @ low["wo"]
    stream = flat(wide["x"])
    u, h = end.forward(y, x=stream)
    # the actor
    state = wide["state"].clone()
    for t in range(T):
        (qt, kt, vt), gt = project(low["x"][:, t])
        ot = at.step(qt, kt, vt, state, reset=reset[:, t])
        ut, ht = end.forward(heads.forward(ot.reshape(B, -1), gate=gt)[0] @ low["wo"], x=wide["x"][:, t])
        near = 2e-4 if dtype == torch.float32 else 6e-2      # (bf16: half a step is 2^-8 of values of a few units, through a handful of layers on either side)
        assert (ht.float() - h.view(B, T, W)[:, t].float()).abs().max() <= near and (ut - u.view(B, T, W)[:, t]).abs().max() <= near, t
    assert (state - last).abs().max() <= (1e-4 if dtype == torch.float32 else 1e-1)
    # its gradients
    gu, gh, gl = n(B * T, W), n(B * T, W).to(h.dtype), 0.1 * n(B, H, D, D)
    r_end = end.backward(y, x=stream, grad_u=gu, grad_h=gh)
    r_heads = heads.backward(flat(o), gate=flat(gate), grad_u=r_end.y @ low["wo"].t().contiguous())
    r = at.backward(r_heads.y.view(B, T, H, D), q, k, v, state=wide["state"], reset=reset, grad_state=gl)
    got = dict(x=r_end.x, after=r_end.after, before=r_end.before, heads=r_heads.after, gate=r_heads.gate, q=r.q, k=r.k, v=r.v, state=r.state, wo=m.t().contiguous() @ r_end.y)
    leaf = {k: t.detach().double().requires_grad_() for k, t in dict(q=q, k=k, v=v, gate=flat(gate), state=wide["state"], heads=wide["heads"], after=wide["after"], before=wide["before"],
                                                                     wo=low["wo"], x=stream).items()}
    rms = lambda z, parts: torch.nn.functional.rms_norm(z.unflatten(-1, (parts, -1)), (z.shape[-1] // parts,), eps=1e-6).flatten(-2)
    s, os = leaf["state"], []
    d = torch.tensor(decay, dtype=torch.float64, device="cuda").view(1, H, 1, 1)
    for t in range(T):
        s = torch.where(reset[:, t].view(B, 1, 1, 1) != 0, 0.0, s) * d + leaf["k"][:, t][..., None] * leaf["v"][:, t][..., None, :]
        os.append((leaf["q"][:, t][..., None] * s).sum(-2) * D ** -0.5)
    mm = rms(flat(torch.stack(os, dim=1)), H) * leaf["heads"] * torch.nn.functional.silu(leaf["gate"])
    uu = leaf["x"] + 0.5 * rms(mm @ leaf["wo"], 1) * leaf["after"]
    hh = rms(uu, 1) * leaf["before"]
    torch.autograd.backward([uu, hh, s], [gu.double(), gh.double(), gl.double()])
    # 2-norms: a handful of layers of roundings of half a step each, in whatever direction
    most = 3e-5 if dtype == torch.float32 else 2e-2
    for k, t in got.items():
        e = leaf[k].grad
        assert (t.double().reshape(e.shape) - e).norm() <= most * e.norm(), k
