"""The norms around a block, with its gate and its residual, against the 64-bit formulas: values and gradients."""
import numpy as np
import pytest
import torch

from tests import memory_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def check(name, got, want, tol):
    got = wide(got)
    assert got.shape == want.shape, name
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], np.broadcast_to(tol, want.shape)[bad][:5])


def table(g, N, D, dtype, ld=0, scale=1.0):
    t = torch.empty((N, D + ld), dtype=DT[dtype], device="cuda").fill_(float("nan"))
    t[:, :D] = scale * torch.randn((N, D), generator=g, device="cuda")
    return t[:, :D]


def make(N, D, dtype, stream, ld=0, x=True, gate="sigmoid", after=True, before=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * N + D)
    a = dict(y=table(g, N, D, dtype, ld), x=table(g, N, D, stream, 2 * ld, 2.0) if x else None, gate=table(g, N, D, dtype, ld) if gate else None)
    w = dict(after=1 + 0.3 * torch.randn(D, generator=g, device="cuda") if after else None, before=1 + 0.3 * torch.randn(D, generator=g, device="cuda") if before else None)
    return a, w, dict(grad_u=table(g, N, D, stream, ld), grad_h=table(g, N, D, dtype, 3 * ld) if before else None)


def run(A, a, w, flow, kind, gate, dtype, stream, groups=1, eps=1e-6, skip=0.9, branch=0.4):
    N, D = a["y"].shape
    norm = A.BlockNorm(D, **w, kind=kind, gate=gate, groups=groups, eps=eps, skip=skip, branch=branch)
    how = dict(after=wide(w["after"]), before=wide(w["before"]), kind=kind, gate_kind=gate, groups=groups, eps=eps, skip=skip, branch=branch)
    want, size = ref.block_norm(*(wide(a[n]) for n in ("y", "x", "gate")), **how)
    u, h = norm.forward(**a)
    stored = stream if a["x"] is not None else dtype
    assert u.dtype == DT[stored] and (h is None) == (w["before"] is None) and (h is None or h.dtype == DT[dtype])
    tol = lambda n, t, rows=1: ref.norm_tolerance(want[n], size[n], t, D, rows)
    check("u", u, want["u"], tol("u", stored))
    if h is not None:
        check("h", h, want["h"], tol("h", dtype))
    want, size = ref.block_norm(*(wide(a[n]) for n in ("y", "x", "gate")), **how, gu=wide(flow["grad_u"]), gh=wide(flow["grad_h"]))
    r = norm.backward(**a, **flow)
    for n, t in (("y", dtype), ("x", stream), ("gate", dtype)):
        if a[n] is None:
            assert getattr(r, n) is None
        else:
            check("grad " + n, getattr(r, n), want[n], tol(n, t))
    for n in ("after", "before"):
        if w[n] is None:
            assert getattr(r, n) is None
        else:
            check("grad " + n, getattr(r, n), want[n], tol(n, "f32", rows=N))
    return norm, u, h, r


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("N,D", [(1, 1), (3, 2), (5, 7), (300, 8), (2, 9), (17, 64), (33, 65), (9, 511), (6, 512), (5, 513), (4, 1000), (3, 1024), (3, 1025), (4, 2048),
                                 (3, 4097), (2, 8191), (2, 16384), (700, 1030)])
def test_sizes(A, dtype, stream, N, D):
    a, w, flow = make(N, D, dtype, stream)
    run(A, a, w, flow, "rms", "sigmoid", dtype, stream)


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", [None, "sigmoid", "silu"])
@pytest.mark.parametrize("x", [True, False])
@pytest.mark.parametrize("after,before", [(True, True), (True, False), (False, True), (False, False)])
def test_forms(A, dtype, stream, kind, gate, x, after, before):
    if not x:
        stream = dtype
    for N, D in ((37, 100), (5, 1300)):
        a, w, flow = make(N, D, dtype, stream, ld=5, x=x, gate=gate, after=after, before=before)
        run(A, a, w, flow, kind, gate, dtype, stream)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,D,groups", [(1, 6, 6), (50, 48, 3), (33, 256, 16), (9, 1000, 8), (7, 999, 37), (3, 4096, 2), (2, 16384, 4), (1000, 60, 5), (4000, 16, 1)])
def test_groups(A, dtype, N, D, groups):
    for kind in ("rms", "layer"):
        a, w, flow = make(N, D, dtype, dtype, before=False)
        run(A, a, w, flow, kind, "silu", dtype, dtype, groups=groups)


def test_many_rows(A):
    """More rows than slots: each goes over several, in the same order every time."""
    a, w, flow = make(9001, 40, "bf16", "f32")
    norm, u, h, r = run(A, a, w, flow, "rms", "sigmoid", "bf16", "f32")
    again = norm.backward(**a, **flow)
    assert all(torch.equal(getattr(r, n), getattr(again, n)) for n in ("y", "x", "gate", "after", "before"))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_no_rows(A, dtype):
    norm = A.BlockNorm(50, after=torch.ones(50), before=torch.ones(50))
    y = torch.empty((0, 50), dtype=DT[dtype], device="cuda")
    u, h = norm.forward(y, x=y)
    assert u.shape == h.shape == (0, 50)
    r = norm.backward(y, x=y, grad_u=y, grad_h=y)
    assert r.y.shape == (0, 50) and (r.after == 0).all() and (r.before == 0).all()


@pytest.mark.parametrize("D", [96, 2000])
def test_one_gradient_alone(A, D):
    """grad_u or grad_h left out counts as zeros."""
    a, w, flow = make(20, D, "f32", "f32")
    norm = A.BlockNorm(D, **w, gate="sigmoid")
    zero = torch.zeros((20, D), device="cuda")
    for k in ("grad_u", "grad_h"):
        got = norm.backward(**a, **{k: flow[k]})
        want = norm.backward(**a, **{k: flow[k], ({"grad_u": "grad_h", "grad_h": "grad_u"}[k]): zero})
        assert all(torch.equal(getattr(got, n), getattr(want, n)) for n in ("y", "x", "gate", "after", "before"))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [40, 1500])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_row(A, dtype, D, what):
    a, w, flow = make(30, D, dtype, dtype)
    norm = A.BlockNorm(D, **w, kind="layer", gate="silu")
    u, h = norm.forward(**a)
    r = norm.backward(**a, **flow)
    rest = torch.arange(30, device="cuda") != 11
    for n in ("y", "x", "gate"):
        b = dict(a, **{n: a[n].clone()})
        b[n][11, 3] = what
        u2, h2 = norm.forward(**b)
        assert torch.equal(u2[rest], u[rest]) and torch.equal(h2[rest], h[rest]) and not torch.isfinite(h2[11]).all()
        r2 = norm.backward(**b, **flow)
        assert all(torch.equal(getattr(r2, m)[rest], getattr(r, m)[rest]) for m in ("y", "x", "gate"))


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_zeros_and_of_one_value(A, kind):
    """The square root's eps is all that is left of them."""
    for D in (64, 1200):
        a, w, flow = make(6, D, "f32", "f32", x=False, gate=None)
        a["y"][0] = 0
        a["y"][1] = 2.0
        a["y"][2] = 1e-20
        run(A, a, w, flow, kind, None, "f32", "f32", eps=1e-3)


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("D", [72, 2048])
def test_over_the_inputs(A, dtype, stream, D):
    """The stream in place, the block's output replaced by the next one's input."""
    a, w, flow = make(40, D, dtype, stream)
    norm = A.BlockNorm(D, **w, gate="sigmoid")
    u, h = norm.forward(**a)
    got = norm.forward(**a, u=a["x"], h=a["y"])
    assert got[0] is a["x"] and got[1] is a["y"] and torch.equal(a["x"], u) and torch.equal(a["y"], h)


def test_gradients_over_the_gradients(A):
    """Through the C entry, as a learner short of memory: grad_x over grad_u, grad_y over grad_h, grad_gate over the gate."""
    a, w, flow = make(33, 500, "bf16", "f32")
    norm = A.BlockNorm(500, **w, gate="silu")
    want = norm.backward(**a, **flow)
    ws = torch.empty(A.accerl_block_norm_workspace(33, 500), dtype=torch.uint8, device="cuda")
    A.accerl_block_norm_grad(a["y"], ws, x=a["x"], gate=a["gate"], after=w["after"], before=w["before"], grad_u=flow["grad_u"], grad_h=flow["grad_h"],
                             grad_y=flow["grad_h"], grad_x=flow["grad_u"], grad_gate=a["gate"], gate_kind="silu")
    assert torch.equal(flow["grad_h"], want.y) and torch.equal(flow["grad_u"], want.x) and torch.equal(a["gate"], want.gate)


def test_values_without_u(A):
    """The norm alone, before the first block."""
    y = torch.randn((50, 300), device="cuda").to(torch.bfloat16)
    w = torch.randn(300, device="cuda")
    norm = A.BlockNorm(300, before=w)
    h = torch.empty_like(y)
    A.accerl_block_norm(y, None, h, before=w)
    assert torch.equal(h, norm.forward(y)[1])


def test_update(A):
    y = torch.randn((5, 60), device="cuda")
    first, second = torch.randn(60, device="cuda"), torch.randn(60, device="cuda")
    norm = A.BlockNorm(60, after=first)
    norm.update(after=second)
    assert torch.equal(norm.forward(y)[0], A.BlockNorm(60, after=second).forward(y)[0])


def test_gradients_against_differences(A):
    """Central differences of the kernels' own fp32 values along random ways."""
    N, D = 12, 96
    a, w, flow = make(N, D, "f32", "f32")
    r = A.BlockNorm(D, **w, kind="layer", gate="silu", branch=0.7).backward(**a, **flow)

    def value(x, v):
        u, h = A.BlockNorm(D, **v, kind="layer", gate="silu", branch=0.7).forward(**x)
        return float((u.double() * flow["grad_u"]).sum() + (h.double() * flow["grad_h"]).sum())
    step = 2.0 ** -8
    for n in ("y", "x", "gate", "after", "before"):
        at = a if n in a else w
        way = torch.randn_like(at[n])
        here = lambda s: value(dict(a, **{n: a[n] + s * way}) if n in a else a, dict(w, **{n: w[n] + s * way}) if n in w else w)
        # two steps: the error of the central difference goes with the square of the step, so that this combination leaves its fourth power
        got = (8 * (here(step) - here(-step)) - (here(2 * step) - here(-2 * step))) / (12 * step)
        want = float((getattr(r, n).double() * way).sum())
        # values of N D terms of size about 3, each off by some ten roundings in either direction: a random walk's 6 deviations over the step; the fourth power
        # of the step times fifth derivatives, which stay below 100 a term here
        assert abs(got - want) <= 6 * (N * D) ** 0.5 * 3 * 10 * ref.U * 18 / (12 * step) + N * D * 100 * step ** 4, n
