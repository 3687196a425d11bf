"""Linear attention where numbers are not finite or leave fp32's range on the way: every result is the recurrence's, and no token's depends on one behind it."""
import numpy as np
import pytest
import torch

from tests import memory_reference as ref
from tests.test_gpu_linear_attention import DT, check, make, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def both(A, a, decay, go, scale=0.125):
    """The kernels' results and the recurrence's, by name."""
    at = A.LinearAttention(decay, scale=scale)
    out, last = at.forward(a["q"], a["k"], a["v"], state=a["state"], reset=a["reset"])
    r = at.backward(go, a["q"], a["k"], a["v"], state=a["state"], reset=a["reset"])
    w, d = {n: wide(a[n]) for n in "qkv"}, np.array(decay)
    arg = dict(reset=wide(a["reset"]), state=wide(a["state"]))
    with np.errstate(all="ignore"):
        o, s = ref.unroll(w["q"], w["k"], w["v"], d, scale, **arg)
        g = ref.unroll_grad(wide(go), w["q"], w["k"], w["v"], d, scale, **arg)
    return {"out": (out, o), "state": (last, s), "grad q": (r.q, g["q"]), "grad k": (r.k, g["k"]), "grad v": (r.v, g["v"]), "grad state": (r.state, g["state"])}


def alike(results):
    """NaN where the recurrence has NaN, infinities of its sign where it has them, numbers elsewhere."""
    for name, (got, want) in results.items():
        got = wide(got)
        assert np.array_equal(np.isnan(got), np.isnan(want)), name
        assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want)), name


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D,E", [(1, 64, 64), (150, 64, 64), (150, 33, 20), (100, 128, 128), (100, 256, 70), (700, 48, 72)])
@pytest.mark.parametrize("which,what", [("q", float("inf")), ("q", -float("inf")), ("k", float("inf")), ("v", float("inf")), ("q", float("nan"))])
def test_infinities_have_the_recurrences_sign(A, dtype, T, D, E, which, what):
    """An infinity of a query meets one row of the state: its output has an infinity of each column's sign, no NaN; and so on through the gradients."""
    B, H = 2, 2
    a = make(B, T, H, H, D, E, dtype, resets=0.01)
    a[which][0, T // 2, 1, 5] = what
    alike(both(A, a, [0.9, 0.99], torch.randn((B, T, H, E), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(DT[dtype])))


def _sizes(a, go, decay, scale=0.125):
    x = {n: np.abs(wide(a[n])) for n in "qkv"}
    arg = dict(reset=wide(a["reset"]), state=np.abs(wide(a["state"])))
    oa, sa = ref.unroll(x["q"], x["k"], x["v"], np.array(decay), scale, **arg)
    ga = ref.unroll_grad(np.abs(wide(go)), x["q"], x["k"], x["v"], np.array(decay), scale, **arg)
    return {"out": oa, "state": sa, "grad q": ga["q"], "grad k": ga["k"], "grad v": ga["v"], "grad state": ga["state"]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("early,late,decay", [("q", "k", [0.9, 0.99]), ("k", "q", [0.0, 1e-9])])
@pytest.mark.parametrize("T,D,E", [(40, 64, 64), (100, 128, 96), (70, 33, 20)])
def test_a_product_past_the_range_that_no_result_holds(A, dtype, early, late, decay, T, D, E):
    """A query and a key of 2^66, whose product fp32 does not hold.  Where the query's token comes first the recurrence never multiplies them; where the key's does,
    a decay of nothing lies between."""
    a = make(2, T, 2, 2, D, E, dtype)
    a[early][0, 5] = 2.0 ** 66
    a[late][0, 12] = 2.0 ** 66
    go = torch.randn((2, T, 2, E), device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(DT[dtype])
    sizes = _sizes(a, go, decay)
    for name, (got, want) in both(A, a, decay, go).items():
        state = "state" in name
        check(name, got, want, ref.unroll_tolerance(want, sizes[name], dtype, T, max(D, E), np.array(decay), state=state))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [150, 700, 2000])
@pytest.mark.parametrize("which", ["k", "v", "state"])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("decay", [[0.1, 0.9], [0.0, 0.9]])
def test_no_decay_ends_what_is_not_finite(A, dtype, T, which, what, decay):
    """Between episodes' borders it goes on to the last token, also where a chunk's or a segment's decay is below what fp32 holds (0.1^64)."""
    a = make(1, T, 2, 2, 48, 72, dtype)
    if which == "state":
        a["state"][0, 0, 5, 3] = what
    else:
        a[which][0, 37, 0, 5] = what
    go = torch.randn((1, T, 2, 72), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(DT[dtype])
    alike(both(A, a, decay, go))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", [(1, 1), (17, 5), (33, 64), (40, 70), (64, 64), (100, 128), (130, 20), (256, 256)])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_a_step_of_an_infinity(A, dtype, Dk, Dv, which):
    """Everything positive, so that each sum that meets it is an infinity."""
    B, H = 2, 2
    g = torch.Generator(device="cuda").manual_seed(Dk)
    draw = lambda *s: (torch.rand(s, generator=g, device="cuda") + 0.5)
    x = dict(q=draw(B, H, Dk).to(DT[dtype]), k=draw(B, H, Dk).to(DT[dtype]), v=draw(B, H, Dv).to(DT[dtype]))
    x[which][0, 1, -1] = float("inf")
    state = draw(B, H, Dk, Dv)
    beside = torch.empty_like(state)
    out = A.LinearAttention([0.9, 0.5]).step(**x, state=state, out_state=beside)
    o, s = ref.unroll(*(wide(x[n])[:, None] for n in "qkv"), np.array([0.9, 0.5]), 1.0, state=wide(state))
    alike({"out": (out, o[:, 0]), "state": (beside, s)})
