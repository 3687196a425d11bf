"""fp16 tokens, whose products with weights of pairs and with the state go through two bf16 parts of each: sums that cancel show what the parts leave out."""
import numpy as np
import pytest
import torch

from tests import memory_reference as ref
from tests.test_gpu_linear_attention import check, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def _numbers(n, step, bits=10):
    """n numbers from 1 to 2 with all kinds of last bits."""
    return 1 + (torch.arange(n, device="cuda", dtype=torch.float64) * step + 4) % 2 ** bits / 2 ** bits


def _tolerance(want, size, more=4):
    """Of a term: the second part of a weight or of the state is rounded, 2^-17 (a part is rounded to nearest, so that the second is 2^-8 at most, and half its last step 2^-9
    of it), and the product of both second parts is left out, 2^-8 2^-8.  Then `more` roundings of fp32 (the weight, its product, the sum, the state), and the result's own."""
    return size * (2.0 ** -17 + 2.0 ** -16 + more * ref.U) + ref.HALF_STEP["f16"] * np.abs(want) * 1.001 + ref.TINY["f16"]


@pytest.mark.parametrize("D", [1, 8, 64])
@pytest.mark.parametrize("back", [False, True])
def test_pairs_that_cancel(A, D, back):
    """x y - z, z being x y in fp16, a third of it: the output of two tokens, and (from the last to the first) the gradient by the first one's key."""
    B, E = 64, 64
    x, y = _numbers(B, 37), _numbers(E, 53)
    z = (x[:, None] * y).half().double()
    at = A.LinearAttention([1.0], scale=1 / 3)
    zeros = lambda *s: torch.zeros(s, device="cuda", dtype=torch.float16)
    size = wide((x[:, None] * y + z) / 3)
    if not back:
        q, k, v = zeros(B, 2, 1, D), zeros(B, 2, 1, D), zeros(B, 2, 1, E)
        q[:, :, 0, 0], k[:, 0, 0, 0], k[:, 1, 0, 0], v[:, 0, 0], v[:, 1, 0] = 1, x, -1, y, z
        got, want = at.forward(q, k, v)[0][:, 1, 0], (x[:, None] * y - z) / 3
        check("out", got, wide(want), _tolerance(wide(want), size))
    else:
        # dk_0 = sum over t of (v_0 . go_t) q_t: the second token's query is y, the first one's z
        q, k, v, go = zeros(B, 2, 1, E), zeros(B, 2, 1, E), zeros(B, 2, 1, D), zeros(B, 2, 1, D)
        v[:, 0, 0, 0], go[:, 1, 0, 0], go[:, 0, 0, 0], q[:, 1, 0], q[:, 0, 0] = 1, x, -1, y, z
        got, want = at.backward(go, q, k, v).k[:, 0, 0], (x[:, None] * y - z) / 3
        check("grad k", got, wide(want), _tolerance(wide(want), size))


@pytest.mark.parametrize("D", [2, 8, 64, 100, 200])
@pytest.mark.parametrize("back", [False, True])
def test_states_that_cancel(A, D, back):
    """x s - t, t being x s in fp32, from a state of s and t and a query (gradient: an output's gradient) of x and -1."""
    B, E = 64, 64
    x, s = _numbers(B, 37), _numbers(E, 52763, bits=23)
    t = (x[:, None] * s).float().double()
    at = A.LinearAttention([1.0])
    zeros = lambda *n: torch.zeros(n, device="cuda", dtype=torch.float16)
    a, other = zeros(B, 1, 1, D), zeros(B, 1, 1, E)
    a[:, 0, 0, 0], a[:, 0, 0, 1] = x, -1
    state = torch.zeros((B, 1, D, E), device="cuda")
    state[:, 0, 0], state[:, 0, 1] = s.float(), t.float()
    want, size = wide(x[:, None] * s.float().double() - t), wide(x[:, None] * s + t)
    if not back:
        check("out", at.forward(a, zeros(B, 1, 1, D), other, state=state)[0][:, 0, 0], want, _tolerance(want, size))
    else:
        r = at.backward(a, other, zeros(B, 1, 1, E), zeros(B, 1, 1, D), state=state.transpose(2, 3).contiguous())
        check("grad q", r.q[:, 0, 0], want, _tolerance(want, size))
