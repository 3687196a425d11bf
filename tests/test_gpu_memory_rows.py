"""The operators of policies with a memory at sizes beyond the other tests': no tokens of shared heads."""
import pytest
import torch

from tests.test_gpu_linear_attention import decays, make

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
