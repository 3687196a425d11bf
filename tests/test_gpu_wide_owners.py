"""DenseInt8 and PolicyLoss as owners: what they keep between calls, who shares it, and what they refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def test_a_call_that_is_refused_stays_refused(A):
    """A layer whose channels do not fit any more: every call goes by their lengths, the first and those that find a workspace."""
    layer = A.DenseInt8(torch.randn((40, 30), device="cuda"), bias=torch.randn(40, device="cuda"))
    x = torch.randn((4, 30), device="cuda")
    layer.forward(x)
    kept = {k: getattr(layer, k) for k in ("w", "w_scale", "bias")}
    for k, v in kept.items():
        setattr(layer, k, v[:17])
        for _ in range(2):
            with pytest.raises(ValueError):
                layer.forward(x)
        setattr(layer, k, v)
    assert torch.equal(layer.forward(x), layer.forward(x, stream=torch.cuda.current_stream()))


def test_a_bias_of_the_host(A):
    """The layer's own bias lies beside its weights."""
    w, b = torch.randn((40, 30), device="cuda"), torch.randn(40, dtype=torch.float64)
    layer = A.DenseInt8(w, bias=b)
    assert layer.bias.is_cuda and torch.equal(layer.bias.cpu(), b.float())
    x = torch.randn((4, 30), device="cuda")
    assert torch.equal(layer.forward(x), A.DenseInt8(w, bias=b.float().cuda()).forward(x))
