"""DenseInt8 and PolicyLoss without a GPU: what they refuse before anything is enqueued, on tensors that claim to lie on one."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("shape", [(39,), (41,), (1,), (40, 1), (1, 40), ()])
def test_a_bias_of_another_length_is_refused_when_the_layer_is_made(A, shape):
    with FakeTensorMode():
        w, bias = torch.empty((40, 30), device="cuda"), torch.empty(shape, device="cuda")
        with pytest.raises(ValueError, match="bias"):
            A.DenseInt8(w, bias=bias)


@pytest.mark.parametrize("shape", [(1,), (39,), (41,), (40, 1), (1, 40), ()])
def test_scales_of_another_length_are_refused(A, shape):
    with FakeTensorMode():
        w, w_scale = torch.empty((40, 30), dtype=torch.int8, device="cuda"), torch.empty(shape, device="cuda")
        with pytest.raises(ValueError, match="scales"):
            A.DenseInt8(w, w_scale)


def test_scales_of_a_float_matrix_are_refused(A):
    with FakeTensorMode():
        w, w_scale = torch.empty((40, 30), device="cuda"), torch.empty(40, device="cuda")
        with pytest.raises(ValueError, match="scales"):
            A.DenseInt8(w, w_scale)
