"""LinearAttention and BlockNorm without a GPU: copies of owners, workspaces by size, launches that no card takes."""
import copy
import ctypes as C
import pickle

import pytest
import torch

from tests.test_memory_ops_cpu import EUNSUPPORTED, attention_args


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def test_copies_of_an_owner(A):
    at = A.LinearAttention([0.0, 0.5, 1.0], scale=0.25, device="cpu")
    for c in (copy.deepcopy(at), pickle.loads(pickle.dumps(at))):
        assert c.H == 3 and c.scale == 0.25 and torch.equal(c.log_decay, at.log_decay) and c._work is not at._work


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("B,H,Dk,Dv", [(1, 1, 64, 64), (2, 4, 128, 100), (40, 3, 64, 64), (1, 16, 256, 256)])
def test_workspaces_of_segments(A, B, H, Dk, Dv, grad):
    """None for a chunk; some states where a sequence is long and sequences are few; never more than 1024 workgroups' and one for each chunk."""
    work = lambda T: A.accerl_linear_attention_workspace(B, T, H, H, Dk, Dv, grad=grad)
    assert work(0) == work(1) == work(64) == work(128) == 0
    workgroups = B * H * ((2 * ((Dk + 63) // 64) if grad else 0) + (Dv + 63) // 64)
    assert (work(1 << 20) > 0) == (workgroups < 192)             # 192 of them: enough without segments, in every type
    for T in (192, 600, 5000, 1 << 20):
        segments = min((T + 63) // 64, 1 + 1024 // (B * H))
        assert work(T) <= (2 if grad else 1) * 4 * (segments * (B * H * Dk * Dv + B * H) + 32)


def test_more_heads_than_a_launch_takes(A):
    """2^22 heads of 256 elements: refused before anything is enqueued (the addresses are never read)."""
    from paper_2211_15023_amd import binding
    lib = A.load_library()
    s = binding._TokenStride(1024, 1024, 256)
    at = lambda i: (i + 1) << 40
    big = dict(B=1 << 20, T=1, H=4, Hk=4, Dk=256, Dv=256, reset=None, lengths=None, q_stride=s, k_stride=s, v_stride=s, out_stride=s, grad_out_stride=s, grad_q_stride=s, grad_k_stride=s,
               grad_v_stride=s, q=at(0), k=at(1), v=at(2), out=at(3), grad_out=at(4), grad_q=at(5), grad_k=at(6), grad_v=at(7), state=None, out_state=None, grad_state=None,
               grad_out_state=None, workspace=None, workspace_bytes=0)
    for dtype in (0, 1, 2):
        a = attention_args(at(9), dtype=dtype, **big)
        for f in (lib.accerl_linear_attention, lib.accerl_linear_attention_grad):
            assert f(C.byref(a), None) == EUNSUPPORTED and "one launch" in A.accerl_last_error()
        a = attention_args(at(9), dtype=dtype, **dict(big, state=at(20), out_state=at(20)))
        assert lib.accerl_linear_attention_step(C.byref(a), None) == EUNSUPPORTED and "one launch" in A.accerl_last_error()


def test_more_shared_gradients_than_a_launch_takes(A):
    """2^25 tokens of 128 elements whose heads are shared: refused before anything is enqueued."""
    from paper_2211_15023_amd import binding
    lib = A.load_library()
    q, kv = binding._TokenStride(256 << 25, 256, 128), binding._TokenStride(128 << 25, 128, 128)
    at = lambda i: (i + 1) << 40
    a = attention_args(at(9), B=1, T=1 << 25, H=2, Hk=1, Dk=128, Dv=128, reset=None, lengths=None, q_stride=q, k_stride=kv, v_stride=kv, grad_out_stride=q, grad_q_stride=q, grad_k_stride=kv,
                       grad_v_stride=kv, q=at(0), k=at(1), v=at(2), grad_out=at(4), grad_q=at(5), grad_k=at(6), grad_v=at(7), state=None, grad_state=None, grad_out_state=None,
                       workspace=at(30), workspace_bytes=1 << 40)
    assert lib.accerl_linear_attention_grad(C.byref(a), None) == EUNSUPPORTED and "shared heads" in A.accerl_last_error()


def test_a_table_for_a_norm_that_is_not_there(A):
    with torch._subclasses.fake_tensor.FakeTensorMode():
        y = torch.empty((3, 8), device="cuda")
        norm = A.BlockNorm(8, after=y[0])
        with pytest.raises(ValueError, match="before the next block"):
            norm.forward(y, h=torch.empty_like(y))
        with pytest.raises(ValueError, match="before the next block"):
            norm.backward(y, grad_h=y)
