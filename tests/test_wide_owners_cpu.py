"""DenseInt8 and PolicyLoss without a GPU: what they refuse before anything is enqueued, on tensors that claim to lie on one."""
import copy
import pickle
import threading

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


@pytest.fixture
def capture(monkeypatch):
    """Says whether the current stream captures: none does here."""
    from paper_2211_15023_amd import binding
    now = [False]
    monkeypatch.setattr(binding, "_captured", lambda stream: now[0], raising=False)
    return now


def _in_thread(f):
    out = []
    t = threading.Thread(target=lambda: out.append(f()))
    t.start()
    t.join()
    return out[0]


def test_a_workspace_belongs_to_one_thread_and_stream(A, capture):
    """Calls of one thread on one stream share a buffer; a call of another thread may come between the launches of this one's."""
    from paper_2211_15023_amd import binding
    w, cpu = binding._Workspaces(), torch.device("cpu")
    mine = w.get(100, 0, cpu)
    assert w.get(64, 0, cpu) is mine and w.kept(0, None) is mine and w.get(101, 0, cpu) is not mine
    mine = w.kept(0, None)
    other = _in_thread(lambda: (w.kept(0, None), w.get(100, 0, cpu)))
    assert other[0] is None and other[1].data_ptr() != mine.data_ptr()
    assert w.get(100, 7, cpu).data_ptr() != mine.data_ptr() and w.kept(0, None) is mine


def test_owners_are_copied_without_their_workspaces(A, capture):
    from paper_2211_15023_amd import binding
    w, cpu = binding._Workspaces(), torch.device("cpu")
    w.get(100, 0, cpu)
    for c in (copy.deepcopy(w), pickle.loads(pickle.dumps(w))):
        assert c.kept(0, None) is None and w.kept(0, None) is not None


def test_a_captured_call_has_a_workspace_of_its_own(A, capture):
    """A graph keeps the address: no later call on its stream, captured or not, gets it from the owner, and none replaces it there."""
    from paper_2211_15023_amd import binding
    w, cpu = binding._Workspaces(), torch.device("cpu")
    eager = w.get(100, 7, cpu)
    capture[0] = True
    captured = [w.get(100, 7, cpu) for _ in range(2)]
    assert len({t.data_ptr() for t in (eager, *captured)}) == 3 and w.kept(7, None) is None
    capture[0] = False
    assert w.get(100, 7, cpu) is eager


def _calls():
    """The calls with tensors that fit, by name, and the names of their tensors."""
    B, n, K = 3, 5, 7
    f = lambda *shape: torch.empty(shape, device="cuda:1")
    packed = torch.empty(4096, dtype=torch.int8, device="cuda:1")
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:1")
    actions, mask = torch.empty(B, dtype=torch.int32, device="cuda:1"), torch.empty((B, n), dtype=torch.uint8, device="cuda:1")
    rows = torch.empty((B, K), dtype=torch.int8, device="cuda:1")
    return {"accerl_quantize_rows": dict(x=f(B, K), out_packed=packed, out_scale=f(B)), "accerl_pack_rows_i8": dict(q=rows, out_packed=packed),
            "accerl_unpack_rows_i8": dict(packed=packed, out_q=rows),
            "accerl_dense_i8": dict(x_packed=packed, x_scale=f(B), w_packed=packed, w_scale=f(n), bias=f(n), K=K, out=f(B, n)),
            "accerl_dense_i8_dynamic": dict(x=f(B, K), w_packed=packed, w_scale=f(n), bias=f(n), out=f(B, n), workspace=work),
            "accerl_action_logprob": dict(logits=f(B, n), mask=mask, actions=actions, out_logp=f(B), out_entropy=f(B), workspace=work),
            "accerl_policy_loss": dict(logits=f(B, n), actions=actions, old_logp=f(B), advantages=f(B), workspace=work, mask=mask, weights=f(B),
                                       ref_logits=f(B, n), ref_logp=f(B), grad_logits=f(B, n), out_loss=f(B), out_logp=f(B), out_kl=f(B), out_entropy=f(B),
                                       out_stats=f(4))}


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
@pytest.mark.parametrize("name", ["accerl_quantize_rows", "accerl_pack_rows_i8", "accerl_unpack_rows_i8", "accerl_dense_i8", "accerl_dense_i8_dynamic",
                                  "accerl_action_logprob", "accerl_policy_loss"])
def test_tensors_of_two_devices_are_refused(A, name):
    with FakeTensorMode():
        good = _calls()[name]
        for k, t in good.items():
            if isinstance(t, torch.Tensor):
                with pytest.raises(ValueError, match="devices"):
                    getattr(A, name)(**dict(good, **{k: torch.empty_like(t, device="cuda:0")}))
