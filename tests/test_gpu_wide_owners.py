"""DenseInt8 and PolicyLoss as owners: what they keep between calls, who shares it, and what they refuse."""
import threading

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


def _threads(work):
    """work(i) in a thread for each of i = 0, 1; all start together, and what one raises is raised here."""
    start, got, wrong = threading.Barrier(2), [None, None], []

    def run(i):
        try:
            start.wait(30)
            got[i] = work(i)
        except BaseException as e:                                 # (shown by the test's own thread)
            wrong.append(e)

    ts = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    if wrong:
        raise wrong[0]
    return got


@pytest.mark.parametrize("M", [16, 300])
def test_two_threads_share_a_layer(A, M):
    """Both on the default stream, each with tokens of its own."""
    layer = A.DenseInt8(torch.randn((1000, 500), device="cuda"))
    x = [torch.randn((M, 500), device="cuda") * 10 ** i for i in range(2)]
    want = [layer.forward(t) for t in x]
    torch.cuda.synchronize()
    got = _threads(lambda i: [layer.forward(x[i]) for _ in range(100)])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i]), i


@pytest.mark.parametrize("B,n", [(3000, 18), (3, 60001)])
def test_two_threads_share_a_loss(A, B, n):
    """Rows of a wavefront, whose sums are added up by a second launch, and rows in pieces."""
    how = A.PolicyLoss(entropy_coef=0.1)
    z = [torch.randn((B, n), device="cuda") * (i + 1) for i in range(2)]
    act, v = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), -1.0, device="cuda")
    want = [how.forward(t, act, v, v) for t in z]
    torch.cuda.synchronize()
    got = _threads(lambda i: [how.forward(z[i], act, v, v) for _ in range(50)])
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert torch.equal(r.stats, want[i].stats) and torch.equal(r.grad, want[i].grad), i
