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


def _replays(graphs, outs, want, rounds=4):
    for _ in range(rounds):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_a_layer_outgrows_what_a_graph_has_seen(A):
    """Captured at 64 tokens on the user's stream, then called there with more, then memory of that stream is taken: the replays give the
    captured call's results and leave that memory alone."""
    layer = A.DenseInt8(torch.randn((300, 200), device="cuda"))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x, many = torch.randn((64, 200), device="cuda"), torch.randn((4096, 200), device="cuda")
        want = layer.forward(x)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = layer.forward(x)
        layer.forward(many)
        taken = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (512, 2048, 16384, 16896, 20480, 65536) for _ in range(20)]
        _replays([graph], [out], [want])
        assert all(bool((t == 7).all()) for t in taken)
        assert torch.equal(layer.forward(x), want)


@pytest.mark.parametrize("side", ["layer", "loss"])
def test_two_graphs_of_one_owner_replayed_at_once(A, side):
    """Captured one after the other on torch's capture stream, replayed on two streams."""
    if side == "layer":
        layer = A.DenseInt8(torch.randn((1000, 500), device="cuda"))
        x = [torch.randn((300, 500), device="cuda") * 10 ** i for i in range(2)]
        call = lambda i: [layer.forward(x[i])]
    else:
        how, v = A.PolicyLoss(entropy_coef=0.1), torch.full((3,), -1.0, device="cuda")
        x, act = [torch.randn((3, 60001), device="cuda") * (i + 1) for i in range(2)], torch.zeros(3, dtype=torch.int32, device="cuda")

        def call(i):
            r = how.forward(x[i], act, v, v)
            return [r.grad, r.stats]
    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], [None, None]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            outs[i] = call(i)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i in range(2):
            for o in outs[i]:
                o.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        call(0)                                                   # an eager call between them
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(o, w) for o, w in zip(outs[i], want[i])), i


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_outputs_lie_where_the_inputs_do(A):
    """Inputs of the device that is not the current one: outputs, workspaces and launches are that device's, in every call."""
    layer = A.DenseInt8(torch.randn((40, 30), device="cuda:1"), bias=torch.randn(40, device="cuda:1"))
    how = A.PolicyLoss()
    x, act, v = torch.randn((4, 30), device="cuda:1"), torch.zeros(4, dtype=torch.int32, device="cuda:1"), torch.zeros(4, device="cuda:1")
    with torch.cuda.device(1):
        want = layer.forward(x)
        loss = how.forward(want, act, v, v)
        torch.cuda.synchronize()
    for _ in range(3):
        y = layer.forward(x)
        r, lp = how.forward(y, act, v, v), how.logprob(y, act)
        torch.cuda.synchronize(1)
        assert all(t.device == x.device for t in (y, r.loss, r.grad, r.stats, *lp))
        assert torch.equal(y, want) and torch.equal(r.grad, loss.grad) and torch.equal(lp[0], loss.logp)


@pytest.mark.parametrize("M", [1, 2, 3, 200])
@pytest.mark.parametrize("shift", [0, 1, -3])
def test_a_layer_writes_over_its_input(A, M, shift):
    """Whole, and shifted by some elements: all tokens are read before a result is written."""
    n = 900
    layer = A.DenseInt8(torch.randn((n, n), device="cuda"), bias=torch.randn(n, device="cuda"))
    table = torch.randn(M * n + 16, device="cuda")
    x, out = (table[8 + s:8 + s + M * n].view(M, n) for s in (0, shift))
    want = layer.forward(x.clone())
    assert layer.forward(x, out=out) is out
    assert torch.equal(out, want)


@pytest.mark.parametrize("M", [2, 40])
def test_a_layer_writes_beside_its_input(A, M):
    """Input and output are columns of one table: rows that lie between each other's, which share nothing."""
    layer = A.DenseInt8(torch.randn((300, 500), device="cuda"))
    table = torch.randn((M, 1000), device="cuda")
    x, out = table[:, 100:600], table[:, 600:900]
    rest, want = table.clone(), layer.forward(x.contiguous())
    layer.forward(x, out=out)
    rest[:, 600:900] = want
    assert torch.equal(table, rest)


@pytest.mark.parametrize("B,n", [(50, 18), (300, 130), (520, 5003), (3, 60001)])
def test_a_gradient_beside_the_logits(A, B, n):
    """Logits, the reference's and the gradient are columns of one table."""
    how = A.PolicyLoss(kl="forward", kl_coef=0.1, entropy_coef=0.1)
    table = torch.randn((B, 3 * n), device="cuda")
    z, zr, g = table[:, n:2 * n], table[:, 2 * n:], table[:, :n]
    act, v = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), -1.0, device="cuda")
    want = how.forward(z.contiguous(), act, v, v, ref_logits=zr.contiguous())
    rest = table.clone()
    got = how.forward(z, act, v, v, ref_logits=zr, grad=g)
    rest[:, :n] = want.grad
    assert torch.equal(table, rest) and torch.equal(got.stats, want.stats) and torch.equal(got.loss, want.loss)
