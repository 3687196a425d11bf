"""Operators of wide policies without a GPU: sizes, refusals, and the 64-bit reference against differences."""
import ctypes as C

import numpy as np
import pytest

from tests import wide_reference as ref

EINVAL, EUNSUPPORTED = -1, -4


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


def aligned(n):
    """Address of n bytes of host memory, 256-byte aligned (refusals never look behind it), and its owner."""
    raw = np.zeros(n + 256, np.uint8)
    return (raw.ctypes.data + 255) // 256 * 256, raw


def test_packed_sizes(A):
    for rows, cols, want in ((0, 1, 0), (1, 1, 2048), (16, 128, 2048), (17, 129, 2 * 4096), (512, 3136, 512 * 3200)):
        assert A.packed_rows_bytes(rows, cols) == want
    for rows, cols, code in ((-1, 4, EINVAL), (4, 0, EINVAL), (4, (1 << 16) + 1, EUNSUPPORTED), ((1 << 24) + 1, 4, EUNSUPPORTED)):
        with pytest.raises(A.AccerlError) as e:
            A.packed_rows_bytes(rows, cols)
        assert e.value.code == code
    assert A.accerl_dense_i8_workspace(1, 1) >= 2048 + 4
    assert A.accerl_dense_i8_workspace(0, 5) >= 0
    assert A.accerl_policy_loss_workspace() > 0


def test_row_calls_refuse(A):
    lib = A.load_library()
    p, own = aligned(1 << 16)
    good = [p, 1, 4, 100, 104, p, p, None]                      # x dtype rows cols ld packed scale stream
    for at, bad, code in ((0, None, EINVAL), (1, 3, EINVAL), (1, -1, EINVAL), (2, -1, EINVAL), (3, 0, EINVAL), (4, 99, EINVAL), (5, None, EINVAL),
                          (5, p + 8, EINVAL), (6, None, EINVAL), (6, p + 2, EINVAL), (0, p + 1, EINVAL), (2, (1 << 24) + 1, EUNSUPPORTED)):
        args = list(good)
        args[at] = bad
        assert lib.accerl_quantize_rows(*args) == code, (at, bad)
        assert A.accerl_last_error()
    assert lib.accerl_quantize_rows(None, 0, 0, 4, 4, None, None, None) == 0          # no rows: nothing to do
    for f, args in ((lib.accerl_pack_rows_i8, [p, 4, 100, 104, p, None]), (lib.accerl_unpack_rows_i8, [p, 4, 100, p, 104, None])):
        for at in (0, 4 if f is lib.accerl_pack_rows_i8 else 3):
            bad = list(args)
            bad[at] = None
            assert f(*bad) == EINVAL
        bad = list(args)
        bad[3 if f is lib.accerl_pack_rows_i8 else 4] = 50
        assert f(*bad) == EINVAL
        bad = list(args)
        bad[1] = 0
        assert f(*bad) == 0


def test_dense_refuses(A):
    lib = A.load_library()
    p, own = aligned(1 << 16)
    # xq sx wq sw bias M N K relu out dtype ld stream
    good = [p, p, p, p, None, 3, 5, 100, 0, p, 1, 5, None]
    for at, bad, code in ((0, None, EINVAL), (0, p + 8, EINVAL), (1, None, EINVAL), (1, p + 1, EINVAL), (2, None, EINVAL), (2, p + 4, EINVAL), (3, None, EINVAL),
                          (4, p + 2, EINVAL), (5, -1, EINVAL), (6, -1, EINVAL), (7, 0, EINVAL), (7, (1 << 16) + 1, EUNSUPPORTED), (9, None, EINVAL),
                          (9, p + 1, EINVAL), (10, 7, EINVAL), (11, 4, EINVAL), (5, (1 << 24) + 1, EUNSUPPORTED), (6, (1 << 24) + 1, EINVAL)):
        args = list(good)
        args[at] = bad
        assert lib.accerl_dense_i8(*args) == code, (at, bad)
    assert lib.accerl_dense_i8(None, None, None, None, None, 0, 5, 100, 0, None, 1, 5, None) == 0
    assert lib.accerl_dense_i8(None, None, None, None, None, 3, 0, 100, 0, None, 1, 0, None) == 0
    n = A.accerl_dense_i8_workspace(3, 100)
    # x dtype ldx wq sw bias M N K relu out dtype ld ws bytes stream
    good = [p, 1, 100, p, p, None, 3, 5, 100, 0, p, 1, 5, p, n, None]
    for at, bad in ((0, None), (0, p + 1), (1, 3), (2, 99), (3, None), (4, None), (10, None), (12, 4), (13, None), (13, p + 8), (14, n - 1)):
        args = list(good)
        args[at] = bad
        assert lib.accerl_dense_i8_dynamic(*args) == EINVAL, (at, bad)


def loss_args(api, p, **change):
    from paper_2211_15023_amd import binding
    a = binding._PolicyLossArgs()
    for k, v in dict(B=3, A=5, dtype=0, kl_kind=2, logits=p, ld_logits=5, ref_logits=p, ld_ref=5, grad_logits=p + 4096, ld_grad=5, actions=p, old_logp=p,
                     advantages=p, clip_low=0.2, clip_high=0.2, scale=1.0, workspace=p, workspace_bytes=api.accerl_policy_loss_workspace()).items():
        setattr(a, k, v)
    for k, v in change.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), EINVAL), (dict(logits=2), EINVAL), (dict(actions=None), EINVAL), (dict(old_logp=None), EINVAL), (dict(advantages=None), EINVAL),
    (dict(ref_logits=None), EINVAL), (dict(kl_kind=1), EINVAL), (dict(kl_kind=4), EINVAL), (dict(kl_kind=-1), EINVAL), (dict(dtype=3), EINVAL),
    (dict(B=-1), EINVAL), (dict(A=0), EINVAL), (dict(ld_logits=4), EINVAL), (dict(ld_ref=4), EINVAL), (dict(ld_grad=4), EINVAL),
    (dict(mask=1, ld_mask=4), EINVAL), (dict(workspace=None), EINVAL), (dict(workspace_bytes=100), EINVAL),
    (dict(clip_low=-0.1), EINVAL), (dict(clip_low=1.1), EINVAL), (dict(clip_high=-0.1), EINVAL), (dict(clip_high=float("nan")), EINVAL),
    (dict(A=(1 << 20) + 1, ld_logits=1 << 21, ld_ref=1 << 21, ld_grad=1 << 21), EUNSUPPORTED), (dict(B=(1 << 31) + 1), EUNSUPPORTED),
    (dict(grad="overlap"), EINVAL), (dict(grad="other stride"), EINVAL), (dict(grad="reference"), EINVAL), (dict(out_loss=2), EINVAL), (dict(out_stats=1), EINVAL)])
def test_loss_refuses(A, change, code):
    lib = A.load_library()
    p, own = aligned(1 << 16)
    grad = change.get("grad")
    if grad is not None:
        change = {"overlap": dict(grad_logits=p + 8), "other stride": dict(grad_logits=p, ld_grad=6, ref_logits=p + 8192),
                  "reference": dict(grad_logits=p + 8192, ref_logits=p + 8192)}[grad]
    assert lib.accerl_policy_loss(C.byref(loss_args(A, p, **change)), None) == code
    assert "policy_loss" in A.accerl_last_error()


def test_loss_takes_nothing(A):
    lib = A.load_library()
    p, own = aligned(4096)
    assert lib.accerl_policy_loss(None, None) == EINVAL
    assert lib.accerl_policy_loss(C.byref(loss_args(A, p, B=0)), None) == 0
    # logits dtype ld mask ldm actions B A logp entropy ws bytes stream
    n = A.accerl_policy_loss_workspace()
    good = [p, 0, 5, None, 0, p, 3, 5, p, None, p, n, None]
    for at, bad in ((0, None), (0, p + 2), (1, 9), (2, 4), (5, None), (6, -1), (7, 0), (8, None), (8, p + 1), (10, None), (10, p + 4), (11, n - 1)):
        args = list(good)
        args[at] = bad
        assert lib.accerl_action_logprob(*args) == EINVAL, (at, bad)
    good[6] = 0
    assert lib.accerl_action_logprob(*good) == 0


@pytest.mark.parametrize("kl", ["none", "sampled", "forward", "reverse"])
def test_reference_gradient_against_differences(kl):
    """The formulas' gradient is the derivative of the formulas' loss: central differences in 64 bits, off by h^2 / 6 of the third derivative (here
    below 50) and by 2^-52 of the loss over h."""
    rng = np.random.default_rng(5)
    B, A, h = 6, 7, 1e-5
    z, zr = rng.normal(size=(B, A)), rng.normal(size=(B, A))
    mask = rng.random((B, A)) < 0.8
    act = rng.integers(0, A, B)
    mask[np.arange(B), act] = True
    old = ref.softmax_rows(z, mask)[0][np.arange(B), act] + rng.choice([-0.5, -0.1, 0.1, 0.5], B)
    kw = dict(mask=mask, w=rng.random(B) + 0.5, kl=kl, zr=zr, ref_lp=old + 0.3, clip_low=0.2, clip_high=0.25, ck=0.7, ch=0.3, scale=0.5)
    adv = rng.normal(size=B)
    g = ref.policy_loss(z, act, old, adv, **kw)["grad"]
    for b in range(B):
        for j in range(A):
            up, down = z.copy(), z.copy()
            up[b, j] += h
            down[b, j] -= h
            d = (ref.policy_loss(up, act, old, adv, **kw)["stats"][0] - ref.policy_loss(down, act, old, adv, **kw)["stats"][0]) / (2 * h)
            assert abs(d - g[b, j]) < 50 * h * h + 1e-14 / h, (b, j, d, g[b, j])
