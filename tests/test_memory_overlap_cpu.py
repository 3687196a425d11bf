"""Outputs of the operators of policies with a memory that overlap inputs or each other: the host's test of strided tensors against one byte by byte, and what the calls
refuse (they look at addresses only)."""
import ctypes as C
import random
import subprocess

import pytest

from tests.test_memory_ops_cpu import EINVAL, attention_args, norm_args
from tests.test_wide_ops_cpu import aligned

SOURCE = r"""
#include "tables.h"
extern "C" int overlap(const int64_t* a, const int64_t* b) {
    using namespace accerl;
    auto of = [](const int64_t* x) { return Strided((const void*)x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]); };
    return share(of(a), of(b));
}
"""


def test_strided_tensors_against_their_bytes(tmp_path):
    from paper_2211_15023_amd import build
    (tmp_path / "t.cpp").write_text(SOURCE)
    subprocess.run([build.CXX, "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t.so")],
                   check=True)
    f = C.CDLL(str(tmp_path / "t.so")).overlap
    call = lambda a, b: bool(f((C.c_int64 * 8)(*a), (C.c_int64 * 8)(*b)))
    rng = random.Random(3)
    seen = [0, 0]

    def tensor(like):
        n = [rng.choice((1, 1, 2, 3, 5)) if rng.random() < 0.98 else 0 for _ in range(3)]
        if like and rng.random() < 0.6:                       # strides of the other one, as parts of one buffer have
            steps = [like[2 * i + 2] for i in range(3)]
        elif rng.random() < 0.5:                              # dense, in some order
            steps, run = [0, 0, 0], 4
            for i in rng.sample(range(3), 3):
                steps[i] = run
                run *= max(n[i], 1) + rng.choice((0, 0, 1))
        else:
            steps = [rng.randint(-30, 60) for _ in range(3)]
        return [rng.randint(400, 620), n[0], steps[0], n[1], steps[1], n[2], steps[2], rng.randint(1, 6)]

    def places(x):
        return {x[0] + i * x[2] + j * x[4] + k * x[6] + e for i in range(x[1]) for j in range(x[3]) for k in range(x[5]) for e in range(x[7])}
    for _ in range(60000):
        a = tensor(None)
        b = tensor(a)
        both = bool(places(a) & places(b))
        assert call(a, b) == both and call(b, a) == both, (a, b)
        seen[both] += 1
    assert min(seen) > 10000
    # heads of 64 floats, tokens and batches of rows that both are parts of: none shared, and all of them with one column more
    row, at = 4 * 1000, 1 << 40
    for batch, token in ((5000 * row, row), (row, 700 * row)):                            # (a part of 5000 tokens, and of 700 environments)
        q = [at, 512, batch, 4096, token, 8, 256, 256]
        assert not call(q, [at + 2048, 512, batch, 4096, token, 4, 256, 256]) and call(q, [at + 2044, 512, batch, 4096, token, 4, 256, 256])
    assert not call([0, 2, 8, 1, 0, 1, 0, 8], [0, 2, 8, 1, 0, 1, 0, 8])                   # nowhere


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


# places of attention_args: log_decay, reset and lengths at p, with q; k 4096, v 8192, state 12288, out 20480, out_state 24576, grad_out 32768, grad_out_state 36864, grad_q 45056,
# grad_k 49152, grad_v 53248, grad_state 57344; a workspace that lies apart
TOKENS, STATES = {"q": 0, "k": 4096, "v": 8192}, 4096
APART = 1 << 16


def _refused(A, name, **change):
    p, own = aligned(1 << 18)
    change = {k: p + v if k != "workspace_bytes" else v for k, v in change.items()}
    change.setdefault("workspace", p + APART)
    assert getattr(A.load_library(), "accerl_" + name)(C.byref(attention_args(p, **change)), None) == EINVAL
    return A.accerl_last_error()


@pytest.mark.parametrize("name", ["linear_attention", "linear_attention_step"])
@pytest.mark.parametrize("at", [0, 4096, 8192, 12288, 12288 + 64, 12288 + STATES - 16, 24576, 24576 + STATES - 16])
def test_outputs_over_tokens_and_states(A, name, at):
    assert "overlap" in _refused(A, name, out=at)
    if at < 24576 and at != 12288:                            # (neither the state itself nor its own place)
        assert "overlap" in _refused(A, name, out_state=at // 16 * 16)


@pytest.mark.parametrize("name,which", [("linear_attention", "log_decay"), ("linear_attention", "reset"), ("linear_attention", "lengths"), ("linear_attention_step", "log_decay"),
                                        ("linear_attention_step", "reset")])
def test_outputs_over_what_else_a_call_reads(A, name, which):
    assert "overlap" in _refused(A, name, **{which: 20480 + 16})
    assert "overlap" in _refused(A, name, **{which: 24576 + 32})


GRADS = {"grad_q": 45056, "grad_k": 49152, "grad_v": 53248, "grad_state": 57344}


@pytest.mark.parametrize("which,at", [(w, at) for w in GRADS for at in (0, 4096, 8192, 12288, 12288 + STATES - 32, 32768, 36864, 36864 + 128, *GRADS.values(), 57344 + STATES - 32)
                                      if at // 4096 != GRADS[w] // 4096])
def test_gradients_over_tokens_states_and_each_other(A, which, at):
    assert "overlap" in _refused(A, "linear_attention_grad", **{which: at})


@pytest.mark.parametrize("which", ["log_decay", "reset", "lengths"])
@pytest.mark.parametrize("at", [45056 + 16, 57344 + 16])
def test_gradients_over_what_else_a_call_reads(A, which, at):
    assert "overlap" in _refused(A, "linear_attention_grad", **{which: at})


@pytest.mark.parametrize("at", [0, 4096, 8192, 12288, 32768, 36864, 45056, 49152, 53248, 57344])
def test_a_workspace_over_what_a_call_has(A, at):
    """(of the gradients of shared heads: 2 x 3 tokens of 4 heads of 8 and 16 floats)"""
    assert "workspace" in _refused(A, "linear_attention_grad", workspace=at)


def test_parts_of_wider_rows(A):
    """An output between or over columns of the rows that the tokens are parts of, of some of their tokens only."""
    from paper_2211_15023_amd import binding
    p, own = aligned(1 << 20)
    s = lambda h: binding._TokenStride(10 * 400, 400, h)                                  # rows of 400 floats, 10 a batch, of which 3 are taken
    rows = dict(q=p, k=p + 4 * 32, v=p + 4 * 48, q_stride=s(8), k_stride=s(8), v_stride=s(16), out_stride=s(16))
    far = {k: p + (1 << 18) + i * 8192 for i, k in enumerate(("log_decay", "reset", "lengths", "state", "out_state", "workspace"))}
    for name in ("linear_attention", "linear_attention_step"):
        for at in (0, 16, 31, 32, 47, 79):                                                # (q 0 .. 31, k 32 .. 47, v 48 .. 79)
            a = attention_args(p, **rows, **far, out=p + 4 * at)
            assert getattr(A.load_library(), "accerl_" + name)(C.byref(a), None) == EINVAL and "overlap" in A.accerl_last_error(), at


def test_a_step_of_wide_heads_over_its_tokens(A):
    """Heads of 128: columns of one workgroup would be written before another has read the query whole."""
    from paper_2211_15023_amd import binding
    p, own = aligned(1 << 22)
    s = binding._TokenStride(512, 512, 128)
    good = dict(B=2, T=1, H=4, Hk=4, Dk=128, Dv=128, q_stride=s, k_stride=s, v_stride=s, out_stride=s, log_decay=p, reset=None, lengths=None,
                **{n: p + (i + 1) * (1 << 19) for i, n in enumerate(("q", "k", "v", "state", "out_state"))})
    for n in "qkv":
        a = attention_args(p, **dict(good, out=good[n]))
        assert A.load_library().accerl_linear_attention_step(C.byref(a), None) == EINVAL and "overlap" in A.accerl_last_error()


# ------------------------------------------------------------------ norms: places of norm_args (3 rows of 20: y 0, x 1024, gate 2048, out_u 4096, out_h 5120, grad_u 6144, grad_h 7168,
# grad_y 8192, grad_x 9216, grad_gate 10240, grad_after 11264, grad_before 12288), the weights and the workspace apart
NORM = dict(after=16384, before=17408, workspace=32768)


def _norm_refused(A, name, **change):
    p, own = aligned(1 << 17)
    a = norm_args(p, workspace_bytes=1 << 16, **{k: p + v for k, v in {**NORM, **change}.items()})
    assert getattr(A.load_library(), "accerl_" + name)(C.byref(a), None) == EINVAL
    return A.accerl_last_error()


@pytest.mark.parametrize("which", ["after", "before"])
@pytest.mark.parametrize("at", [4096, 4096 + 160, 5120, 5120 + 40])
def test_norms_over_their_weights(A, which, at):
    assert "overlaps" in _norm_refused(A, "block_norm", **{which: at})


@pytest.mark.parametrize("which", ["after", "before"])
@pytest.mark.parametrize("at", [8192, 8192 + 116, 9216, 9216 + 236, 10240])
def test_gradients_of_norms_over_the_weights(A, which, at):
    assert "overlaps" in _norm_refused(A, "block_norm_grad", **{which: at})


@pytest.mark.parametrize("which,at", [(w, at) for w in ("grad_after", "grad_before") for at in (0, 1024, 2048 + 40, 6144, 7168, 8192, 9216 + 80, 10240, 16384 + 4, 17408 - 4)] +
                         [("grad_after", 12288), ("grad_after", 12288 - 4), ("grad_before", 11264), ("grad_before", 11264 + 76)])
def test_weights_gradients_over_rows_and_weights_in_part(A, which, at):
    assert "overlap" in _norm_refused(A, "block_norm_grad", **{which: at})


@pytest.mark.parametrize("at", [0, 1024, 2048, 6144, 7168, 8192, 9216, 10240, 11264, 12288, 16384, 17408])
def test_a_norms_workspace_over_what_a_call_has(A, at):
    assert "workspace" in _norm_refused(A, "block_norm_grad", workspace=at)
