"""The example of the operators of policies with a memory: it runs, and its gradients are those of the same policy in 64 bits."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import memory_policy
    finally:
        sys.path.pop(0)
    return memory_policy


def test_example_runs(example):
    said = []
    rewards = example.main(rounds=3, say=said.append)
    assert len(rewards) == 3 and all(math.isfinite(r) and 0 <= r <= 1 for r in rewards) and len(said) == 2


def _logits(example, w, seen, state, reset):
    """The policy token by token in 64 bits, and its memory at the end."""
    H, D = example.HEADS, example.DIM
    rms = lambda z: torch.nn.functional.rms_norm(z, z.shape[-1:], eps=1e-6)
    decay = torch.tensor(example.Policy.DECAY, dtype=torch.float64, device="cuda").view(1, H, 1, 1)
    rows = []
    for t in range(seen.shape[1]):
        x = seen[:, t] @ w["embed"]
        q, k, v, gate = ((rms(x) * w["first"]) @ w["wide"]).chunk(4, dim=-1)
        q, k, v = (z.unflatten(-1, (H, D)) for z in (q, k, v))
        state = torch.where(reset[:, t].view(-1, 1, 1, 1) != 0, 0.0, state) * decay + k[..., None] * v[..., None, :]
        o = (q[..., None] * state).sum(-2) * D ** -0.5
        m = rms(o).flatten(1) * w["heads"] * torch.nn.functional.silu(gate)
        rows.append((rms(x + m @ w["back"]) * w["last"]) @ w["out"])
    return torch.stack(rows, dim=1), state


def test_gradients_of_the_example(example):
    g = torch.Generator(device="cuda").manual_seed(5)
    policy = example.Policy(g)
    B, T = 6, 40
    seen = torch.randn((B, T, example.SIGNS + 2), generator=g, device="cuda")
    reset = (torch.rand((B, T), generator=g, device="cuda") < 0.1).to(torch.uint8)
    state = torch.randn((B, example.HEADS, example.DIM, example.DIM), generator=g, device="cuda")
    by = torch.randn((B * T, example.SIGNS), generator=g, device="cuda")
    leaf = {n: t.double().requires_grad_() for n, t in policy.weights.items()}
    logits, last = _logits(example, leaf, seen.double(), state.double(), reset)
    torch.autograd.backward([logits], [by.view(logits.shape).double()])
    got = []

    def loss(x):
        got.append(x)
        return by
    grads = policy.learn(seen, state, reset, loss)
    # fp32 throughout, roundings of 2^-24 through a handful of layers and products of up to 256 terms: 2-norms
    near = lambda a, b, n: (a.double() - b).norm() <= 2e-5 * b.norm() or pytest.fail(f"{n}: {float((a.double() - b).norm() / b.norm())}")
    near(got[0], logits.detach().flatten(0, 1), "logits")
    assert set(grads) == set(leaf)
    for n, t in leaf.items():
        near(grads[n], t.grad, n)
    # the actor's steps
    carried = state.clone()
    rows = torch.stack([policy.step(seen[:, t], carried, reset[:, t]) for t in range(T)], dim=1)
    near(rows, logits.detach(), "steps")
    near(carried, last.detach(), "memory")
