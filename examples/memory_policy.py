"""An actor and a learner whose policy remembers: the operators of policies with a memory as they are used together.

The policy is one block: a norm, projections, linear attention with a decay for each head (LinearAttention), its heads normed and gated (BlockNorm with groups), a
projection, and the block's end with the norm before the logits (BlockNorm).  The actor goes step by step and carries the memory from one unroll to the
next; the learner works on a whole unroll at once, from the memory that the actor began it with, takes the clipped loss (PolicyLoss) and continues the
operators' gradients into the weights.  The task: a sign is shown when an episode begins and asked for at its end; with nothing remembered every answer is a guess.

    python examples/memory_policy.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2211_15023_amd as A  # noqa: E402

SIGNS, WIDTH, HEADS, DIM = 8, 64, 4, 16
ENVIRONMENTS, EPISODE, UNROLL = 256, 12, 30


class Policy:
    DECAY = [0.9, 0.97, 0.99, 0.999]

    def __init__(self, generator):
        draw = lambda *s: torch.randn(s, generator=generator, device="cuda") / s[0] ** 0.5
        inner = HEADS * DIM
        # columns of wide: queries, keys, values, gate
        self.weights = dict(embed=draw(SIGNS + 2, WIDTH), wide=draw(WIDTH, 4 * inner), back=draw(inner, WIDTH), out=0.1 * draw(WIDTH, SIGNS),
                            first=torch.ones(WIDTH, device="cuda"), heads=torch.ones(inner, device="cuda"), last=torch.ones(WIDTH, device="cuda"))
        self.memory = A.LinearAttention(self.DECAY, scale=DIM ** -0.5)
        self.first = A.BlockNorm(WIDTH, before=self.weights["first"])
        self.heads = A.BlockNorm(inner, after=self.weights["heads"], gate="silu", groups=HEADS)
        self.last = A.BlockNorm(WIDTH, before=self.weights["last"])

    def project(self, h):
        q, k, v, gate = (h @ self.weights["wide"]).chunk(4, dim=-1)
        return *(t.unflatten(-1, (HEADS, DIM)) for t in (q, k, v)), gate

    def step(self, seen, state, reset):
        """One step of every environment: logits; the memory is updated in place."""
        w = self.weights
        x, h = self.first.forward(seen @ w["embed"])
        q, k, v, gate = self.project(h)
        o = self.memory.step(q, k, v, state, reset=reset)
        m, _ = self.heads.forward(o.flatten(1), gate=gate)
        return self.last.forward(m @ w["back"], x=x)[1] @ w["out"]

    def learn(self, seen, state, reset, loss):
        """Gradients of an unroll, by the weights' names; loss: logits [B T, actions] -> their gradient."""
        B, T, _ = seen.shape
        w = {n: t.requires_grad_() for n, t in self.weights.items()}
        leaf = lambda t: t.detach().requires_grad_()
        for t in w.values():
            t.grad = None
        # forwards; what the operators return begins a graph of its own
        x = (seen @ w["embed"]).flatten(0, 1)
        u, h = self.first.forward(x)
        h = leaf(h)
        q, k, v, gate = self.project(h.unflatten(0, (B, T)))
        gate = gate.flatten(0, 1)
        o, _ = self.memory.forward(q, k, v, state=state, reset=reset)
        o = o.flatten(2).flatten(0, 1)
        m = leaf(self.heads.forward(o, gate=gate)[0])
        y = m @ w["back"]
        hh = leaf(self.last.forward(y, x=u)[1])
        logits = hh @ w["out"]
        # and back
        torch.autograd.backward([logits], [loss(logits.detach())])
        end = self.last.backward(y, x=u, grad_h=hh.grad)
        torch.autograd.backward([y], [end.y])
        heads = self.heads.backward(o, gate=gate, grad_u=m.grad)
        r = self.memory.backward(heads.y.view(B, T, HEADS, DIM), q, k, v, state=state, reset=reset)
        torch.autograd.backward([q, k, v, gate], [r.q, r.k, r.v, heads.gate])
        begin = self.first.backward(x, grad_u=end.x, grad_h=h.grad)
        torch.autograd.backward([x], [begin.y])
        grads = {n: t.grad for n, t in w.items() if t.grad is not None}
        for t in w.values():
            t.requires_grad_(False)
        return dict(grads, first=begin.before, heads=heads.after, last=end.before)

    def update(self):
        """The norms take the weights as they are now."""
        self.first.update(before=self.weights["first"])
        self.heads.update(after=self.weights["heads"])
        self.last.update(before=self.weights["last"])


def main(rounds=40, epochs=4, say=print):
    A.load_library()
    g = torch.Generator(device="cuda").manual_seed(1)
    policy = Policy(g)
    loss = A.PolicyLoss(clip_low=0.2, clip_high=0.2)
    optimizer = torch.optim.Adam(policy.weights.values(), lr=3e-3)
    B, T = ENVIRONMENTS, UNROLL
    state = torch.zeros((B, HEADS, DIM, DIM), device="cuda")
    age = torch.randint(0, EPISODE, (B,), generator=g, device="cuda")            # of an environment's episode
    sign = torch.randint(0, SIGNS, (B,), generator=g, device="cuda")
    rewards = []
    for i in range(rounds):
        # the actor
        before = state.clone()
        steps = []
        for _ in range(T):
            begins, asks = age == 0, age == EPISODE - 1
            sign = torch.where(begins, torch.randint(0, SIGNS, (B,), generator=g, device="cuda"), sign)
            seen = torch.zeros((B, SIGNS + 2), device="cuda")
            seen[:, :SIGNS] = torch.nn.functional.one_hot(sign, SIGNS) * begins[:, None]
            seen[:, SIGNS], seen[:, SIGNS + 1] = asks.float(), 1.0
            reset = begins.to(torch.uint8)
            logits = policy.step(seen, state, reset)
            u = torch.rand(logits.shape, generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)
            action = (logits - torch.log(-torch.log(u))).argmax(dim=1).to(torch.int32)
            logp, _ = loss.logprob(logits, action)
            steps.append((seen, reset, action, logp, (action == sign).float() * asks, asks))
            age = (age + 1) % EPISODE
        seen, reset, action, logp, reward, asked = (torch.stack(t, dim=1) for t in zip(*steps))
        mean = float(reward.sum() / asked.sum())
        advantage = ((reward - mean) * asked).flatten()
        # the learner
        for _ in range(epochs):
            grads = policy.learn(seen, before, reset, lambda x: loss.forward(x, action.flatten(), logp.flatten(), advantage).grad)
            for n, t in policy.weights.items():
                t.grad = grads[n]
            optimizer.step()
            policy.update()
        rewards.append(mean)
        if i % 10 == 0 or i == rounds - 1:
            say(f"round {i:3d}: {mean:.1%} of the signs remembered")
    return rewards


if __name__ == "__main__":
    main()
