"""An actor and a learner over a wide action set: the operators of wide policies as they are used together.

The actor's head is an int8 dense layer that quantises its inputs with a scale for each state (DenseInt8); it samples from the logits and
stores the log-probabilities of what it took (PolicyLoss.logprob).  The learner computes the logits again with its own weights, takes the
clipped loss with a KL term to the policy it started from (PolicyLoss.forward; the advantages are the round's rewards, normalised), continues
the gradient into the weights, and hands the actor the new ones, quantised anew (DenseInt8.update).  The task: every state has its own best
actions out of 2000, found by trying.

    python examples/wide_policy.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2211_15023_amd as A  # noqa: E402

FEATURES, ACTIONS, STATES = 64, 2000, 4096


def sample(logits, generator):
    """One action a row, as drawn from softmax(logits): the largest of logit + Gumbel noise."""
    u = torch.rand(logits.shape, generator=generator, device=logits.device).clamp_(1e-20, 1 - 1e-7)
    return (logits.float() - torch.log(-torch.log(u))).argmax(dim=1).to(torch.int32)


def main(rounds=60, epochs=2, say=print):
    A.load_library()
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    truth = draw(ACTIONS, FEATURES) / FEATURES ** 0.5             # the reward of action a in state x is truth[a] . x
    w = 0.01 * draw(ACTIONS, FEATURES)                            # the learner's weights
    start = w.to(torch.bfloat16)
    momentum = torch.zeros_like(w)
    head = A.DenseInt8(w)
    loss = A.PolicyLoss(clip_low=0.2, clip_high=0.25, kl="forward", kl_coef=1e-3, entropy_coef=1e-3)
    rewards = []
    for r in range(rounds):
        # the actor
        x = draw(STATES, FEATURES).to(torch.bfloat16)
        logits = head.forward(x)
        action = sample(logits, g)
        old_logp, entropy = loss.logprob(logits, action)
        reward = (truth[action.long()] * x).sum(dim=1)
        advantage = (reward - reward.mean()) / reward.std()
        # the learner
        reference = x @ start.t()
        for _ in range(epochs):
            own = x @ w.to(torch.bfloat16).t()
            got = loss.forward(own, action, old_logp, advantage, ref_logits=reference)
            momentum = 0.9 * momentum + (got.grad.t() @ x).float()
            w = w - 2.0 * momentum
        head.update(w)
        rewards.append(float(reward.mean()))
        if r % 10 == 0 or r == rounds - 1:
            _, kl, _, clipped = got.stats.tolist()
            say(f"round {r:3d}: reward {rewards[-1]:.3f}, KL to the start {kl:.3f}, entropy {float(entropy.mean()):.2f}, outside the borders {clipped:.1%}")
    return rewards


if __name__ == "__main__":
    main()
