"""The example of the operators of wide policies learns its task."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_learns():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import wide_policy
    finally:
        sys.path.pop(0)
    rewards = wide_policy.main(rounds=30, say=lambda *_: None)
    # rewards of a random action: mean 0, spread 1 / sqrt(4096) over a round's mean
    assert abs(rewards[0]) < 0.2 and rewards[-1] > rewards[0] + 0.3, rewards
