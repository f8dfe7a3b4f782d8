"""The sequence operators run together as they would be used: actors, replay buffer and learner of examples/replay_sequences.py."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_actors_learn_from_replayed_stretches():
    import replay_sequences
    losses = replay_sequences.main(iterations=80, report=None)
    early, late = sum(losses[:5]) / 5, sum(losses[-5:]) / 5
    # a policy without memory cannot get below MEMORY^2 of the targets' variance
    assert early > 2 * late and late < 0.5 * replay_sequences.MEMORY ** 2 * early, (early, late)
