"""The local step's operators together, as a worker runs them: the loss falls, and no bounded wait ran out."""
from __future__ import annotations

import pytest

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu


def test_workers_train_a_decoder_through_the_hierarchy():
    from paper_2506_04531_b200.examples import local_steps
    losses, counters = local_steps.run(rounds=48, log=None)
    first, last = sum(losses[:4]) / 4, sum(losses[-4:]) / 4
    assert last < 0.8 * first, (first, last)
    assert counters["t"] > 0
    assert not step.fault()
