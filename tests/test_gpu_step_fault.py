"""The mark that a bounded wait leaves when it runs out."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu


def test_the_mark_is_read_after_what_any_stream_has_been_given():
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    step.fault()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)      # a tenth of a second
        done.record()
    assert not step.fault()
    assert done.query()
