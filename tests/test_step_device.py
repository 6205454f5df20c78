"""Which device is current after a call, with stand-ins for the library and for two devices."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import step


class Library:
    """Calls that leave device 1 current, as the C functions do with the device in their arguments."""
    def __init__(self, status):
        self.status, self.current = status, 0

    def halos_rope(self, args):
        self.current = 1
        return self.status

    def halos_step_fault(self, device, out):
        self.current = device
        return self.status

    def halos_step_error(self):
        return b"as asked"


@pytest.mark.parametrize("status", [0, 4])
@pytest.mark.parametrize("call", [lambda: step._call("halos_rope", b"", 1), lambda: step.fault(1)])
def test_the_callers_device_stays_current(monkeypatch, call, status):
    lib = Library(status)
    monkeypatch.setattr(step, "_lib", lib)
    monkeypatch.setattr(step, "_current_device", lambda: lib.current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: lib.current)
    monkeypatch.setattr(step, "_set_device", lambda d: setattr(lib, "current", d))
    if status:
        with pytest.raises(step.HalosError):
            call()
    else:
        call()
    assert lib.current == 0
