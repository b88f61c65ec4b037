"""A workspace that two threads' calls grow at the same time, on the CPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def test_a_call_gets_what_it_asked_for(B):
    """Whatever another thread's call puts in place between a growth and its return, or between the look and the return."""
    class Contended(B.Workspace):
        @property
        def buf(self):
            return self.held

        @buf.setter
        def buf(self, t):
            self.held = t
            if t.numel() > 1 << 20:  # the other thread, whose call saw the small buffer too
                self.held = torch.zeros(1 << 17, dtype=torch.uint8)
    ws = Contended(torch.device("cpu"))
    assert ws.get(1 << 16).numel() == 1 << 16
    assert ws.get(2 << 20).numel() >= 2 << 20
    assert ws.get(1 << 17).numel() >= 1 << 17
