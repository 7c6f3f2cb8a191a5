"""ops.check takes a device as torch does: a number, a torch.device or a name,
with an index or without."""
import pytest
import torch

from paper_2608_15438_gb300 import neuroute as nr
from paper_2608_15438_gb300 import ops


@pytest.fixture
def asked(monkeypatch):
    seen = []

    class Lib:
        @staticmethod
        def nr_ops_status(device):
            seen.append(device)
            return 0

    monkeypatch.setattr(nr, "lib", lambda: Lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    return seen


def test_devices(asked):
    for d in (2, torch.device("cuda", 2), torch.device("cuda:2"), "cuda:2"):
        ops.check(d)
    ops.check()
    ops.check(torch.device("cuda"))  # the current one
    ops.check("cuda")
    assert asked == [2, 2, 2, 2, 0, 3, 3] and all(type(d) is int for d in asked)


def test_other_devices_are_refused(asked):
    for d in ("cpu", torch.device("cpu")):
        with pytest.raises(ValueError, match="CUDA"):
            ops.check(d)
    assert asked == []
