"""The rotary table on the device that it belongs to: a launch on another one would write to an address that is not its own.  No GPU: stand-ins for tensors and devices."""
import contextlib

import pytest
import torch

from paper_2511_05534_b200 import binding as F


class Table:
    """What a call looks at of a tensor."""
    dtype, is_cuda = torch.int64, True

    def __init__(self, pairs, index, at=1 << 20):
        self.shape, self.device, self.at = (pairs,), torch.device("cuda", index), at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


class Library:
    def __init__(self):
        self.seen = []

    def flowmm_rotary_table(self, p, table, stream):
        self.seen.append((table, stream, torch.cuda.current_device()))
        return 0


@pytest.fixture
def two_devices(monkeypatch):
    """Device 0 is the current one; streams are named after their devices."""
    now, lib = [0], Library()

    @contextlib.contextmanager
    def device(d):
        index = torch.device(d).index
        before, now[0] = now[0], now[0] if index is None else index
        yield
        now[0] = before
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    monkeypatch.setattr(F, "load", lambda: lib)
    return lib


def test_a_table_elsewhere_is_refused(two_devices):
    p = F.RotaryParams(1, 1, 1, 64, 1)
    F.flowmm_rotary_table(p, Table(32, 0))
    assert two_devices.seen == [(1 << 20, 100, 0)]
    with pytest.raises(ValueError, match="current device"):
        F.flowmm_rotary_table(p, Table(32, 1))
    assert len(two_devices.seen) == 1


def test_a_table_is_allocated_and_written_where_it_is_asked_for(two_devices, monkeypatch):
    p = F.RotaryParams(1, 1, 1, 64, 1)
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: Table(n, torch.cuda.current_device() if torch.device(device).index is None else torch.device(device).index))
    for device, index in (("cuda", 0), ("cuda:0", 0), ("cuda:1", 1), (torch.device("cuda", 1), 1)):
        assert F.alloc_rotary_table(p, device).device.index == index
        assert two_devices.seen.pop() == (1 << 20, 100 + index, index)
        assert torch.cuda.current_device() == 0


def test_a_table_on_the_cpu_is_refused():
    p = F.RotaryParams(1, 1, 1, 64, 1)
    with pytest.raises(ValueError, match="CUDA"):
        F.flowmm_rotary_table(p, torch.zeros(32, dtype=torch.int64))
