"""Tensors on another device than the current one, without a device: the handle of a default stream is 0 everywhere and names the current device's."""
import pytest

from paper_2407_09453_amd import binding, f8


class _Tensor:
    is_cuda = True

    def __init__(self, at):
        self.device = at

    def get_device(self):
        return self.device


@pytest.fixture
def devices(monkeypatch):
    """Two devices, 0 the current one; side streams by their handle."""
    import torch
    state = {"now": 0, "streams": {0: 0, 1: 0}, "set": []}
    monkeypatch.setattr(binding, "_raw_stream", lambda d: state["streams"][d])
    monkeypatch.setattr(binding, "_several", None)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["now"])
    return state


def test_a_default_stream_elsewhere_is_refused(devices):
    assert binding._current_stream(_Tensor(0)) == 0
    with pytest.raises(RuntimeError, match="cuda:1, but the current device is cuda:0"):
        binding._current_stream(_Tensor(1))
    devices["streams"][1] = 77  # a stream of its own says where it belongs
    assert binding._current_stream(_Tensor(1)) == 77
    devices["streams"][1], devices["now"] = 0, 1
    assert binding._current_stream(_Tensor(1)) == 0


def test_one_device_is_not_asked_about(devices, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: pytest.fail("asked"))
    assert binding._current_stream(_Tensor(0)) == 0 and binding._several is False


@pytest.mark.parametrize("handle", [0, 55])
def test_a_stream_given_by_handle_brings_its_device(devices, monkeypatch, handle):
    """... and the call runs with that device current, whether the handle is that of its current stream or not."""
    import torch

    class Stream:
        def __init__(self, handle, device):
            self.handle, self.device = handle, type("D", (), {"index": device})

    def set_stream(s):
        devices["now"], devices["streams"][s.device.index] = s.device.index, s.handle
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d: Stream(devices["streams"][d], d))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d: Stream(0, d))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device: Stream(h, device))
    monkeypatch.setattr(torch.cuda, "set_stream", set_stream)
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: devices.update(now=d))
    t = _Tensor(1)
    seen = []
    f8._on_stream(handle, t, lambda: seen.append((devices["now"], binding._current_stream(t))))
    assert seen == [(1, handle)] and devices["now"] == 0 and devices["streams"] == {0: 0, 1: 0}
