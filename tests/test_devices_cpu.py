"""Entry points make their tensors' device current before they allocate or launch (one GPU is enough to run, none to test this)."""
import inspect

import pytest
import torch

from paper_2312_08874_amd import binding

ENTRIES = sorted(n for n, f in vars(binding).items() if inspect.isfunction(f) and n.startswith(("agent_", "prepare_")))


class _Devices:
    """torch's idea of the current device, without any."""

    def __init__(self, monkeypatch):
        self.current = 0
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.current, raising=False)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        outer = self

        class device:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.before, outer.current = outer.current, self.index

            def __exit__(self, *_):
                outer.current = self.before
        monkeypatch.setattr(torch.cuda, "device", device)


class _Tensor(torch.Tensor):
    def get_device(self):
        return self.at


def _tensor(device):
    t = torch.empty(1).as_subclass(_Tensor)
    t.at = device
    return t


def test_every_entry_point_is_covered():
    assert len(ENTRIES) >= 23
    for name in ENTRIES:
        assert hasattr(getattr(binding, name), "__wrapped__"), name


@pytest.mark.parametrize("first", [_tensor, lambda d: {"note": 5, "b1_col": None, "b1_row": _tensor(d)}])
def test_the_first_tensors_device_is_current_in_the_call_alone(monkeypatch, first):
    devices = _Devices(monkeypatch)

    @binding._on_its_device
    def entry(t, *a, **k):
        return devices.current, a, k
    for at in (0, 1, 3):
        devices.current = at
        for own in (0, 1, 3):
            assert entry(first(own), 5, key=6) == (own, (5,), {"key": 6}) and devices.current == at
            assert entry(t=first(own), key=6) == (own, (), {"key": 6}) and devices.current == at
        assert entry(first(-1))[0] == at      # not on a GPU: refused further on


def test_a_prepared_call_returns_to_the_device_it_was_prepared_on(monkeypatch):
    devices = _Devices(monkeypatch)
    seen = []

    def call(*args):
        seen.append((devices.current, args))
        return len(args)
    devices.current = 2
    prepared = binding.PreparedCall(call, "call", (), None)
    prepared()
    devices.current = 0
    prepared()
    assert seen == [(2, ()), (2, ())] and devices.current == 0
    with pytest.raises(binding.AgentAttnError):
        binding.PreparedCall(lambda: -2, "call", (), None)()
