"""CPU checks of what the binding of the eight-bit operators does by itself."""
from types import SimpleNamespace

import pytest
import torch

from paper_2607_27042_amd import binding


def test_tensors_and_streams_of_one_device(monkeypatch):
    """A launch goes to the current device: what lies on another one is refused."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    on = [SimpleNamespace(device=torch.device("cuda", i)) for i in range(2)]
    host = torch.zeros(1)
    binding._one_device("f", (on[0], None, on[0], host), None)
    binding._one_device("f", (on[0],), on[0])
    for tensors, stream in (((on[0], on[1]), None), ((on[1], on[1]), None), ((on[0],), on[1])):
        with pytest.raises(ValueError, match="f: a tensor or the stream is on cuda:1"):
            binding._one_device("f", tensors, stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    binding._one_device("f", (on[1], on[1]), on[1])


def test_every_call_checks_its_device(monkeypatch):
    seen = []
    monkeypatch.setattr(binding, "_one_device", lambda name, tensors, stream: seen.append((name, tensors, stream)))
    monkeypatch.setattr(binding, "load", lambda: SimpleNamespace(f=lambda *a: 0))
    binding._enqueue("f", (1, 2), ("t",), "s", False)
    assert callable(binding._enqueue("f", (1,), ("u",), None, True))
    assert seen == [("f", ("t",), "s"), ("f", ("u",), None)]


def test_slots_of_positions_outside():
    """Positions before the first token, past the table and in pages that are none have no slot."""
    cache = object.__new__(binding.Cache)
    cache.page_size = 16
    table = torch.tensor([[3, 0, -1], [5, 2, 7]], dtype=torch.int32)
    slots = cache.slots(table, torch.tensor([-3, 46], dtype=torch.int32), 5)
    assert slots.tolist() == [-1, -1, -1, 48, 49, 7 * 16 + 14, 7 * 16 + 15, -1, -1, -1]
    assert cache.slots(table, torch.tensor([30, -2 ** 31], dtype=torch.int32), 3).tolist() == [14, 15, -1, -1, -1, -1]
    assert cache.slots(table[:, :0], torch.tensor([0, 1], dtype=torch.int32), 2).tolist() == [-1] * 4
