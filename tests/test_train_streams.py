"""Streams given to the training operators, as far as that needs no GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2410_05589_b200 import binding as b


def test_a_stream_of_another_device_is_refused(monkeypatch):
    here = torch.device("cuda", 0)
    for current in (0, 1):
        monkeypatch.setattr(b, "_device", lambda: current)
        with pytest.raises(b.PsError, match="another device"):
            b._on(here, SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))


def test_the_current_stream_of_the_tensors_device_needs_nothing(monkeypatch):
    monkeypatch.setattr(b, "_device", lambda: 0)
    assert b._on(torch.device("cuda", 0), None) is b._HERE
