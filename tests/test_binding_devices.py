"""What the binding does with devices, memory and streams, seen on the CPU: the
tensors are stand-ins without memory (FakeTensor), the library is a recorder that
launches nothing."""
from __future__ import annotations


import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2606_28560_gb300 as fa
from paper_2606_28560_gb300 import binding as B

BF, F32, I64, U8 = torch.bfloat16, torch.float32, torch.int64, torch.uint8


class Library:
    """Every ..._bytes function asks for 1000 bytes; every other call is recorded and succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 1000
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def library(monkeypatch):
    """A library that records, on a machine whose current device is cuda:0."""
    rec = Library()
    monkeypatch.setattr(B, "lib", lambda: rec)
    monkeypatch.setattr(B, "_residual_bytes", lambda *a: 1000)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: 256)
    with FakeTensorMode():
        yield rec


def xent(device):
    x, w = torch.empty(4, 8, dtype=BF, device=device), torch.empty(16, 8, dtype=BF, device=device)
    return x, w, torch.empty(4, dtype=I64, device=device)


def row(device, n=4):
    return torch.empty(n, dtype=F32, device=device)


def heads(device, n):
    return [torch.empty(1, 2, 16, 64, dtype=BF, device=device) for _ in range(n)]


OFFSETS = np.array([1.0, 2.0, 3.0], dtype=np.float32)

# every compute call of the binding, on tensors of one device
CALLS = {
    "linear_xent_fwd": lambda d, **k: fa.linear_xent_fwd(*xent(d), **k),
    "linear_xent_bwd": lambda d, **k: fa.linear_xent_bwd(*xent(d), row(d), row(d), **k),
    "clip_grads": lambda d, **k: fa.clip_grads([row(d), row(d, 9)], 1.0, **k),
    "grad_norm": lambda d, **k: fa.grad_norm([row(d), row(d, 9)], **k),
    "fwd": lambda d, **k: fa.fwd(*heads(d, 3), 1.0, OFFSETS, 8, **k),
    "bwd": lambda d, **k: fa.bwd(*heads(d, 3), torch.empty(1, 2, 16, dtype=F32, device=d), *heads(d, 1), 1.0, OFFSETS, 8, **k),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_of_the_current_device(name, library):
    CALLS[name]("cuda:0")
    assert len(library.calls) == 1


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_of_another_device_are_refused(name, library):
    with pytest.raises(ValueError, match="current device is cuda:0"):
        CALLS[name]("cuda:1")
    assert not library.calls


@pytest.mark.parametrize("given", ["k", "out", "lse"])
def test_attention_tensors_of_two_devices_are_refused(given, library):
    q, k, v = heads("cuda:0", 3)
    other = {"k": heads("cuda:1", 1)[0], "out": heads("cuda:1", 1)[0], "lse": torch.empty(1, 2, 16, device="cuda:1")}[given]
    with pytest.raises(ValueError, match="one CUDA device"):
        if given == "k":
            fa.fwd(q, other, v, 1.0, OFFSETS, 8)
        else:
            fa.fwd(q, k, v, 1.0, OFFSETS, 8, **{given: other})
    assert not library.calls


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("kind", ["cpu", "another device", "strided", "expanded"])
def test_workspaces_that_are_not_the_devices_memory_are_refused(kind, name, library):
    device = {"cpu": "cpu", "another device": "cuda:1"}.get(kind, "cuda:0")
    ws = {"strided": lambda: torch.empty(8192, dtype=U8, device=device)[::2],
          "expanded": lambda: torch.empty(1, dtype=U8, device=device).expand(4096)}.get(
              kind, lambda: torch.empty(4096, dtype=U8, device=device))()
    with pytest.raises(ValueError, match="workspace"):
        CALLS[name]("cuda:0", workspace=ws)
    assert not library.calls


@pytest.mark.parametrize("name", list(CALLS))
def test_a_workspace_of_the_device_is_used(name, library):
    CALLS[name]("cuda:0", workspace=torch.empty(4096, dtype=U8, device="cuda:0"))
    assert len(library.calls) == 1
