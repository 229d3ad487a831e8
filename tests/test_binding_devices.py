"""What the binding does with devices, memory and streams, seen on the CPU: the
tensors are stand-ins without memory (FakeTensor), the library is a recorder that
launches nothing."""
from __future__ import annotations


import contextlib

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
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
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


class Stream:
    """A stand-in stream; `now` is the current one."""
    device, device_index = torch.device("cuda:0"), 0

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def streams(library, monkeypatch):
    """(caller's stream, another, what was allocated under which stream, what was recorded with which)."""
    caller, other, now, allocated, recorded = Stream(11), Stream(22), [], [], []
    now.append(caller)

    @contextlib.contextmanager
    def under(s):
        now.append(s)
        yield
        now.pop()

    def logged(make):
        def call(*a, **k):
            t = make(*a, **k)
            allocated.append((t, now[-1]))
            return t
        return call

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(B, "_raw_stream", lambda index: now[-1].cuda_stream)
    monkeypatch.setattr(torch, "empty", logged(torch.empty))
    monkeypatch.setattr(torch, "empty_like", logged(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append((t, s)))
    return caller, other, allocated, recorded


def flat(values):
    for v in values:
        if torch.is_tensor(v):
            yield v
        elif isinstance(v, (list, tuple)):
            yield from flat(v)


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_of_a_call_on_another_stream(name, library, streams, monkeypatch):
    caller, other, allocated, recorded = streams
    given = []
    for f in ("linear_xent_fwd", "linear_xent_bwd", "clip_grads", "grad_norm", "fwd", "bwd"):
        def spy(*a, real=getattr(fa, f), **k):
            given.extend(flat(a))
            allocated.clear()                     # what the test made for its arguments
            return real(*a, **k)
        monkeypatch.setattr(fa, f, spy)
    results = list(flat([CALLS[name]("cuda:0", stream=other)]))
    (_, args), = library.calls
    assert args[-1] == other.cuda_stream
    # outputs and workspace come from the stream that uses them; nothing given or returned is
    # handed on while the other stream may still use it
    assert allocated and all(s is other for _, s in allocated)
    assert given and all(any(t is r and s is other for r, s in recorded) for t in given)
    bases = {id(t) for t, _ in allocated}
    for t in results:
        assert any(t is r and s is caller for r, s in recorded) and (id(t) in bases or t._base is not None)


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_of_a_call_on_the_current_stream(name, library, streams):
    caller, _, allocated, recorded = streams
    CALLS[name]("cuda:0", stream=caller)
    CALLS[name]("cuda:0")
    assert [args[-1] for _, args in library.calls] == [caller.cuda_stream] * 2
    assert not recorded and all(s is caller for _, s in allocated)


def _sizes(*tensors):
    return {t.numel() * t.element_size() for t in tensors}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_on_another_stream_keeps_its_memory(name):
    """The other stream starts late.  Meanwhile the arguments are dropped and the
    caller's stream allocates and fills blocks of every size that the call has."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def rand(*shape, dtype=BF):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    N, D, V = 300, 136, 4001
    x, w = rand(N, D), rand(V, D)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    q, k, v, do = (rand(2, 4, 300, 64) for _ in range(4))
    values = [rand(20001, dtype=F32), rand(70001)]
    lse, z = fa.linear_xent_fwd(x, w, t)[1], fa.fwd(q, k, v, 1.0, OFFSETS, 8)[1]
    args, call, need = {
        "linear_xent_fwd": ((x, w, t), fa.linear_xent_fwd, B.lib().fibattn_linear_xent_fwd_workspace_bytes(N, D, V, 1)),
        "linear_xent_bwd": ((x, w, t, lse, rand(N, dtype=F32)), fa.linear_xent_bwd,
                            B.lib().fibattn_linear_xent_bwd_workspace_bytes(N, D, V, 1)),
        "clip_grads": ((values[0], values[1]), lambda *a, **s: fa.clip_grads(a, 1.0, out=[torch.empty_like(i) for i in a], **s),
                       B.lib().fibattn_clip_grads_workspace_bytes(2)),
        "grad_norm": ((values[0], values[1]), lambda *a, **s: fa.grad_norm(a, **s), B.lib().fibattn_clip_grads_workspace_bytes(2)),
        "fwd": ((q, k, v), lambda *a, **s: fa.fwd(*a, 1.0, OFFSETS, 8, **s), B.fwd_workspace_bytes(2, 4, 300, 8, 3, BF)),
        "bwd": ((q, k, v, z, do), lambda *a, **s: fa.bwd(*a, 1.0, OFFSETS, 8, **s), B.bwd_workspace_bytes(2, 4, 300, 8, 3, BF)),
    }[name]
    want = list(flat([call(*args)]))
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        given = [a.clone() for a in args]
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            torch.cuda._sleep(20_000_000)         # some 10 ms
        got = call(*given, stream=other)
        del given
        for n in sorted(_sizes(*args, *want) | {need}):
            junk = [torch.full((n,), 0x7f, dtype=U8, device="cuda") for _ in range(8)]
            del junk
        torch.cuda.current_stream().wait_stream(other)
        assert all(torch.equal(a, b) for a, b in zip(flat([got]), want))
        del got


def test_lse_and_dloss_at_any_offset(library, monkeypatch):
    """Views 4 and 12 bytes off a boundary go to the library as aligned copies."""
    lse, dloss = row("cuda:0"), row("cuda:0")
    at = {id(lse): 260, id(dloss): 268}
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: at.get(id(t), 4096))
    fa.linear_xent_bwd(*xent("cuda:0"), lse, dloss)
    (name, args), = library.calls
    assert name == "fibattn_linear_xent_bwd" and args[3] == 4096 and args[4] == 4096
