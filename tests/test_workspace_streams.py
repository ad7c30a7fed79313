"""The workspace that a wrapper makes belongs to the stream that it launches on.  Stand-ins for tensors, streams, allocations and the
library; no device."""
import contextlib

import pytest
import torch

from paper_2507_17346_b200 import binding as B
from tests.test_norm_host import Tensor

POOL, SIDE, CURRENT = 0x9000, 0x7700, 0x5500


class Stream:
    """What torch makes of an address: for 0 one of its own pool's streams, which is not the default one."""

    def __init__(self, address=0, device=None):
        self.cuda_stream, self.device = address or POOL, device


class Default(Stream):
    def __init__(self, device=None):
        self.cuda_stream, self.device = 0, device


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 64
        return lambda *a: self.calls.append((name, a)) or B.DECO_OK


@pytest.fixture
def made(monkeypatch):
    """-> (the library's calls, the streams on which workspaces were made)."""
    lib, on, current = Library(), [], [CURRENT]

    @contextlib.contextmanager
    def use(stream):
        before, current[0] = current[0], stream.cuda_stream
        yield
        current[0] = before

    def empty(nbytes, dtype, device):
        assert (nbytes, dtype, device) == (64, torch.uint8, 0)
        on.append(current[0])
        return Tensor(device, (nbytes,), dtype)

    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B, "_queries", (lambda: 0, lambda device: CURRENT))
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", Default)
    return lib.calls, on


def call(name, stream, **more):
    f = lambda *s: Tensor(0, s)  # noqa: E731
    if name == "deco_layernorm_grad":
        B.deco_layernorm_grad(f(3, 40), f(3), f(3), f(40), f(3, 40), f(3, 40), dweight=f(40), stream=stream, **more)
    else:
        packed = (Tensor(0, (3, 64), torch.int8), Tensor(0, (3, 2), torch.uint8))
        B.deco_weight_grad8(f(3, 5), packed, f(5, 40), stream=stream, **more)


@pytest.mark.parametrize("name", ["deco_layernorm_grad", "deco_weight_grad8"])
@pytest.mark.parametrize("stream,address", [(None, CURRENT), (0, 0), (Default(0), 0), (SIDE, SIDE), (Stream(SIDE), SIDE), (1, 0)])
def test_a_workspace_belongs_to_the_stream_of_its_call(made, name, stream, address):
    """Also for the default stream, by its address, as torch's object, or by the runtime's name for it (1)."""
    calls, on = made
    call(name, stream)
    assert [c[0] for c in calls] == [name] and on == [address]
    assert calls[0][1][-1] == (address if stream != 1 else 1)


@pytest.mark.parametrize("name", ["deco_layernorm_grad", "deco_weight_grad8"])
def test_the_per_thread_stream_needs_the_callers_workspace(made, name):
    """One address (2), another stream in each thread: nothing can be kept for it."""
    calls, on = made
    with pytest.raises(ValueError, match="workspace"):
        call(name, 2)
    assert not calls and not on
    call(name, 2, workspace=Tensor(0, (64,), torch.uint8))
    assert calls[0][1][-1] == 2 and not on
