"""The wrappers of the token log probabilities and the orthogonalised updates take tensors of one device only: the
current one, or the handle's.  Stand-ins for tensors and for the library; no device."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B

HANDLE, D = 0x5000, 12


class Tensor:
    """What the wrappers look at in a CUDA tensor."""

    is_cuda = True

    def __init__(self, device, shape, dtype=torch.float32):
        self.device_index, self.shape, self.dtype = device, torch.Size(shape), dtype

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000 * (self.device_index + 1)


class Library:
    """Accepts every call and keeps its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or B.DECO_OK


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(B, "load", lambda: fake)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(B, "_stream", lambda stream: ("stream of", 0))
    monkeypatch.setattr(B, "_stream_on", lambda stream, device: ("stream of", device), raising=False)
    monkeypatch.setitem(getattr(B, "_orth_handles", {}), HANDLE, (D, 1))
    return fake


def rejected(lib, fn, *args, **kw):
    with pytest.raises(ValueError, match="is on cuda:"):
        fn(*args, **kw)
    assert lib.calls == []


def logprob_args(device, **other):
    dev = lambda name: other.get(name, device)  # noqa: E731
    f = lambda name, *s: Tensor(dev(name), s)  # noqa: E731
    return {"logits": f("logits", 3, 7), "targets": Tensor(dev("targets"), (3,), torch.int64), "lse": f("lse", 3),
            "entropy": f("entropy", 3), "top_idx": Tensor(dev("top_idx"), (3, 2), torch.int32), "logprob": f("logprob", 3),
            "top_logprob": f("top_logprob", 3, 2), "grad": f("grad", 3, 7), "g_logprob": f("g_logprob", 3),
            "g_entropy": f("g_entropy", 3), "g_top": f("g_top", 3, 2)}


FORWARD = ["logits", "targets", "logprob", "entropy", "lse", "top_idx", "top_logprob"]
BACKWARD = ["logits", "targets", "lse", "grad", "g_logprob", "entropy", "g_entropy", "top_idx", "g_top"]


@pytest.mark.parametrize("fn,names", [("deco_token_logprobs", FORWARD), ("deco_token_logprobs_grad", BACKWARD)])
def test_token_logprobs_stay_on_the_current_device(lib, fn, names):
    pick = lambda a: {k: a[k] for k in names}  # noqa: E731
    for name in names:
        rejected(lib, getattr(B, fn), **pick(logprob_args(0, **{name: 1})))
    rejected(lib, getattr(B, fn), **pick(logprob_args(1)))             # all together elsewhere
    getattr(B, fn)(**pick(logprob_args(0)))
    assert [c[0] for c in lib.calls] == [fn] and lib.calls[0][1][-1] == ("stream of", 0)


def test_orth_stays_on_the_handles_device(lib):
    """The handle's device is 1 here, the current one 0."""
    def args(x=1, out=1, momentum=1):
        return Tensor(x, (D,)), Tensor(out, (D,), torch.bfloat16), Tensor(momentum, (D,))
    for wrong in ({"x": 0}, {"out": 0}, {"momentum": 0}, {"x": 0, "out": 0, "momentum": 0}):
        rejected(lib, B.deco_orth_run, HANDLE, *args(**wrong))
    rejected(lib, B.deco_apply_update_orth, 0x6000, HANDLE, Tensor(0, (D,)))
    B.deco_orth_run(HANDLE, *args())
    B.deco_apply_update_orth(0x6000, HANDLE, Tensor(1, (D,)))
    assert [c[1][-1] for c in lib.calls] == [("stream of", 1)] * 2
    B.deco_orth_get_stats(HANDLE)
    assert lib.calls[-1][0] == "deco_orth_get_stats" and lib.calls[-1][1][1] == ("stream of", 1)
