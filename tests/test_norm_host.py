"""The norm, the 8-bit checkpoints and the weight gradients on the host: tensors of one device only, refusals before any
device call, and launches that fail.  No device."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2507_17346_b200 import binding as B
from paper_2507_17346_b200 import build

F32, BF16, P = B.DECO_F32, B.DECO_BF16, 1 << 20


class Tensor:
    """What the wrappers look at in a CUDA tensor."""

    is_cuda = True

    def __init__(self, device, shape, dtype=torch.float32):
        self.device_index, self.shape, self.dtype = device, torch.Size(shape), dtype

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def size(self, i):
        return self.shape[i]

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
        if name.endswith("_workspace"):
            return lambda *a: 64
        return lambda *a: self.calls.append((name, a)) or B.DECO_OK


@pytest.fixture
def fake(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream_on", lambda stream, device: ("stream of", device))
    return lib


def call(name, device=0, **other):
    """The wrapper with all its tensors on `device`, the named ones elsewhere."""
    d = lambda n: other.get(n, device)  # noqa: E731
    f = lambda n, *s: Tensor(d(n), s)  # noqa: E731
    packed = (Tensor(d("codes"), (3, 64), torch.int8), Tensor(d("exponents"), (3, 2), torch.uint8))
    room = Tensor(d("workspace"), (64,), torch.uint8)
    if name == "deco_layernorm":
        B.deco_layernorm(f("x", 3, 40), f("weight", 40), f("bias", 40), f("y", 3, 40), mean=f("mean", 3), rstd=f("rstd", 3),
                         add=f("add", 3, 40), total=f("total", 3, 40), packed=packed)
    elif name == "deco_layernorm_grad":
        B.deco_layernorm_grad(packed if "codes" in other or "exponents" in other else f("x", 3, 40), f("mean", 3), f("rstd", 3),
                              f("weight", 40), f("dy", 3, 40), f("dx", 3, 40), dweight=f("dweight", 40), dbias=f("dbias", 40),
                              add=f("add", 3, 40), workspace=room)
    elif name == "deco_pack8":
        B.deco_pack8(f("x", 3, 40), packed)
    elif name == "deco_unpack8":
        B.deco_unpack8(packed, f("y", 3, 40))
    else:
        B.deco_weight_grad8(f("dy", 3, 5), packed, f("dw", 5, 40), db=f("db", 5), workspace=room)


NAMES = {"deco_layernorm": ["x", "weight", "bias", "y", "mean", "rstd", "add", "total", "codes", "exponents"],
         "deco_layernorm_grad": ["x", "mean", "rstd", "weight", "dy", "dx", "dweight", "dbias", "add", "workspace", "codes", "exponents"],
         "deco_pack8": ["x", "codes", "exponents"], "deco_unpack8": ["y", "codes", "exponents"],
         "deco_weight_grad8": ["dy", "dw", "db", "workspace", "codes", "exponents"]}


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_one_device(fake, name):
    for tensor in NAMES[name]:
        with pytest.raises(ValueError, match="is on cuda:"):
            call(name, **{tensor: 1})
    with pytest.raises(ValueError, match="is on cuda:"):
        call(name, device=1)                                       # all together elsewhere
    assert fake.calls == []
    call(name)
    assert [c[0] for c in fake.calls] == [name] and fake.calls[0][1][-1] == ("stream of", 0)


# ------------------------------------------------------------------- the library, without a device

GOOD = {
    "deco_layernorm": dict(x=P, dtype=F32, rows=2, cols=64, x_stride=64, add=P, add_stride=64, sum=2 * P, sum_stride=64, weight=P, bias=P,
                           eps=1e-5, y=3 * P, y_stride=64, mean=P, rstd=P, codes=P, exponents=P, stream=None),
    "deco_layernorm_grad": dict(x=P, dtype=F32, rows=2, cols=64, x_stride=64, codes=None, exponents=None, mean=P, rstd=P, weight=P, dy=P,
                                dy_stride=64, add=P, add_stride=64, dx=P, dx_stride=64, dweight=P, dbias=P, grad_dtype=F32, accumulate=0,
                                workspace=P, workspace_bytes=1 << 20, stream=None),
    "deco_pack8": dict(x=P, dtype=F32, rows=2, cols=64, x_stride=64, codes=P, exponents=P, stream=None),
    "deco_unpack8": dict(codes=P, exponents=P, rows=2, cols=64, y=P, dtype=F32, y_stride=64, stream=None),
    "deco_weight_grad8": dict(dy=P, dtype=F32, rows=2, out=64, dy_stride=64, codes=P, exponents=P, cols=64, dw=P, db=P, grad_dtype=F32,
                              transposed=0, accumulate=0, workspace=P, workspace_bytes=1 << 24, stream=None),
}
BAD = {
    "deco_layernorm": [dict(x=None), dict(y=None), dict(x=P + 2), dict(add=P + 1), dict(sum=2 * P + 2), dict(y=3 * P + 3), dict(weight=P + 1),
                       dict(bias=P + 2), dict(mean=P + 1), dict(rstd=P + 3), dict(codes=P + 8), dict(codes=None), dict(exponents=None),
                       dict(dtype=2), dict(cols=0), dict(cols=1 << 25), dict(x_stride=63), dict(add_stride=63), dict(y_stride=1),
                       dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(add=None), dict(y=2 * P),
                       dict(y=P, y_stride=65), dict(sum=P, sum_stride=65), dict(rows=1 << 28), dict(x_stride=1 << 41)],
    "deco_layernorm_grad": [dict(x=None), dict(codes=P, exponents=P), dict(x=None, codes=P), dict(x=None, codes=P + 4, exponents=P),
                            dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(x=P + 1), dict(dy=P + 2), dict(dx=P + 2),
                            dict(add=P + 2), dict(mean=P + 1), dict(weight=P + 2), dict(dweight=P + 2), dict(dbias=P + 1),
                            dict(grad_dtype=BF16, dbias=P + 1), dict(dtype=-1), dict(grad_dtype=3), dict(cols=0), dict(dy_stride=63),
                            dict(dx=P, dx_stride=65), dict(workspace=None), dict(workspace=P + 8), dict(rows=1 << 28)],
    "deco_pack8": [dict(x=None), dict(codes=None), dict(exponents=None), dict(x=P + 2), dict(codes=P + 1), dict(cols=0), dict(x_stride=63),
                   dict(dtype=5)],
    "deco_unpack8": [dict(y=None), dict(codes=None), dict(exponents=None), dict(y=P + 2), dict(codes=P + 1), dict(cols=0), dict(y_stride=63),
                     dict(dtype=5)],
    "deco_weight_grad8": [dict(dy=None), dict(codes=None), dict(exponents=None), dict(dw=None), dict(dy=P + 2), dict(codes=P + 8),
                          dict(dw=P + 2), dict(db=P + 1), dict(out=0), dict(cols=0), dict(dy_stride=63), dict(dtype=9), dict(grad_dtype=9),
                          dict(workspace=None), dict(workspace=P + 4), dict(rows=1 << 28), dict(cols=1 << 25)],
}


def invoke(lib, name, **change):
    return getattr(lib, name)(*dict(GOOD[name], **change).values())


@pytest.mark.parametrize("name", GOOD)
def test_refusals_come_before_any_device_call(name):
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no kernel could be launched")
    build.build()
    lib = B.load()
    for change in BAD[name]:
        assert invoke(lib, name, **change) == B.DECO_ERR_INVALID_ARG, change
    if "workspace" in GOOD[name]:
        assert invoke(lib, name, workspace_bytes=16) == B.DECO_ERR_CAPACITY
    if name != "deco_weight_grad8" and name != "deco_layernorm_grad":
        assert invoke(lib, name, rows=0) == B.DECO_OK                # nothing to do
    assert invoke(lib, name) == B.DECO_ERR_CUDA                      # nothing wrong but the missing device


def test_workspace_sizes():
    build.build()
    lib = B.load()
    assert lib.deco_layernorm_grad_workspace(0, 64) == 0 and lib.deco_layernorm_grad_workspace(5, 0) == 0
    sizes = [lib.deco_layernorm_grad_workspace(r, c) for r, c in ((1, 64), (100, 64), (100000, 64), (100000, 8192), (100, 100000))]
    assert all(s > 0 for s in sizes) and sizes[:4] == sorted(sizes[:4])
    assert lib.deco_layernorm_grad_workspace(1 << 27, 8192) < 1 << 26     # it does not grow with the rows
    a = lib.deco_weight_grad8_workspace(P, BF16, 1000, 64, 64, 64, F32)
    assert a < lib.deco_weight_grad8_workspace(P + 2, BF16, 1000, 64, 64, 64, F32) < lib.deco_weight_grad8_workspace(P, F32, 1000, 64, 64, 64, F32)


@pytest.fixture(scope="module")
def logged(tmp_path_factory):
    """The two files (their device code unassembled) with a runtime that launches nothing."""
    at = tmp_path_factory.mktemp("fake")
    here = os.path.dirname(os.path.abspath(__file__))
    more = at / "more.cpp"
    more.write_text('#include <cuda_runtime_api.h>\nextern "C" cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t)'
                    ' { return cudaSuccess; }\n')
    so = str(at / "libnorm_fake.so")
    cmd = [os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1", "-shared", "-cudart",
           "none", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-o", so,
           os.path.join(build.CSRC, "deco_norm.cu"), os.path.join(build.CSRC, "deco_wgrad.cu"), os.path.join(here, "fake_cudart.cpp"),
           str(more)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    lib = ctypes.CDLL(so)
    for name in GOOD:
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = B.SIGNATURES[name]
    lib.fake_reset.argtypes = [ctypes.c_int64]
    lib.fake_reset.restype = None
    lib.cudaGetLastError.restype = ctypes.c_int
    return lib


@pytest.mark.parametrize("name,change,launches", [
    ("deco_layernorm", {}, 1), ("deco_layernorm", dict(x=5 * P + 4), 1), ("deco_layernorm", dict(cols=20000, **{k + "_stride": 20000 for k in ("x", "add", "sum", "y")}), 1),
    ("deco_layernorm_grad", {}, 2), ("deco_layernorm_grad", dict(x=5 * P + 4), 2), ("deco_layernorm_grad", dict(dweight=None, dbias=None), 1),
    ("deco_layernorm_grad", dict(cols=20000, **{k + "_stride": 20000 for k in ("x", "add", "dy", "dx")}), 3), ("deco_layernorm_grad", dict(rows=0), 1),
    ("deco_pack8", {}, 1), ("deco_unpack8", {}, 1), ("deco_weight_grad8", {}, 2), ("deco_weight_grad8", dict(rows=0), 0)])
def test_a_failed_launch_is_reported_and_leaves_no_error_behind(logged, name, change, launches):
    change = dict(change)
    if "workspace" in GOOD[name]:
        change.setdefault("workspace_bytes", 1 << 26)
    logged.fake_reset(0)
    assert invoke(logged, name, **change) == B.DECO_OK
    for n in range(1, launches + 1):
        logged.fake_reset(n)
        assert invoke(logged, name, **change) == B.DECO_ERR_CUDA, n
        assert logged.cudaGetLastError() == 0
        logged.fake_reset(0)
        assert invoke(logged, name, **change) == B.DECO_OK
    logged.fake_reset(launches + 1)
    assert invoke(logged, name, **change) == B.DECO_OK               # there was no further launch to fail
