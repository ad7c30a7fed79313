"""Runtime calls before a launch that fail (looking up the driver's entry point, asking for the device, allowing shared memory): the call
says so, leaves no error behind for the next one, and the next one succeeds.  Against a CUDA runtime that launches nothing; no device."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_17346_b200 import binding as B
from paper_2507_17346_b200 import build
from tests.test_norm_host import GOOD, invoke

# calls that fail a given number of times, and leave their error pending
FAILING = r"""
#include <cuda_runtime_api.h>
static cudaError_t pending = cudaSuccess;
static int lookups = 0, devices = 0, attributes = 0;
extern "C" {
cudaError_t plain_last_error();
cudaError_t plain_entry_point(const char *, void **, unsigned, unsigned long long, cudaDriverEntryPointQueryResult *);
void fail_next(int l, int d, int a) { lookups = l; devices = d; attributes = a; pending = cudaSuccess; }
static cudaError_t failed(int *n) { return *n > 0 ? --*n, pending = cudaErrorUnknown : cudaSuccess; }
cudaError_t cudaGetLastError() { const cudaError_t e = pending; pending = cudaSuccess; return e != cudaSuccess ? e : plain_last_error(); }
cudaError_t cudaGetDevice(int *d) { *d = 0; return failed(&devices); }
cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return failed(&attributes); }
cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetDriverEntryPointByVersion(const char *n, void **fn, unsigned v, unsigned long long f, cudaDriverEntryPointQueryResult *r)
{
    *fn = nullptr;
    const cudaError_t e = failed(&lookups);
    return e != cudaSuccess ? e : plain_entry_point(n, fn, v, f, r);
}
}
"""


@pytest.fixture
def lib(tmp_path_factory):
    """The three files (their device code unassembled), loaded anew for each test: what they keep, they have yet to find."""
    if not hasattr(lib_path, "so"):
        lib_path.so = lib_path(tmp_path_factory.mktemp("lookup"))
    at = tmp_path_factory.mktemp("copy") / "liblookup.so"
    at.write_bytes(open(lib_path.so, "rb").read())
    lib = ctypes.CDLL(str(at))
    for name in list(GOOD) + ["deco_orth_init", "deco_orth_destroy"]:
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = B.SIGNATURES[name]
    return lib


def lib_path(at):
    here = os.path.dirname(os.path.abspath(__file__))
    nvcc = [os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1", "-Xcompiler", "-fPIC",
            "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC]
    (at / "failing.cpp").write_text(FAILING)
    renamed = ["-DcudaGetLastError=plain_last_error", "-DcudaGetDevice=plain_device", "-DcudaFuncSetAttribute=plain_attribute",
               "-DcudaGetDriverEntryPointByVersion=plain_entry_point"]
    so = str(at / "liblookup.so")
    for cmd in (nvcc + renamed + ["-c", "-o", str(at / "fake.o"), os.path.join(here, "fake_cudart.cpp")],
                nvcc + ["-shared", "-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", so] +
                [os.path.join(build.CSRC, f) for f in ("deco_norm.cu", "deco_wgrad.cu", "deco_orth.cu")] +
                [str(at / "failing.cpp"), str(at / "fake.o")]):
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stdout + res.stderr
    return so


def fails_once_and_leaves_nothing(lib, call, fail):
    lib.fail_next(*fail)
    assert call() == B.DECO_ERR_CUDA
    assert lib.cudaGetLastError() == 0
    assert call() == B.DECO_OK                                     # a failure that passes is not kept
    assert lib.cudaGetLastError() == 0


@pytest.mark.parametrize("fail", [(1, 0, 0), (0, 1, 0), (0, 0, 1)])
def test_weight_grad(lib, fail):
    fails_once_and_leaves_nothing(lib, lambda: invoke(lib, "deco_weight_grad8", workspace_bytes=1 << 26), fail)


@pytest.mark.parametrize("fail", [(0, 1, 0), (0, 0, 1)])
@pytest.mark.parametrize("name", ["deco_layernorm", "deco_layernorm_grad"])
def test_norm(lib, name, fail):
    fails_once_and_leaves_nothing(lib, lambda: invoke(lib, name), fail)


def test_orth_init(lib):
    mats = (B.deco_matrix * 1)()
    mats[0].offset, mats[0].rows, mats[0].cols = 0, 300, 200
    opt, h = B.deco_orth_options(), ctypes.c_void_p()
    opt.momentum = 0.9
    fails_once_and_leaves_nothing(lib, lambda: lib.deco_orth_init(ctypes.byref(h), 60000, mats, 1, ctypes.byref(opt)), (1, 0, 0))
    lib.deco_orth_destroy(h)
