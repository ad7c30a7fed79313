"""deco_orth_run and deco_token_logprobs when a launch fails, against a CUDA runtime that only keeps a log (fake_cudart.cpp; no device, no
kernel runs): whatever fails, the caller's stream waits for what was enqueued on the handle's own stream."""
import ctypes
import os
import subprocess

import pytest

from paper_2507_17346_b200 import binding as B
from paper_2507_17346_b200 import build

LAUNCH, LAUNCH_FAILED, RECORD, WAIT = 1, 2, 3, 4
CALLER = 0x77


class Entry(ctypes.Structure):
    _fields_ = [("op", ctypes.c_uint32), ("unused", ctypes.c_uint32), ("stream", ctypes.c_uint64),
                ("event", ctypes.c_uint64)]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    """The two files (their device code unassembled) with the runtime of this test."""
    so = str(tmp_path_factory.mktemp("fake") / "liborth_fake.so")
    cmd = [os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1",
           "-shared", "-cudart", "none", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic", "-I",
           os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-o", so, os.path.join(build.CSRC, "deco_orth.cu"),
           os.path.join(build.CSRC, "deco_logprobs.cu"),
           os.path.join(os.path.dirname(os.path.abspath(__file__)), "fake_cudart.cpp")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    lib = ctypes.CDLL(so)
    for name in ("deco_orth_init", "deco_orth_run", "deco_orth_destroy", "deco_token_logprobs"):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = B.SIGNATURES[name]
    lib.fake_reset.argtypes = [ctypes.c_int64]
    lib.fake_reset.restype = None
    lib.fake_log.argtypes = [ctypes.POINTER(Entry), ctypes.c_uint64]
    lib.fake_log.restype = ctypes.c_uint64
    return lib


def run(lib, h, fail_at):
    lib.fake_reset(fail_at)
    status = lib.deco_orth_run(h, 0x10000, B.DECO_F32, 0x20000, 0x30000, CALLER)
    room = (Entry * 4096)()
    return status, list(room[:lib.fake_log(room, 4096)])


def joined(log):
    """Every launch on another stream than the caller's lies before a record there for which the caller's waits."""
    for i, e in enumerate(log):
        if e.op == LAUNCH and e.stream != CALLER:
            records = [(j, r.event) for j, r in enumerate(log) if j > i and r.op == RECORD and r.stream == e.stream]
            if not any(w.op == WAIT and w.stream == CALLER and w.event == ev and k > j
                       for j, ev in records for k, w in enumerate(log)):
                return False
    return True


@pytest.mark.parametrize("shapes,workspace", [([(64, 147), (300, 200)], 0),
                                              ([(64, 900), (100, 128), (1, 5000), (300, 200), (520, 400)], 1)])
def test_a_failed_launch_leaves_nothing_unordered(lib, shapes, workspace):
    mats = (B.deco_matrix * len(shapes))()
    at = 0
    for m, (r, c) in zip(mats, shapes):
        m.offset, m.rows, m.cols = at, r, c
        at += r * c + 3
    opt = B.deco_orth_options()
    opt.momentum, opt.workspace_bytes = 0.9, workspace
    h = ctypes.c_void_p()
    assert lib.deco_orth_init(ctypes.byref(h), at, mats, len(shapes), ctypes.byref(opt)) == B.DECO_OK
    try:
        status, log = run(lib, h, 0)
        count = sum(e.op == LAUNCH for e in log)
        assert status == B.DECO_OK and joined(log) and any(e.op == LAUNCH and e.stream != CALLER for e in log)
        for n in range(1, count + 1):
            status, log = run(lib, h, n)
            assert status == B.DECO_ERR_CUDA and sum(e.op == LAUNCH_FAILED for e in log) == 1
            assert joined(log), "launch %d of %d" % (n, count)
            status, log = run(lib, h, 0)                           # its error is not the next pass's
            assert status == B.DECO_OK and sum(e.op == LAUNCH for e in log) == count
    finally:
        lib.deco_orth_destroy(h)


@pytest.mark.parametrize("rows,vocab", [(1, 32000), (2000, 1000)])   # on eight CTAs, and on one
def test_a_failed_call_of_token_logprobs_leaves_no_error_behind(lib, rows, vocab):
    def call(fail_at):
        lib.fake_reset(fail_at)
        return lib.deco_token_logprobs(0x10000, B.DECO_F32, rows, vocab, vocab, 0x20000, 1.0, 0x30000, None, None, 0,
                                       None, None, CALLER)
    assert call(0) == B.DECO_OK
    assert call(1) == B.DECO_ERR_CUDA
    lib.cudaGetLastError.restype = ctypes.c_int
    assert lib.cudaGetLastError() == 0 and call(0) == B.DECO_OK
