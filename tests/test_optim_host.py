"""The host side of the optimizer calls, without a GPU: csrc/co3_optim.cu linked with a runtime of host memory (fake_cudart.c), in
which copies and fills are late as the real one may have them."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2203_09044_b200 import binding as b, build

TESTS = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    d = tmp_path_factory.mktemp("fake_cudart")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-fmad=false", "-Xcompiler", "-fPIC", "-I", build.INCLUDE,
                    "-I", build.CSRC, "-c", os.path.join(build.CSRC, "co3_optim.cu"), "-o", str(d / "optim.o")], check=True)
    subprocess.run(["gcc", "-O1", "-fPIC", "-c", os.path.join(TESTS, "fake_cudart.c"), "-o", str(d / "fake.o")], check=True)
    # symbolic: this process may hold the real runtime already
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", str(d / "optim.o"), str(d / "fake.o"), "-o", str(d / "fake.so")], check=True)
    L = C.CDLL(str(d / "fake.so"))
    L.co3_adamw_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(b.AdamwConfig)]
    L.co3_adamw_destroy.argtypes = [C.c_void_p]
    L.co3_adamw_status.argtypes = [C.c_void_p, C.POINTER(C.c_uint32), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.c_int32]
    L.co3_adamw_steps_export.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
    L.co3_adamw_steps_import.argtypes = [C.c_void_p, C.c_int64]
    L.fake_written.restype = C.c_long
    return L


class Handle:
    """A handle of the library with the fake runtime."""

    def __init__(self, L, sizes=(1000, 5), betas=(0.9, 0.999), eps=1e-8):
        n = np.array(sizes, np.int64)
        cfg = b.AdamwConfig(len(n), n.ctypes.data_as(C.POINTER(C.c_int64)), None, b.F32, b.F32, b.NONE, 32, betas[0], betas[1], eps, 0.0, 0, 0)
        self.L, self.h = L, C.c_void_p()
        assert L.co3_adamw_create(C.byref(self.h), C.byref(cfg)) == b.OK

    def __enter__(self):
        return self

    def __exit__(self, *_):
        self.L.fake_set_device(0)
        self.L.co3_adamw_destroy(self.h)

    def status(self, clear):
        f, e, s = C.c_uint32(), C.c_uint64(), C.c_uint64()
        return self.L.co3_adamw_status(self.h, C.byref(f), C.byref(e), C.byref(s), clear), (f.value, e.value, s.value)

    def steps(self):
        n = C.c_int64(-1)
        return self.L.co3_adamw_steps_export(self.h, C.byref(n)), n.value

    def set_steps(self, n):
        return self.L.co3_adamw_steps_import(self.h, n)


@pytest.mark.parametrize("sizes", [(1000, 5), (0,)])
def test_nothing_is_left_to_be_copied_when_a_call_returns(fake, sizes):
    """A step on a stream that does not wait for the null stream may follow at once."""
    with Handle(fake, sizes) as h:
        assert fake.fake_waiting() == 0
        assert h.set_steps(7) == b.OK and fake.fake_waiting() == 0
        assert h.status(clear=1) == (b.OK, (0, 0, 0)) and fake.fake_waiting() == 0
        assert h.steps() == (b.OK, 7)


def test_with_another_device_current_every_call_is_refused(fake):
    """As the norm and the step refuse it; a wait would be for the wrong device."""
    with Handle(fake) as h:
        assert h.set_steps(3) == b.OK
        fake.fake_set_device(1)
        before = fake.fake_calls()
        assert h.steps() == (b.EINVAL, -1) and h.set_steps(9) == b.EINVAL
        assert h.status(clear=0)[0] == b.EINVAL and h.status(clear=1)[0] == b.EINVAL
        assert fake.fake_calls() == before
        fake.fake_set_device(0)
        assert h.steps() == (b.OK, 3)


def test_clearing_the_status_writes_nothing_else(fake):
    """Not the step count, which another thread's step may have moved on since it was read."""
    with Handle(fake) as h:
        assert h.set_steps(3) == b.OK
        fake.fake_advance()
        assert h.status(clear=1) == (b.OK, (0, 0, 0))
        assert h.steps() == (b.OK, 4)


def test_setting_the_steps_leaves_the_status(fake):
    """... and the tickets, which a step that another thread has begun may hold."""
    with Handle(fake) as h:
        fake.fake_written()
        assert h.set_steps(3) == b.OK
        assert fake.fake_written() <= 40                # count, two powers, two corrections, key
