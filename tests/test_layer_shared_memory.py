"""The shared memory that the layer's kernels ask for, on a CPU with a fake runtime.

A kernel's limit belongs to the kernel, not to the call: two host threads whose calls set different limits for one kernel can do so
between each other's setting and launch, and the launch of the larger one fails.  So the limits have to be the same whatever
a call's sizes are."""
import ctypes
import itertools
import os
import subprocess

import pytest

import fake_cuda as F
from paper_2608_03676_b200 import NormParams, RouteParams
from paper_2608_03676_b200.build import OBJ, SOURCES, build

AT = [F.DEVICE + (i << 36) for i in range(16)]
WITHOUT_A_LIMIT = 46 * 1024                      # 48 KB, less what a kernel declares


class Event(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_long), ("limit", ctypes.c_long), ("launched", ctypes.c_long)]


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    build()
    folder = str(tmp_path_factory.mktemp("limits"))
    here = os.path.dirname(os.path.abspath(__file__))
    obj, lib = os.path.join(folder, "fake_limits.o"), os.path.join(folder, "libtaot_limits.so")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["gcc", "-O1", "-fPIC", "-I", os.path.join(cuda, "include"), "-c", os.path.join(here, "fake_limits.c"), "-o", obj], check=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", lib, obj] + [os.path.join(OBJ, src.replace(".cu", ".o")) for src in SOURCES], check=True)
    so = ctypes.CDLL(lib)
    so.limits_event.restype = ctypes.POINTER(Event)
    return so


def ptr(a):
    return None if a is None else ctypes.c_void_p(a)


def route(so, dtype, N, E, k, groups, bias):
    p = RouteParams(ctypes.sizeof(RouteParams), dtype, 1, N, E, k, 1, groups, max(1, groups // 2), 1, 1, 1.0, E, E)
    so.fake_reset()
    assert so.taot_route(ctypes.byref(p), ptr(AT[1]), ptr(AT[2] if bias else None), None, ptr(AT[3]), ptr(AT[4]), ptr(F.CALLER)) == 0


def norm_grad(so, dtype, N, D, ld, dweight):
    p = NormParams(ctypes.sizeof(NormParams), dtype, N, D, 0, 0.0, 0, ld, ld, ld, ld, ld)
    so.fake_reset()
    assert so.taot_rms_norm_backward(ctypes.byref(p), ptr(AT[1]), None, ptr(AT[2]), ptr(AT[3]), ptr(AT[4]), ptr(AT[5]), ptr(AT[6] if dweight else None),
                                     ptr(AT[7]), ptr(F.CALLER)) == 0


def check(so, since):
    """Limits set and bytes launched since, by kernel: one limit at most, and enough."""
    limits, most = {}, {}
    for i in range(since, so.limits_count()):
        e = so.limits_event(i).contents
        if e.limit >= 0:
            limits.setdefault(e.kernel, set()).add(e.limit)
        else:
            most[e.kernel] = max(most.get(e.kernel, 0), e.launched)
    assert most
    for kernel, bytes_ in most.items():
        set_ = limits.get(kernel, set())
        assert len(set_) <= 1, set_
        assert bytes_ <= max([WITHOUT_A_LIMIT] + list(set_))


def test_the_routers_limits_do_not_depend_on_a_calls_sizes(so):
    since = so.limits_count()
    for dtype, N, E, groups, bias in itertools.product(range(3), (4, 1 << 20), (8, 16, 32, 64, 96, 128, 200, 256, 512, 768, 1024), (1, 2, 8), (False, True)):
        for k in (1, 4, 8, 16):
            if k <= max(1, groups // 2) * (E // groups):
                route(so, dtype, N, E, k, groups, bias)
    check(so, since)


def test_the_norms_gradients_limits_do_not_depend_on_a_calls_sizes(so):
    since = so.limits_count()
    for dtype, D, odd, dweight in itertools.product(range(3), (1, 64, 256, 512, 1000, 1024, 2048, 4096, 8192, 12288, 20000), (0, 1), (True, False)):
        for N in (1, 5, 100000):
            norm_grad(so, dtype, N, D, D + odd, dweight)
    check(so, since)
