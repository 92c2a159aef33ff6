"""The router's exponential in 64 bits, its source compiled for the CPU, against exponentials of more digits."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2608_03676_b200.build import CSRC

AROUND = """
#include <cmath>
#include <cstdint>
#include <cstring>
using std::fma; using std::fmax; using std::fmin;
static int __double2loint(double v) { uint64_t u; memcpy(&u, &v, 8); return (int)(uint32_t)u; }
static double __hiloint2double(int hi, int lo) { uint64_t u = (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo; double v; memcpy(&v, &u, 8); return v; }
%s
extern "C" void exps(const double* x, double* y, long n) { for (long i = 0; i < n; ++i) y[i] = exp_of(x[i]); }
"""


@pytest.fixture(scope="module")
def exp_of(tmp_path_factory):
    text = open(os.path.join(CSRC, "route_common.cuh")).read()
    body = re.search(r"^__device__ __forceinline__ (double exp_of\(double x\)\n\{.*?^\})", text, re.S | re.M).group(1)
    folder = tmp_path_factory.mktemp("exp")
    src, lib = str(folder / "exp.cpp"), str(folder / "exp.so")
    with open(src, "w") as f:
        f.write(AROUND % body)
    subprocess.run(["g++", "-O1", "-ffp-contract=off", "-shared", "-fPIC", src, "-o", lib], check=True)
    so = ctypes.CDLL(lib)

    def call(x):
        x = np.ascontiguousarray(x, dtype=np.float64)
        y = np.empty_like(x)
        so.exps(x.ctypes.data_as(ctypes.c_void_p), y.ctypes.data_as(ctypes.c_void_p), ctypes.c_long(len(x)))
        return y
    return call


def ulps(y, x):
    """How many ulps of the result it is off, by exponentials with 64 bits of mantissa."""
    if np.finfo(np.longdouble).nmant < 63:
        pytest.skip("no type of more digits here")
    want = np.exp(x.astype(np.longdouble))
    return np.abs((y.astype(np.longdouble) - want) / np.spacing(np.maximum(np.abs(y), 2.0 ** -1022)).astype(np.longdouble)).astype(np.float64)


def test_an_ulp(exp_of):
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-700, 700, 400000), rng.uniform(-40, 0, 400000), rng.normal(0, 1, 400000), rng.normal(0, 1e-6, 100000),
                        np.arange(-700, 700), np.arange(-1000, 1000) * np.log(2) / 2, np.nextafter(np.arange(-900, 900) * np.log(2) / 2, 0)])
    x = x[(x > -708) & (x < 709)]
    off = ulps(exp_of(x), x)
    assert off.max() <= 1.0, (off.max(), x[off.argmax()])


def test_results_below_the_normal_numbers_are_rounded_once(exp_of):
    x = np.random.default_rng(2).uniform(-745.2, -708.4, 200000)
    assert ulps(exp_of(x), x).max() <= 1.0


def test_the_ends(exp_of):
    y = exp_of(np.array([0.0, -0.0, -746.0, -1e300, -np.inf, 710.0, 1e300, np.inf]))
    assert y.tolist() == [1.0, 1.0, 0.0, 0.0, 0.0, np.inf, np.inf, np.inf]


def test_it_rises(exp_of):
    """Logits in order have scores in order: fp32 neighbours never change places."""
    x = np.sort(np.random.default_rng(3).uniform(-87, 0, 200000).astype(np.float32)).astype(np.float64)
    assert (np.diff(exp_of(x)) >= 0).all()
