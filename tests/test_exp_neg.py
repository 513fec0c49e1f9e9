"""The 64-bit exponential of the sampling kernel (csrc/sample.cu), its source compiled for
the host, against 40-digit decimals.

Bound on its relative error: the table's rounding and the last fma's, 2^-53 each; the
series' next term, (ln 2 / 128)^6 / 720 < 2^-54.6; r's rounding and those of the series,
each 2^-53 of a number below 2^-7, three of them.  Together below 2.4 * 2^-53."""
import ctypes as C
import os
import re
import subprocess
from decimal import Decimal, getcontext

import numpy as np
import pytest

from helpers import ROOT

getcontext().prec = 40

HARNESS = """
#include <cmath>
#include <cstdint>
#include <cstring>
#define __device__
#define __forceinline__ inline
static uint64_t bits(double x) { uint64_t b; std::memcpy(&b, &x, 8); return b; }
static int __double2loint(double x) { return static_cast<int>(static_cast<uint32_t>(bits(x))); }
static int __double2hiint(double x) { return static_cast<int>(static_cast<uint32_t>(bits(x) >> 32)); }
static double __hiloint2double(int hi, int lo) {
  const uint64_t b = static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo);
  double x;
  std::memcpy(&x, &b, 8);
  return x;
}
using std::fma;
%s
extern "C" void run(const double* x, int n, double* y) { for (int i = 0; i < n; ++i) y[i] = exp_neg(x[i]); }
"""


def _source():
    return open(os.path.join(ROOT, "paper_2608_10139_gb300", "csrc", "sample.cu")).read()


@pytest.fixture(scope="module")
def exp_neg(tmp_path_factory):
    src = _source()
    table = re.search(r"__device__ const double kExp2\[64\] = \{.*?\};", src, flags=re.S).group(0)
    body = re.search(r"__device__ __forceinline__ double exp_neg\(double x\) \{.*?\n\}", src, flags=re.S).group(0)
    d = tmp_path_factory.mktemp("exp")
    (d / "e.cpp").write_text(HARNESS % (table + "\n" + body))
    # products and sums are rounded apart, as written: only the fmas are fused
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-o", str(d / "e.so"),
                    str(d / "e.cpp")], check=True)
    f = C.CDLL(str(d / "e.so")).run
    f.argtypes = [C.c_void_p, C.c_int, C.c_void_p]

    def run(x):
        x = np.ascontiguousarray(x, np.float64)
        y = np.empty_like(x)
        f(x.ctypes.data, len(x), y.ctypes.data)
        return y
    return run


def _errors(x, y):
    """Relative errors in units of 2^-53."""
    out = []
    for a, b in zip(x, y):
        e = Decimal(float(a)).exp()
        out.append(abs(float((Decimal(float(b)) - e) / e)) * 2.0 ** 53)
    return np.array(out)


def test_the_table_is_rounded_right():
    rows = re.search(r"kExp2\[64\] = \{(.*?)\};", _source(), flags=re.S).group(1)
    values = [float.fromhex(v) for v in re.findall(r"0x1\.[0-9a-f]+p\+0", rows)]
    assert len(values) == 64
    for j, v in enumerate(values):
        assert v == float(Decimal(2) ** (Decimal(j) / 64)), j


def test_the_two_parts_of_ln2():
    parts = [float.fromhex(v) for v in re.findall(r"fma\(w, -(0x1\.[0-9a-f]+p-\d+)", _source())]
    assert len(parts) == 2
    lo, hi = sorted(parts)
    assert abs(Decimal(hi) + Decimal(lo) - Decimal(2).ln() / 64) < Decimal(2) ** -90
    assert float(hi * 2.0 ** 39).is_integer()  # 33 bits: w * hi is exact for whole numbers below 2^20


def test_errors_stay_within_the_bound(exp_neg):
    rng = np.random.default_rng(0)
    step = float(Decimal(2).ln() / 64)
    whole = rng.integers(0, 64000, 1500)
    x = np.concatenate([
        -rng.random(1500) * 700, -np.exp(rng.uniform(-60, 6.5, 1500)),
        -(whole + 0.5) * step, -np.nextafter((whole + 0.5) * step, 0), -np.nextafter((whole + 0.5) * step, 1e9),  # r largest
        -whole * step, -np.arange(0, 700, 1.0), -(2.0 ** -np.arange(0.0, 80.0)),
        -rng.random(500).astype(np.float32).astype(np.float64) * 20])
    x = x[x >= -700]
    e = _errors(x, exp_neg(x))
    assert e.max() <= 2.4, (e.max(), x[e.argmax()])


def test_ends(exp_neg):
    x = np.array([0.0, -0.0, -5e-324, -1e-300, -700.0, np.nextafter(-700.0, -1e9), -1e308, -np.inf])
    y = exp_neg(x)
    assert (y[:4] == 1).all() and (y[5:] == 0).all()
    assert abs(float((Decimal(float(y[4])) - Decimal(-700).exp()) / Decimal(-700).exp())) <= 2.4 * 2.0 ** -53
