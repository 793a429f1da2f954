"""What a logit weighs in cr_sample (csrc/sample_weights.h), compiled for the host
from the code that the kernel runs, against exp((x - x_0) / T) in 64 bits."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_35139_amd", "csrc")
SHIM = """
#include <hip/hip_runtime.h>
#include "sample_weights.h"
using namespace cr;
// the weights of n logits in a row whose largest is top, and the lowest one told apart
extern "C" float weights(float top, double c, int shift, const float* x, int n, u64* out) {
  double table[kExpTable];
  for (int j = 0; j < kExpTable; ++j) table[j] = Weigher::entry(j, top, c, ldexp(1., shift));
  const Weigher w = Weigher::of(table, top, c);
  for (int i = 0; i < n; ++i) out[i] = w(x[i]);
  return w.lowest;
}
"""
F = np.float32
LOWEST = -np.finfo(np.float32).max
TEMPERATURES = [float(F(10.0 ** e)) for e in range(-30, 31)] + [0.3, 0.7, 1.3, 2.0 ** -149, 3e38]
TOPS = [0.0, 1e-38, 1e-20, 1e-6, 0.1, 1.0, 8.0, 20.0, 127.0, 1e3, 6e4, 1e6, 1e8, 1.1e9, 2e9, 1e10,
        1e11, 1e12, 1e13, 1e30, 3e38]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    compiler = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    if not os.path.exists(compiler):
        pytest.skip("ROCm toolchain not found")
    d = tmp_path_factory.mktemp("weights")
    src, out = d / "weights.hip", d / "weights.so"
    src.write_text(SHIM)
    r = subprocess.run([compiler, "--offload-arch=gfx950", "-O2", "-std=c++17", "-shared", "-fPIC",
                        "-I", CSRC, str(src), "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    lib = ctypes.CDLL(str(out))
    lib.weights.restype = ctypes.c_float
    lib.weights.argtypes = [ctypes.c_float, ctypes.c_double, ctypes.c_int, ctypes.c_void_p,
                            ctypes.c_int, ctypes.c_void_p]
    return lib


def _below(x, n):
    out = [F(x)]
    with np.errstate(over="ignore"):
        for _ in range(n):
            out.append(np.nextafter(out[-1], F(-np.inf)))
    return out


def _factor(t):
    return 64 * 1.4426950408889634074 / t


@pytest.mark.parametrize("shift", [44, 42])
def test_weights_of_every_temperature(lib, shift):
    """Every weight is off by half a step and 2^-44 of itself: the series' next term is 3.9e-14 of
    it, the exponent's own rounding up to 31 * 2^-53 on either side, the rest a few 2^-53.  So
    what weighs nothing has weight 0, however small the temperature and however large the logits."""
    looked_at = 0
    for t in TEMPERATURES:
        for top in (F(s * x) for x in TOPS for s in (1, -1)):
            c = _factor(t)
            if not abs(float(top) * c) < 2.0 ** 48:
                continue
            with np.errstate(over="ignore"):
                far = (float(top) - t * np.linspace(0, 60, 121)).astype(F)
            x = np.array(_below(top, 300) + list(far) + [LOWEST], dtype=F)
            x = x[np.isfinite(x)]
            out = np.zeros(len(x), dtype=np.uint64)
            lowest = lib.weights(top, c, shift, x.ctypes.data, len(x), out.ctypes.data)
            x = np.concatenate([x, np.array(_below(lowest, 3) + [np.nextafter(F(lowest), top)], dtype=F)])
            x = np.ascontiguousarray(x[np.isfinite(x)])
            out = np.zeros(len(x), dtype=np.uint64)
            lib.weights(top, c, shift, x.ctypes.data, len(x), out.ctypes.data)
            ref = np.exp((x.astype(np.float64) - float(top)) / t) * 2.0 ** shift
            off = np.abs(out.astype(np.float64) - ref)
            bad = off > 0.5 + 1e-6 + 2.0 ** -44 * ref
            assert not bad.any(), (t, float(top), x[bad][:4], out[bad][:4], ref[bad][:4])
            looked_at += len(x)
    assert looked_at > 100000


def test_where_all_other_logits_are_too_far(lib):
    """From |x_0 c| = 2^48 on no weight is formed: the float below the largest weighs nothing."""
    for t in TEMPERATURES:
        for x in TOPS:
            for top in (F(x), F(-x)):
                below = float(np.nextafter(top, F(-np.inf)))
                if abs(float(top) * _factor(t)) >= 2.0 ** 48:
                    assert math.exp(max((below - float(top)) / t, -745.0)) * 2.0 ** 44 < 0.5
