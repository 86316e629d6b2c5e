"""T ln p of a min-p cutoff: the kernel's function, compiled for the host from its own source with IEEE
arithmetic in place of CUDA's functions of the same rounding, against fl32 of the FP64 product."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2607_20791_gb300.build import CSRC

SHIMS = r"""
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#define __device__
#define __noinline__
#define __forceinline__ inline
static inline float __fadd_rn(float a, float b) { return a + b; }
static inline float __fsub_rn(float a, float b) { return a - b; }
static inline float __fmul_rn(float a, float b) { return a * b; }
static inline float __fdiv_rn(float a, float b) { return a / b; }
static inline float __fmaf_rn(float a, float b, float c) { return fmaf(a, b, c); }
static inline uint32_t __float_as_uint(float a) { uint32_t u; memcpy(&u, &a, 4); return u; }
static inline float __uint_as_float(uint32_t u) { float a; memcpy(&a, &u, 4); return a; }
#include "log_pair.cuh"
int main() {
  float in[2];
  while (fread(in, 4, 2, stdin) == 2) {
    const float out = rgd::scaled_log(in[0], in[1]);
    fwrite(&out, 4, 1, stdout);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def scaled_log(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("scaled_log")
    (at / "main.cpp").write_text(SHIMS)
    res = subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-I", CSRC, str(at / "main.cpp"), "-o", str(at / "main")],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(temp, p):
        pairs = np.stack([np.asarray(temp, np.float32), np.asarray(p, np.float32)], -1)
        out = subprocess.run([str(at / "main")], input=pairs.tobytes(), capture_output=True, timeout=300).stdout
        return np.frombuffer(out, np.float32)
    return run


def _want(temp, p):
    with np.errstate(over="ignore", divide="ignore"):
        return (np.asarray(temp, np.float32).astype(np.float64) * np.log(np.asarray(p, np.float32).astype(np.float64))).astype(np.float32)


def test_a_product_past_fp32_is_minus_infinity(scaled_log):
    """A finite temperature times a logarithm may be past fp32's range: everything is kept then."""
    temp, p = (a.ravel() for a in np.meshgrid([3.3e36, 1e37, 1e38, 3.4e38], [1.2e-38, 1e-30, 0.01, 0.3, 0.9]))
    want = _want(temp, p)
    assert np.isneginf(want).any() and np.isfinite(want).any()
    assert np.array_equal(scaled_log(temp, p), want)


def test_the_ends_of_the_range(scaled_log):
    temp = np.array([1.0, 0.5, 3e38, 1e-30, 2.0])
    assert np.array_equal(scaled_log(temp, np.zeros(5)), np.full(5, -np.inf, np.float32))
    assert np.array_equal(scaled_log(temp, np.ones(5)), np.zeros(5, np.float32))
    assert not np.isnan(scaled_log(temp, np.full(5, 1e-45))).any()


def test_rounded_once(scaled_log):
    """Pairs whose product lies within 1e-6 of an ulp from half way between two floats, and random ones over the range."""
    near = np.array([[0x40cf8728, 0x3f3b5801], [0x4107e9cf, 0x3cafb2e0]], np.uint32).view(np.float32)
    assert np.array_equal(scaled_log(*near.T), _want(*near.T))
    rng = np.random.default_rng(0)
    n = 2_000_000
    temp = np.concatenate([rng.uniform(0.01, 20, n), np.exp2(rng.uniform(-149, 128, n))]).astype(np.float32)
    p = np.concatenate([rng.random(n), np.exp2(rng.uniform(-149, 0, n))]).astype(np.float32)
    ok = np.isfinite(temp) & (temp > 0) & (p > 0) & (p <= 1)
    temp, p = temp[ok], p[ok]
    got, want = scaled_log(temp, p), _want(temp, p)
    wrong = np.flatnonzero(got != want)
    assert wrong.size == 0, [(float(temp[i]).hex(), float(p[i]).hex(), got[i], want[i]) for i in wrong[:5]]
