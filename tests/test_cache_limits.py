"""Sizes at which the cache's entry points have to refuse, on the host, before any launch."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2607_20791_gb300 import binding
from paper_2607_20791_gb300.build import CSRC, INCLUDE, build

P = 1 << 12  # any non-NULL, 16-byte aligned stand-in pointer


@pytest.fixture(scope="module")
def lib():
    return binding.load_library(build())


@pytest.mark.parametrize("rows, cols", [(1 << 15, 1 << 16), (1 << 26, 32), (0x7fffffff, 2), (46341, 46341)])
def test_reserve_refuses_more_table_entries_than_it_counts(lib, rows, cols):
    """Rows that each want all of their entries add up to more than the kernel's 32-bit sums hold: what is past
    them would be taken as places among the free pages."""
    s = ctypes.byref(binding.CacheShape(num_layers=1, num_pages=10, num_kv_heads=1, page_size=16, head_dim=8))
    # (host addresses stand in for the tensors, so a call that were let through would be launched: the workspace is too small
    # for it, and which of the two it is refused for shows)
    assert lib.rgd_cache_reserve(s, rows, cols, P, P, P, None, P, P, P, None, P, 0, None, None) == binding.RGD_ERR_UNSUPPORTED
    assert b"entries" in lib.rgd_last_error_string()
    assert lib.rgd_cache_reserve(s, 1 << 15, (1 << 16) - 1, P, P, P, None, P, P, P, None, P, 0, None, None) == binding.RGD_ERR_INVALID_ARG
    assert b"too small" in lib.rgd_last_error_string()


GRID = r"""
#include <cstdio>
#include "common.h"
int rgd::set_error(int code, const char*, ...) { return code; }
int main() {
  const int64_t items[] = {1, 8, 9, 9728, 9729, 1ll << 31, 1ll << 34, (1ll << 34) + 1, 1ll << 35, 1ll << 56};
  for (int64_t n : items) printf("%d ", rgd::blocks_for(n, 8, 1216));
  printf("%d\n", rgd::blocks_for(0x7fffffff, 8));
  return 0;
}
"""


def test_blocks_of_more_work_than_32_bits_count(tmp_path):
    """A copy of many pages in many layers and heads has more pieces than an int: its grid is still the most there is."""
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    if not os.path.exists(os.path.join(inc, "cuda_runtime.h")) or not shutil.which("g++"):
        pytest.skip("no CUDA headers or no g++")
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(GRID)
    stubs = tmp_path / "stubs.cpp"
    stubs.write_text('#include <cuda_runtime.h>\nextern "C" const char* cudaGetErrorString(cudaError_t) { return "fake"; }\n')
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-I", INCLUDE, "-I", inc, str(src), str(stubs), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert [int(x) for x in res.stdout.split()] == [1, 1, 2, 1216, 1216, 1216, 1216, 1216, 1216, 1216, 268435456]


def test_rows_next_to_the_last_int_are_refused(lib):
    """A kernel's last block has a few rows too many, whose numbers have to stay an int for it to leave them out."""
    s = ctypes.byref(binding.CacheShape(num_layers=1, num_pages=10, num_kv_heads=1, page_size=16, head_dim=8))

    def refused(rc):
        assert rc == binding.RGD_ERR_INVALID_ARG and b"too many" in lib.rgd_last_error_string()
    for rows in (0x7fffffff, 0x7fffffff - 1023):
        refused(lib.rgd_cache_trim(rows, 1, 10, P, P, None, P, None, None))
        refused(lib.rgd_cache_fork(rows, P, P, 2, 1, 10, P, P, P, None, None))
        refused(lib.rgd_cache_write(s, 0, rows, 1, P, P, 0, 0, P, 1, P, P, None, P, P, None, None))
        refused(lib.rgd_cache_reserve(s, rows, 1, P, P, P, None, P, P, P, None, P, 1 << 60, None, None))
    refused(lib.rgd_cache_write(s, 0, 0x3fffffff, 2, P, P, 0, 0, P, 1, P, P, None, P, P, None, None))
