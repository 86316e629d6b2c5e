"""Sizes at which the cache's entry points have to refuse, on the host, before any launch."""
import ctypes

import pytest

from paper_2607_20791_gb300 import binding
from paper_2607_20791_gb300.build import build

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
