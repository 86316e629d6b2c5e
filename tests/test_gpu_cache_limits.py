"""Cache pages at the limits of their arguments."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding
from test_gpu_cache import Cache

pytestmark = pytest.mark.gpu


def test_a_row_of_more_tokens_than_there_are_values_for_is_reported(gpu_lib):
    c = Cache(5, 2, 12, 1, 2, 64, seed=11)
    t = c.torch
    assert c.grow(np.array([4, 4, 4, 4, 4])).all()
    before = c.k.clone()
    x = t.ones(5, 2, 2, 64, dtype=t.bfloat16, device="cuda")
    n = np.array([1, 5, -1, 0, 9])
    active = c.dev([1, 1, 1, 1, 0], t.uint8)
    for rows, want in (([1, 2, 2, 0, 9], 0), (n, binding.RGD_DEV_BAD_PAGE), ([0, 3, 0, 0, 0], binding.RGD_DEV_BAD_PAGE),
                       ([0, 0, -1, 0, 0], binding.RGD_DEV_BAD_PAGE)):
        c.status.zero_()
        c.k.copy_(before)
        binding.rgd_cache_write(c.shape, 0, x, x, c.dev(rows, t.int32), c.table, c.length, active, c.k, c.v, dev_status=c.status)
        t.cuda.synchronize()
        assert int(c.status.item()) == want, rows
        # what there is a value for is written, nothing else
        pool, was = c.k.view(12, 2, 16, 64), before.view(12, 2, 16, 64)
        slots = np.zeros((12, 16), bool)
        for r, count in enumerate(rows):
            if r < 4:
                slots[int(c.table[r, 0]), 4:4 + min(max(count, 0), 2)] = True
        at = t.from_numpy(slots).cuda()[:, None, :, None].expand(12, 2, 16, 64)
        assert bool((pool[at] == 1).all()) and t.equal(pool[~at].view(t.int16), was[~at].view(t.int16))


def test_write_takes_one_head_of_any_stride(gpu_lib):
    """Keys and values as [rows, heads, tokens, D] of one head, transposed: the same as copied dense."""
    c, d = Cache(3, 2, 10, 1, 1, 64, seed=12), Cache(3, 2, 10, 1, 1, 64, seed=12)
    t = c.torch
    k, v = (t.randn(3, 1, 4, 64, device="cuda").bfloat16().transpose(1, 2) for _ in range(2))
    assert k.stride(2) != 64
    for cache, dense in ((c, False), (d, True)):
        n, ok = cache.dev([4, 2, 3], t.int32), t.zeros(3, dtype=t.uint8, device="cuda")
        binding.rgd_cache_reserve(cache.shape, cache.table, cache.length, n, None, cache.refs, cache.k, cache.v, ok, cache.ws,
                                  dev_status=cache.status)
        x = (k.clone(memory_format=t.contiguous_format), v.clone(memory_format=t.contiguous_format)) if dense else (k, v)
        binding.rgd_cache_write(cache.shape, 0, *x, n, cache.table, cache.length, ok, cache.k, cache.v, dev_status=cache.status)
        t.cuda.synchronize()
        assert int(cache.status.item()) == 0
    assert t.equal(c.k.view(t.int16), d.k.view(t.int16)) and t.equal(c.v.view(t.int16), d.v.view(t.int16))
