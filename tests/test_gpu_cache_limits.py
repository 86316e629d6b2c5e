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
