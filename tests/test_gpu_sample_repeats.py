"""Sampling called back to back with four blocks a row in several rounds over the SMs: the same result every time.

Rows of such a call start while others of it are searched, and the next call's blocks while this one's last rows
are: a word of shared memory that were given out again before every thread has read it would show here."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding
from test_gpu_sample_top import _logits, _params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, vocab, dtype, kind, calls", [(310, 70001, "bf16", "zipf", 200), (310, 35001, "f32", "normal", 200),
                                                             (512, 152064, "bf16", "normal", 60)])
def test_same_result_every_time(gpu_lib, rows, vocab, dtype, kind, calls):
    import torch
    x = _logits(rows, vocab, kind, dtype, 31).cuda()
    t, k, p, m, u = (torch.as_tensor(a, device="cuda") for a in _params(rows, np.random.default_rng(32)))
    k = k.int()
    out = [torch.zeros(rows, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first, wrong = None, torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(calls):
        binding.rgd_sample_top(x, None, t, k, p, m, u, None, *out, dev_status=status)
        if first is None:
            first = [o.clone() for o in out]
        wrong += sum((a != b).sum() for a, b in zip(out, first))
    assert int(status.item()) == 0 and int(wrong.item()) == 0
    assert bool((first[0] >= 0).all()) and bool((first[1] >= 1).all())
