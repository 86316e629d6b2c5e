"""Draft verification at the ends of its parameters' ranges, vs the fp64 oracle."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("certain", [False, True])
def test_a_cutoff_past_fp32_keeps_everything(gpu_lib, certain):
    """T ln p_min below fp32's range is -inf: every row is decided, and the workspace serves the next call."""
    c = Case(24, 3, 600, "f32", seed=21, certain=certain, temps=(3.3e36, 1e37, 1e38, 3e38), min_ps=(0.01, 1e-30, 0.3), probe_every=100)
    c.active[:] = 1
    with np.errstate(over="ignore"):
        c.run().check()
    assert not bool(c.ws.any())
    after = Case(24, 3, 600, "f32", seed=22)
    after.run(workspace=c.ws).check()
    assert not bool(c.ws.any())


def test_the_cutoff_is_the_samplers_bit_for_bit(gpu_lib):
    """A token at fl32(T ln p_min) below the largest logit is kept, one an ulp lower is not."""
    import torch
    rng = np.random.default_rng(23)
    rows = 20000
    near = np.array([[0x40cf8728, 0x3f3b5801], [0x4107e9cf, 0x3cafb2e0]], np.uint32).view(np.float32)
    temp = np.concatenate([near[:, 0], rng.uniform(0.01, 20, rows - 2).astype(np.float32)])
    min_p = np.concatenate([near[:, 1], rng.uniform(1e-5, 1 - 1e-5, rows - 2).astype(np.float32)])
    cut = (temp.astype(np.float64) * np.log(min_p.astype(np.float64))).astype(np.float32)
    logits = np.zeros((rows, 3, 4), np.float32)  # (the largest is 0)
    logits[:, :, 1] = cut[:, None]
    logits[:, :, 2] = np.nextafter(cut, np.float32(-np.inf))[:, None]
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    tokens = np.tile(np.array([1, 2], np.int32), (rows, 1))
    out, acc = torch.empty(rows, 3, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    prob, status = torch.empty(rows, 2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(binding.rgd_verify_draft_workspace_size(rows, 2), dtype=torch.uint8, device="cuda")
    binding.rgd_verify_draft(d(logits), None, d(tokens), None, None, d(temp), d(min_p), torch.rand(rows, 2, device="cuda"),
                             torch.rand(rows, device="cuda"), None, out, acc, prob, ws, vocab=3, dev_status=status)
    prob = prob.cpu().numpy()
    assert int(status.item()) == 0
    assert (prob[:, 0] > 0).all() and (prob[:, 1] == 0).all()


@pytest.mark.parametrize("vocab", [200, 40000])
@pytest.mark.parametrize("certain", [False, True])
def test_positions_behind_a_rejection_set_no_status(gpu_lib, certain, vocab):
    """Logits that are not finite and uniforms out of range at positions a row does not get to are no error."""
    c = Case(6, 3, vocab, "f32", seed=24, certain=certain, temps=(1.0,), min_ps=(0.0,), probe_every=100)
    c.active[:], c.n[:], c.probe[:] = 1, 3, [0, 0, 0, 0, 1, 1]
    c.tokens[:, 0] = 5
    c.t[:, 0, 5] = -np.inf  # (rejected in sample rows and greedy ones)
    c.t[0:2, 1:], c.t[2, 2:], c.t[4:, 1:] = np.nan, np.inf, -np.inf
    c.au[1, 1:], c.au[3, 2] = np.nan, 1.5
    c.run()
    assert int(c.status.item()) == 0
    out, acc = c.out.cpu().numpy(), c.acc.cpu().numpy()
    assert (acc == 0).all() and (out[:, 0] >= 0).all() and (out[:, 0] != 5).all() and (out[:, 1:] == -1).all()
    # ... and are one where it gets to them
    c.au[:], c.tokens[:, 0] = 0, np.nanargmax(c.t[:, 0].numpy(), -1)
    c.run()
    assert int(c.status.item()) == binding.RGD_DEV_BAD_PARAM
    assert (c.out.cpu().numpy()[[0, 1, 4, 5]] == -1).all() and (c.acc.cpu().numpy()[[0, 1, 4, 5]] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
def test_masks_of_the_types_lowest_value(gpu_lib, certain, dtype):
    """Masked logits hold the lowest finite value; a position of nothing but masked ones is uniform over the vocabulary."""
    import torch
    c = Case(30, 2, 1500, dtype, seed=25, certain=certain, temps=(1.0, 0.5, 0.0, 3e38), min_ps=(0.0, 0.1), probe_every=9)
    low = torch.finfo(c.t.dtype).min
    c.t[:, :, 200:1400] = low
    c.t[:, 2, 1400:] = low
    if c.q is not None:
        c.q[:, :, 100:1450] = low
    c.t[::7, 0] = low
    c.t[3::11, 1, 7] = -low  # (the largest logit the largest value: differences are past the range)
    c.active[:] = 1
    with np.errstate(over="ignore"):
        c.run().check()
    assert not bool(c.ws.any())
