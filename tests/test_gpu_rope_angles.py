"""The angle of a rotation, at every position an int32 holds and for any fractions of a turn.

(1, 0) becomes (cos t, sin t).  The angle is cut to 2^-32 of a turn and rounded to fp32, by 2^-26 of a turn at most:
2 pi (2^-26 + 2^-32) < 9.6e-8 radians.  Cosine and sine are off by two units of fp32 each (2^-23 for values up to 1),
across the angle by 2^-23 (|cos| + |sin|) <= 1.7e-7."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [binding.RGD_ROPE_HALF, binding.RGD_ROPE_PAIRS])
@pytest.mark.parametrize("dim", [128, 80, 34])
def test_angles_of_any_position(gpu_lib, layout, dim):
    import torch
    rng = np.random.default_rng(dim)
    half = dim // 2
    turns = rng.integers(0, 1 << 63, half, dtype=np.uint64) * np.uint64(2) + np.uint64(1)
    turns[:4] = [0, 1, (1 << 64) - 1, 1 << 63]
    pos = rng.integers(-1 << 31, 1 << 31, 500).astype(np.int32)
    pos[:6] = [0, 1, -1, (1 << 31) - 1, -1 << 31, 500000]
    x = torch.zeros(len(pos), 1, dim)
    if layout == binding.RGD_ROPE_HALF:
        x[..., :half] = 1
    else:
        x[..., ::2] = 1
    out = torch.zeros(len(pos), 1, dim, device="cuda")
    shape = binding.RopeShape(num_q_heads=1, num_k_heads=0, head_dim=dim, rotary_dim=dim, layout=layout, norm=0, eps=0.0, magnitude=1.0)
    binding.rgd_qk_rope(shape, x.cuda(), None, torch.from_numpy(pos).cuda(), torch.from_numpy(turns.view(np.int64)).cuda(), None, None, out, None)
    y = out[:, 0].double().cpu().numpy()
    cos, sin = (y[:, :half], y[:, half:]) if layout == binding.RGD_ROPE_HALF else (y[:, ::2], y[:, 1::2])
    # (whole numbers modulo 2^64, then the fraction of a turn in [-1/2, 1/2))
    part = (pos.astype(np.int64).view(np.uint64)[:, None] * turns[None, :]).view(np.int64).astype(np.float64)
    t = 2 * np.pi * part * 2.0 ** -64
    across = sin * np.cos(t) - cos * np.sin(t)
    assert np.abs(across).max() <= 2 * np.pi * (2.0 ** -26 + 2.0 ** -32) + 2.0 ** -23 * np.sqrt(2)
    assert np.abs(cos * np.cos(t) + sin * np.sin(t) - 1).max() <= 2.0 ** -23 * np.sqrt(2) + 1e-12
