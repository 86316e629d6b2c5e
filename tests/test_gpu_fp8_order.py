"""8-bit products: which calls give the same bits, and scales far from 1."""
import numpy as np
import pytest

from oracle import dense
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m, n, k", [(2048, 1280, 8192), (300, 1280, 4096), (80, 640, 2048)])
def test_same_strides_give_the_same_bits(gpu_lib, m, n, k):
    """Rows of y on 16 bytes or off them may be summed in another order (parts of k by several blocks or by one); calls
    with one stride agree bit for bit, wherever their tensors lie, and strides agree within the products' tolerance:
    twice (128 * 2^-23 + (10 + k / 128) 2^-24) of the sum of magnitudes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x, w = (torch.randint(0, 0x70, (r, k), generator=g, device="cuda", dtype=torch.uint8) for r in (m, n))
    sx, sw = (torch.rand(r, k // 128, generator=g, device="cuda") + 0.01 for r in (m, -(-n // 128)))
    results = []
    for pad in (0, 1):
        same = []
        for _ in range(2):
            y = torch.zeros(m, n + pad, device="cuda")
            binding.rgd_fp8_matmul(x.clone(), sx, w.clone(), sw, y[:, :n])
            same.append(y[:, :n])
        assert torch.equal(*same)
        results.append(same[0].double())
    # (no value is negative, so that the results are the sums of magnitudes)
    tol = 2 * (128 * 2.0 ** -23 + (10 + k / 128) * 2.0 ** -24) * results[0].abs()
    assert bool(((results[0] - results[1]).abs() <= tol).all())


@pytest.mark.parametrize("m", [3, 200])
def test_scales_far_from_one(gpu_lib, m):
    """A block's sum is multiplied by its scales' product, rounded to fp32: scales that undo each other leave it, and
    products past fp32's range are infinite or 0."""
    import torch
    n, k = 256, 256
    rng = np.random.default_rng(m)
    x, w = (rng.integers(0x30, 0x40, (r, k)).astype(np.uint8) for r in (m, n))
    sums, _ = dense.product(x, np.ones((m, 2)), w, np.ones((2, 2)))
    dev = [torch.from_numpy(a).cuda() for a in (x, w)]
    for up, down, want in ((2.0 ** 119, 2.0 ** -119, sums), (2.0 ** -109, 2.0 ** 109, sums), (2.0 ** -60, 2.0 ** -60, sums * 2.0 ** -120),
                           (2.0 ** 90, 2.0 ** 90, np.full(sums.shape, np.inf)), (2.0 ** -90, 2.0 ** -90, np.zeros(sums.shape))):
        y = torch.zeros(m, n, device="cuda")
        binding.rgd_fp8_matmul(dev[0], torch.full((m, 2), up, device="cuda"), dev[1], torch.full((2, 2), down, device="cuda"), y)
        got = y.double().cpu().numpy()
        if np.isinf(want).all():
            assert np.array_equal(got, want)
        else:
            assert (np.abs(got - want) <= (128 * 2.0 ** -23 + 12 * 2.0 ** -24) * want).all()
