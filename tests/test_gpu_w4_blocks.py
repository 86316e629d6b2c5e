"""Products with 4-bit weights whose x does not fit shared memory: k goes in blocks, with the sums of a block's
tiles kept between them, vs the formula in fp64.

The bound: a product of a bf16 with a whole number of 4 bits is exact in fp32; a group's products are summed
in the tensor core's fp32 accumulator (at most 2^-23 of the sum of magnitudes for each of up to 128 terms),
scaled (one rounding) and summed over the groups, the warps and at most 16 blocks of k (K / 32 + 64 + 16
roundings of 2^-24): in all at most (129 + K / 64 + 40) 2^-23 sum |x| |w|."""
import pytest

from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _inputs(m, n, k, group, zeros, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + m + n + k)
    groups = -(-k // group)
    x = torch.randn(m, k, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = (torch.rand(n, groups, generator=g, device="cuda") + 0.1).to(torch.bfloat16 if k % 3 else torch.float32)
    z = torch.randint(0, 16, (n, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return x, w, s, z


def _check(m, n, k, group, zeros):
    import torch
    x, w, s, z = _inputs(m, n, k, group, zeros)
    y = torch.full((m, n + 3), -7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.rgd_w4_matvec(x, w, s, z, group, y, dev_status=status)
    assert int(status.item()) == 0 and bool((y[:, n:] == -7).all())
    of = torch.arange(k, device="cuda") // group
    xd = x.double()
    for a in range(0, n, 4096):
        part = w[a:a + 4096]
        q = torch.stack((part & 15, part >> 4), -1).flatten(1)[:, :k].double()
        wide = (q - (8.0 if z is None else z[a:a + 4096][:, of].double())) * s[a:a + 4096][:, of].double()
        tol = (169 + k / 64) * 2.0 ** -23 * (xd.abs() @ wide.abs().T)
        off = (y[:, a:min(a + 4096, n)].double() - xd @ wide.T).abs() - tol
        assert float(off.max()) <= 0, (a, float(off.max()))


# (one tile to a block of the grid, a few, more than are kept at a time; k in 2 to 4 blocks; rows of W on 16 bytes and off)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("m, n, k, group", [
    (5, 4000, 8192, 64), (8, 5000, 8192, 128), (5, 5000, 9001, 32), (8, 9000, 9001, 64), (5, 9000, 9001, 128), (6, 5000, 14336, 32),
    (7, 9000, 14336, 64), (5, 8192, 14336, 128), (12, 4096, 5120, 128), (16, 4096, 5120, 32), (12, 5000, 8192, 64), (16, 9000, 9001, 32),
    (12, 5000, 9001, 128), (16, 5000, 14336, 64), (20, 5000, 8192, 32), (20, 4000, 9001, 128), (33, 5000, 5120, 64),
    (5, 120000, 6144, 128), (12, 90000, 4099, 32),
])
def test_blocks_of_k(gpu_lib, m, n, k, group, zeros):
    _check(m, n, k, group, zeros)


@pytest.mark.parametrize("m, n, k, group", [
    (12, 2000, 8192, 32), (5, 2000, 14336, 64), (5, 2000, 9001, 128), (20, 2000, 9001, 64), (3, 70, 131072, 128), (5, 70, 65536, 64),
    (12, 70, 65536, 32), (5, 33, 100001, 128), (20, 70, 70002, 128),
])
def test_blocks_of_k_in_a_cluster(gpu_lib, m, n, k, group):
    """Few tiles of long rows: the blocks of a cluster share a tile, and each one's part of k goes in blocks."""
    _check(m, n, k, group, n % 2 == 1)


@pytest.mark.parametrize("m, n, k, group", [(5, 120000, 6144, 128), (12, 9000, 9001, 32), (16, 5000, 14336, 64), (12, 2000, 8192, 32)])
def test_same_result_every_time(gpu_lib, m, n, k, group):
    """The sums kept between blocks of k and the rings that the next block fills: read before they change."""
    import torch
    x, w, s, z = _inputs(m, n, k, group, True, seed=1)
    first, y = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    binding.rgd_w4_matvec(x, w, s, z, group, first)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        binding.rgd_w4_matvec(x, w, s, z, group, y)
        wrong += (y != first).sum()
    assert int(wrong.item()) == 0
