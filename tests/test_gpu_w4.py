"""Products with 4-bit weights on the GPU vs the fp64 oracle.

The bound, from the kernel's steps: a product of a bf16 with a whole number of 4 bits is
exact in fp32; a group's products are summed in the tensor core's fp32 accumulator (at
most 2^-23 of the sum of magnitudes for each of up to 128 terms), scaled (one rounding) and
summed over the groups and the warps (at most K / 32 + 64 roundings of 2^-24): in all at
most (129 + K / 64 + 32) 2^-23 sum |x| |w|; a bf16 result is the fp32 one, rounded."""
import numpy as np
import pytest

from oracle import drafting
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _run(m, n, k, group, zeros=False, scales="bf16", out="f32", seed=0, pad=0, stream=None, x=None):
    import torch
    g = torch.Generator().manual_seed(seed * 1000 + m + n + k)
    groups = -(-k // group)
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = torch.randn(m, k, generator=g).to(torch.bfloat16) if x is None else x
    w = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8)
    s = (torch.rand(n, groups, generator=g) + 0.1).to(kind[scales])
    z = torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8) if zeros else None
    y = torch.full((m, n + pad), -7.0, dtype=kind[out], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = [x.cuda(), w.cuda(), s.cuda(), None if z is None else z.cuda()]
    torch.cuda.synchronize()
    binding.rgd_w4_matvec(*args, group, y, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert (y[:, n:] == -7).all()
    if out == "bf16":
        whole = torch.zeros((m, n), device="cuda")
        binding.rgd_w4_matvec(*args, group, whole, dev_status=status)
        assert torch.equal(y[:, :n], whole.to(torch.bfloat16))
        got = whole.double().cpu().numpy()
    else:
        got = y[:, :n].double().cpu().numpy()
    xd, sd = x.double().numpy(), s.double().numpy()
    ref = drafting.w4_product(xd, w.numpy(), sd, None if z is None else z.numpy(), group)
    mag = np.abs(xd) @ np.abs(drafting.w4_matrix(w.numpy(), sd, None if z is None else z.numpy(), group, k)).T
    tol = (161 + k / 64) * 2.0 ** -23 * mag + 1e-30
    worst = np.abs(got - ref) - tol
    assert (worst <= 0).all(), (np.abs(got - ref).max(), np.unravel_index(worst.argmax(), worst.shape))
    return y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 64, 96, 127, 128, 160, 255, 256, 352, 512, 1000, 1024, 2730])
def test_lengths(gpu_lib, k, zeros, group):
    _run(3, 50, k, group, zeros, seed=1)


@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 15, 16, 17, 24, 31, 32, 33, 40, 70])
@pytest.mark.parametrize("n, k", [(1, 64), (15, 300), (33, 512), (257, 768)])
def test_rows(gpu_lib, m, n, k):
    _run(m, n, k, 64, True, "f32", "bf16" if m % 2 else "f32", seed=2)


@pytest.mark.parametrize("m, n, k, group", [(1, 4096, 4096, 128), (5, 5000, 4096, 128), (12, 2100, 4096, 32), (20, 2100, 2048, 64),
                                            (3, 40, 16384, 128), (16, 70, 20000, 32), (32, 40, 9000, 128), (2, 20011, 512, 128),
                                            (8, 20011, 1366, 32), (1, 1, 65536, 128), (9, 5000, 2730, 32), (30, 3000, 1111, 64)])
@pytest.mark.parametrize("scales, out", [("bf16", "f32"), ("f32", "bf16")])
def test_sizes(gpu_lib, m, n, k, group, scales, out):
    _run(m, n, k, group, k % 3 == 0, scales, out, seed=3, pad=5)


@pytest.mark.parametrize("m, n, k, group", [(3, 60007, 200, 128), (5, 40000, 512, 64), (2, 50001, 600, 32), (12, 40003, 384, 128),
                                            (9, 30000, 300, 32), (6, 60000, 1024, 128)])
@pytest.mark.parametrize("zeros", [False, True])
def test_warps_with_whole_tiles(gpu_lib, m, n, k, group, zeros):
    """So many rows of W that a warp's share holds tiles of its own and parts of tiles shared with others."""
    _run(m, n, k, group, zeros, seed=6)


@pytest.mark.parametrize("m, n, k, group", [(5, 128256, 4096, 128), (1, 128256, 4096, 64), (12, 128256, 4096, 128),
                                            (8, 128256, 4096, 32), (5, 128256, 2730, 128), (13, 20011, 2730, 32)])
def test_same_result_every_time(gpu_lib, m, n, k, group):
    """A place in the ring is copied over only once it has been read: what comes early gives other sums."""
    import torch
    x = torch.randn(m, k, device="cuda").to(torch.bfloat16)
    w = torch.randint(0, 256, (n, (k + 1) // 2), device="cuda", dtype=torch.uint8)
    s = torch.rand(n, -(-k // group), device="cuda").to(torch.bfloat16)
    first, y = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    binding.rgd_w4_matvec(x, w, s, None, group, first)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        binding.rgd_w4_matvec(x, w, s, None, group, y)
        wrong += (y != first).sum()
    assert int(wrong.item()) == 0


def test_every_weight_and_zero_point(gpu_lib):
    """Each 4-bit value against each zero point, exactly: x picks one weight at a time."""
    import torch
    k = 64
    x = torch.zeros(k, k, dtype=torch.bfloat16)
    x[range(k), range(k)] = 1.0
    w = torch.randint(0, 256, (48, 32), generator=torch.Generator().manual_seed(4), dtype=torch.uint8)
    z = torch.arange(96, dtype=torch.uint8).reshape(48, 2) % 16
    s = torch.ones(48, 2)
    y = torch.zeros(k, 48, device="cuda")
    binding.rgd_w4_matvec(x.cuda(), w.cuda(), s.cuda(), z.cuda(), 32, y)
    want = drafting.w4_unpack(w.numpy(), k) - z.numpy().astype(int)[:, np.arange(k) // 32]
    assert np.array_equal(y.cpu().numpy().T, want)


def test_infinities_and_nan_stay_in_their_row_of_x(gpu_lib):
    import torch
    for m in (3, 10, 20):
        x = torch.randn(m, 200).to(torch.bfloat16)
        x[1, 7] = float("inf")
        x[2, 100] = float("nan")
        w = torch.randint(0, 256, (40, 100), dtype=torch.uint8) | 0x11  # (no weight of q = 8: 0 x inf)
        y = torch.zeros(m, 40, device="cuda")
        binding.rgd_w4_matvec(x.cuda(), w.cuda(), torch.ones(40, 7, device="cuda"), None, 32, y)
        y = y.cpu()
        assert torch.isfinite(y[0]).all() and torch.isfinite(y[3:]).all()
        assert torch.isinf(y[1]).all() and torch.isnan(y[2]).all()


@pytest.mark.parametrize("k", [33, 201, 202, 203, 1111, 1114])
def test_rows_of_x_off_alignment_end_where_they_end(gpu_lib, k):
    """A vector of x that holds the end of a row holds the start of the next."""
    import torch
    x = torch.randn(5, k).to(torch.bfloat16)
    x[1, 0], x[3, -1] = float("inf"), float("nan")
    w = torch.randint(0, 256, (40, (k + 1) // 2), dtype=torch.uint8) | 0x11
    y = torch.zeros(5, 40, device="cuda")
    binding.rgd_w4_matvec(x.cuda(), w.cuda(), torch.ones(40, -(-k // 64), device="cuda"), None, 64, y)
    y = y.cpu()
    assert torch.isfinite(y[[0, 2, 4]]).all()
    assert torch.isinf(y[1]).all() and torch.isnan(y[3]).all()


def test_stream_graph_and_repeat(gpu_lib):
    import torch
    side = torch.cuda.Stream()
    a = _run(4, 300, 640, 32, True, seed=5, stream=side)
    b = _run(4, 300, 640, 32, True, seed=5)
    assert torch.equal(a, b)
    x, w = torch.randn(4, 640, device="cuda").bfloat16(), torch.randint(0, 256, (300, 320), device="cuda", dtype=torch.uint8)
    s, y = torch.rand(300, 5, device="cuda"), torch.zeros(4, 300, device="cuda")
    binding.rgd_w4_matvec(x, w, s, None, 128, y)
    want = y.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.rgd_w4_matvec(x, w, s, None, 128, y, stream=side)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
