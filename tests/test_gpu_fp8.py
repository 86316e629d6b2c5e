"""8-bit quantisation and products on the GPU vs the oracle.

Codes and scales are the oracle's exactly: each is one operation, rounded to nearest.

Products, from the kernel's steps: a product of two e4m3 values is exact in fp32 (8 bits of mantissa); a block's up to
128 are summed in the tensor core's fp32 accumulator (at most 2^-23 of the sum of magnitudes for each), scaled by two
scales (one rounding each with the addition's) and summed over the blocks and up to 8 parts of k: at most
(128 * 2^-23 + (2 + K / 128 + 8) 2^-24) sum |x| |w|; a bf16 result is off by 2^-8 of itself more."""
import numpy as np
import pytest

from oracle import dense
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _quantize(x, each, q_stride=None, stream=None):
    import torch
    rows, cols = x.shape
    q = torch.full((rows, q_stride or (cols + 15) // 16 * 16), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((-(-rows // each), -(-cols // 128)), -1.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    binding.rgd_fp8_quantize(x, q, s, each, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    assert bool((q[:, cols:] == 0x55).all())
    return q, s, int(status.item())


@pytest.mark.parametrize("each", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 128), (3, 15), (2, 16), (5, 129), (127, 300), (128, 128), (129, 1000), (300, 257), (2, 4096), (1, 20000)])
def test_quantize(gpu_lib, rows, cols, dtype, each):
    import torch
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    x[:, ::7] *= 0.0
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    want, scales = dense.quantize(x.float().numpy(), each)
    for stride in (None, cols + 3):
        q, s, status = _quantize(x.cuda(), each, stride)
        assert status == 0 and np.array_equal(s.cpu().numpy(), scales) and np.array_equal(q[:, :cols].cpu().numpy(), want)
    wide = torch.zeros(rows, cols + 5, dtype=x.dtype, device="cuda")
    wide[:, 1:cols + 1] = x.cuda()
    q, s, status = _quantize(wide[:, 1:cols + 1], each)  # rows off 16 bytes
    assert np.array_equal(q[:, :cols].cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scales)


@pytest.mark.parametrize("each", [1, 128])
def test_quantize_extremes(gpu_lib, each):
    import torch
    rows = [[0.0] * 8, [3e38, -1e38] + [0.0] * 6, [1e-44, -1e-45] + [0.0] * 6, [2.0 ** -100] * 8, [2.0 ** -99, 2.0 ** -110] * 4, [-0.0] * 8]
    for row in rows:
        x = torch.tensor([row])
        want, scales = dense.quantize(x.numpy(), each)
        q, s, status = _quantize(x.cuda(), each)
        assert status == 0 and np.array_equal(s.cpu().numpy(), scales) and np.array_equal(q[:, :8].cpu().numpy(), want)
    for bad in (float("inf"), float("nan"), -float("inf")):
        x = torch.ones(2, 300)
        x[0, 130] = bad
        q, s, status = _quantize(x.cuda(), each)
        s, odd = s.cpu(), torch.zeros(s.shape, dtype=torch.bool)
        odd[0, 1] = True
        assert status == binding.RGD_DEV_BAD_PARAM and torch.equal(~torch.isfinite(s), odd)
        q = dense.decode_e4m3(q[:, :300].cpu().numpy())
        assert (q[0, :128] == 448).all() and (q[1, 256:] == 448).all()


def _matmul(m, n, k, out="f32", seed=0, pad=0, same=True, x_pad=0, stream=None):
    import torch
    g = torch.Generator().manual_seed(seed + m + n + k)
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[out]
    stride = (k + 15) // 16 * 16 + x_pad
    steps = -(-k // 128)
    codes = [torch.randint(0, 256, (r, stride), generator=g, dtype=torch.uint8) for r in (m, n)]
    for c in codes:
        c[:, :k][(c[:, :k] & 0x7f) == 0x7f] = 0x11  # (no NaN in what counts; behind it there may be)
    sx, sw = torch.rand(m, steps, generator=g) + 0.01, torch.rand(-(-n // 128), steps, generator=g) + 0.01
    y = torch.full((m, n + pad), -7.0, dtype=kind, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (codes[0].cuda(), sx.cuda(), codes[1].cuda(), sw.cuda())
    torch.cuda.synchronize()
    binding.rgd_fp8_matmul(*args, y[:, :n] if pad else y, k=k, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and bool((y[:, n:] == -7).all())
    want, mag = dense.product(codes[0][:, :k].numpy(), sx.numpy(), codes[1][:, :k].numpy(), sw.numpy())
    tol = (128 * 2.0 ** -23 + (10 + k / 128) * 2.0 ** -24) * mag + 1e-30
    if out == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    off = np.abs(y[:, :n].double().cpu().numpy() - want)
    assert (off <= tol).all(), ((off - tol).max(), np.unravel_index((off - tol).argmax(), off.shape))
    return y


@pytest.mark.parametrize("k", [1, 15, 16, 31, 32, 100, 127, 128, 129, 255, 256, 384, 500, 1000, 1024, 1153])
def test_lengths(gpu_lib, k):
    _matmul(3, 50, k)
    _matmul(140, 130, k, "bf16")


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 80, 96, 97, 112, 127, 128, 129, 160, 255, 256, 257, 300])
def test_rows(gpu_lib, m):
    for n, k, out in ((1, 40, "f32"), (127, 300, "bf16"), (128, 1024, "f32"), (129, 640, "bf16"), (500, 200, "f32")):
        _matmul(m, n, k, out, pad=m % 3)


@pytest.mark.parametrize("m, n, k", [(700, 1000, 300), (2600, 2560, 130), (2433, 2312, 260), (5000, 1304, 128), (513, 9001, 140), (20000, 40, 200),
                                     (1, 40000, 512), (100, 21000, 260), (40, 300, 16000), (300, 260, 9000), (128, 128, 20000), (2, 5, 70000)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_sizes(gpu_lib, m, n, k, out):
    _matmul(m, n, k, out)


def test_padded_rows_and_outputs(gpu_lib):
    _matmul(30, 200, 300, pad=8, x_pad=64)
    _matmul(2600, 2561, 200, "bf16", pad=7)  # rows of y that start on 16 bytes and do not end there
    _matmul(2600, 2562, 200, "f32", pad=2)
    _matmul(2600, 2561, 200, "bf16", pad=1)  # and that do not start there
    _matmul(2600, 2568, 200, "bf16", pad=8)
    _matmul(2600, 2564, 200, "f32", pad=8)
    _matmul(2600, 2500, 200, "bf16", pad=12, x_pad=16)
    _matmul(2600, 2500, 200, "f32", pad=4)


@pytest.mark.parametrize("m, n, k", [(5, 3000, 4096), (80, 6144, 4096), (300, 2000, 1024), (3000, 4000, 1024)])
def test_same_result_every_time(gpu_lib, m, n, k):
    import torch
    x, w = (torch.randint(0, 0x70, (r, k), device="cuda", dtype=torch.uint8) for r in (m, n))
    sx, sw = torch.rand(m, k // 128, device="cuda"), torch.rand(-(-n // 128), k // 128, device="cuda")
    first, y = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    binding.rgd_fp8_matmul(x, sx, w, sw, first)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(100):
        binding.rgd_fp8_matmul(x, sx, w, sw, y)
        wrong += (y != first).sum()
    assert int(wrong.item()) == 0


def test_every_value_against_one(gpu_lib):
    """Each of the 254 values, picked one at a time, exactly; the type's and the operands' order."""
    import torch
    codes = torch.tensor([c for c in range(256) if c & 0x7f != 0x7f], dtype=torch.uint8)
    x = torch.zeros(254, 256, dtype=torch.uint8)
    x[range(254), range(254)] = 0x38  # 1
    for m, w in ((254, codes.repeat(3, 1)), (2, codes.repeat(300, 1))):
        wide = torch.zeros(w.shape[0], 256, dtype=torch.uint8)
        wide[:, :254] = w
        y = torch.empty(m, w.shape[0], device="cuda")
        binding.rgd_fp8_matmul(x[:m].cuda(), torch.ones(m, 2, device="cuda"), wide.cuda(),
                               torch.ones(-(-w.shape[0] // 128), 2, device="cuda"), y)
        assert np.array_equal(y.cpu().numpy(), np.repeat(dense.decode_e4m3(codes.numpy())[:m, None], w.shape[0], 1))


def test_nan_and_infinities_stay_in_their_rows(gpu_lib):
    import torch
    for m, n in ((4, 300), (100, 140), (300, 300), (2600, 2600)):
        x, w = (torch.full((r, 256), 0x38, dtype=torch.uint8) for r in (m, n))
        x[1, 200], w[5, 3] = 0x7f, 0xff  # NaN
        sx, sw = torch.ones(m, 2), torch.ones(-(-n // 128), 2)
        sx[2, 1], sx[3, 0] = float("inf"), float("nan")
        y = torch.empty(m, n, device="cuda")
        binding.rgd_fp8_matmul(x.cuda(), sx.cuda(), w.cuda(), sw.cuda(), y)
        y = y.cpu()
        odd = ~torch.isfinite(y)
        want = torch.zeros_like(odd)
        want[1:4], want[:, 5] = True, True
        assert torch.equal(odd, want) and bool((y[0, :5] == 256).all())


def test_quantize_then_multiply(gpu_lib):
    """Random activations and weights through both: near the product of what they were made from, by the type's 2^-4."""
    import torch
    x, w = torch.randn(70, 1000, device="cuda").bfloat16(), torch.randn(200, 1000, device="cuda").bfloat16()
    qx, sx, _ = _quantize(x, 1)
    qw, sw, _ = _quantize(w, 128)
    y = torch.empty(70, 200, device="cuda")
    binding.rgd_fp8_matmul(qx, sx, qw, sw, y, k=1000)
    # each factor is off by 2^-4 of itself at most, and by half of the smallest step of its block, 2^-10 / 448 of the largest
    xd, wd = x.double().abs().cpu(), w.double().abs().cpu()
    tiny = 2.0 ** -10 / 448 * xd.max() * wd.max() * 1000 * 2
    tol = (2 * 2.0 ** -4 + 2.0 ** -8 + 1e-4) * (xd @ wd.T) + tiny
    assert bool(((y.double().cpu() - x.double().cpu() @ w.double().cpu().T).abs() <= tol).all())


def test_stream_and_graph(gpu_lib):
    import torch
    side = torch.cuda.Stream()
    a = _matmul(60, 400, 700, seed=5, stream=side)
    b = _matmul(60, 400, 700, seed=5)
    assert torch.equal(a, b)
    x = torch.randn(60, 700, device="cuda")
    q, s = torch.zeros(60, 704, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(60, 6, device="cuda")
    w, sw = torch.randint(0, 0x70, (400, 704), device="cuda", dtype=torch.uint8), torch.rand(4, 6, device="cuda")
    y = torch.zeros(60, 400, device="cuda")
    binding.rgd_fp8_quantize(x, q, s)
    binding.rgd_fp8_matmul(q, s, w, sw, y, k=700)
    want = y.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.rgd_fp8_quantize(x, q, s, stream=side)
        binding.rgd_fp8_matmul(q, s, w, sw, y, k=700, stream=side)
    for t in (q.view(torch.uint8), s, y):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_two_calls_at_once(gpu_lib):
    import torch
    sides = [torch.cuda.Stream() for _ in range(2)]
    cases = []
    for m, n, k in ((80, 6144, 2048), (2048, 4096, 1024)):
        x, w = (torch.randint(0, 0x70, (r, k), device="cuda", dtype=torch.uint8) for r in (m, n))
        cases.append((x, torch.rand(m, k // 128, device="cuda"), w, torch.rand(-(-n // 128), k // 128, device="cuda"), torch.empty(m, n, device="cuda")))
    alone = []
    for c in cases:
        binding.rgd_fp8_matmul(*c)
        alone.append(c[4].clone())
        c[4].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for side, c in zip(sides, cases):
            binding.rgd_fp8_matmul(*c, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(c[4], a) for c, a in zip(cases, alone))


def test_offsets_past_32_bits(gpu_lib):
    """Rows of y past 2^32 bytes, and rows of weights past them."""
    import torch
    m, n, k = 9000, 262144, 128
    x = torch.randint(0, 0x70, (m, k), device="cuda", dtype=torch.uint8)
    w = torch.randint(0, 0x70, (n, k), device="cuda", dtype=torch.uint8)
    sx, sw = torch.rand(m, 1, device="cuda"), torch.rand(n // 128, 1, device="cuda")
    y = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    binding.rgd_fp8_matmul(x, sx, w, sw, y)
    torch.cuda.synchronize()
    rows, cols = [0, 4095, 8191, 8192, m - 1], [0, 128, n - 129, n - 1]
    want, mag = dense.product(x[rows].cpu().numpy(), sx[rows].cpu().numpy(), w[cols].cpu().numpy(), np.ones((1, 1)))
    want, mag = (a * sw.cpu().numpy()[np.array(cols) // 128, 0] for a in (want, mag))
    off = np.abs(y[rows][:, cols].double().cpu().numpy() - want)
    assert (off <= 2.0 ** -8 * np.abs(want) + 200 * 2.0 ** -23 * mag).all()
    del y
    n, k = 40000, 131072  # 5.2e9 bytes of weights
    w = torch.zeros(n, k, dtype=torch.uint8, device="cuda")
    w[n - 1, k - 1] = w[n // 2, 5] = 0x38
    x = torch.full((2, k), 0x38, dtype=torch.uint8, device="cuda")
    y = torch.empty(2, n, device="cuda")
    binding.rgd_fp8_matmul(x, torch.ones(2, k // 128, device="cuda"), w, torch.ones(-(-n // 128), k // 128, device="cuda"), y)
    assert y.nonzero().tolist() == [[0, n // 2], [0, n - 1], [1, n // 2], [1, n - 1]] and float(y.sum()) == 4
