"""Head norms and rotation on the GPU vs the fp64 oracle.

The bound, from the kernel's steps, relative to S = |a| + |b| of a pair after the norm and its weights, times the
magnitude: the angle is off by 2^-32 of a turn and by its rounding to 24 bits of a half turn (2^-25 pi < 1e-7),
sine and cosine by 2 units each (2^-22 with the magnitude's rounding), the norm's sum by up to (log2 D + D / 32 + 2)
roundings of fp32 (half of which reach its root) and its root by 2^-22; weights, products and sums by six roundings of 2^-24: in
all under (1e-7 + 3 * 2^-22 + (40 + 6) * 2^-24) S < 4e-6 S for D up to 1024.  A bf16 result is off by 2^-8 of itself
more, the result of fp32 rounded."""
import numpy as np
import pytest

from oracle import dense
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _case(tokens, heads, kv, dim, rot, layout="half", norm=True, scaling="none", dtype="bf16", weights="bf16", seed=0, far=4000, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed + tokens + dim + rot)
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}
    turns, magnitude = binding.rgd_rope_frequencies(rot, 10000.0, scaling, 8.0, 1024.0)
    freq, _ = dense.frequencies(rot, 10000.0, scaling, 8.0, 1024.0)
    shape = binding.RopeShape(num_q_heads=heads, num_k_heads=kv, head_dim=dim, rotary_dim=rot,
                              layout=binding.RGD_ROPE_HALF if layout == "half" else binding.RGD_ROPE_PAIRS, norm=int(norm), eps=1e-5,
                              magnitude=magnitude)
    qkv = (2 * torch.randn(tokens, (heads + 2 * kv) * dim + pad, generator=g)).to(kind[dtype])
    w = None if weights is None or not norm else [(1 + 0.3 * torch.randn(dim, generator=g)).to(kind[weights]) for _ in range(2)]
    pos = torch.randint(-far, far, (tokens,), generator=g, dtype=torch.int32)
    return shape, turns, freq, qkv, w, pos


def _views(qkv, shape):
    hq, hk, d = shape.num_q_heads, shape.num_k_heads, shape.head_dim
    body = qkv[..., :(hq + 2 * hk) * d].unflatten(-1, (hq + 2 * hk, d))
    return body[..., :hq, :], body[..., hq:hq + hk, :], body[..., hq + hk:, :]


def _agrees(got, x, pos, shape, freq, weight, layout, dtype):
    eps = shape.eps if shape.norm else None
    w = None if weight is None else weight.double().numpy()
    x = x.double().numpy()
    want = dense.rotate(x, pos.numpy(), freq, layout, shape.magnitude, w, eps)
    plain = np.abs(dense.rotate(x, 0 * pos.numpy(), 0 * freq, layout, 1.0, w, eps))
    size = plain.copy()  # |a| + |b| of each value's pair
    h = len(freq)
    a, b = (slice(0, h), slice(h, 2 * h)) if layout == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    size[..., a] = size[..., b] = (plain[..., a] + plain[..., b]) * abs(shape.magnitude)
    tol = 4e-6 * size + 1e-30
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= tol).all(), (off - tol).max()


def _run(layout="half", dtype="bf16", stream=None, **kw):
    import torch
    shape, turns, freq, qkv, w, pos = _case(layout=layout, dtype=dtype, **kw)
    dev = qkv.cuda()
    q, k, _ = _views(dev, shape)
    q_out = torch.full((qkv.shape[0], shape.num_q_heads, shape.head_dim), 7.0, dtype=qkv.dtype, device="cuda")
    k_out = torch.full((qkv.shape[0], shape.num_k_heads, shape.head_dim), 7.0, dtype=qkv.dtype, device="cuda")
    wq, wk = (None, None) if w is None else (w[0].cuda(), w[1].cuda())
    before = dev.clone()
    torch.cuda.synchronize()
    binding.rgd_qk_rope(shape, q, k, pos.cuda(), turns.cuda(), wq, wk, q_out, k_out, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(dev, before)
    for got, x, i in ((q_out, _views(qkv, shape)[0], 0), (k_out, _views(qkv, shape)[1], 1)):
        _agrees(got, x, pos, shape, freq, None if w is None else w[i], layout, dtype)
    return q_out, k_out


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim, rot", [(64, 64), (128, 128), (128, 64), (80, 20), (96, 24), (256, 64), (72, 72), (72, 36), (8, 8), (2, 2),
                                      (10, 6), (36, 34), (66, 66), (512, 512), (1024, 256), (1000, 6), (64, 0), (33, 0), (37, 30), (5, 2)])
def test_sizes(gpu_lib, dim, rot, dtype, layout):
    _run(layout, dtype, tokens=5, heads=3, kv=2, dim=dim, rot=rot)


@pytest.mark.parametrize("heads, kv", [(1, 1), (7, 1), (32, 8), (5, 5), (64, 3), (1, 0), (0, 9)])
@pytest.mark.parametrize("tokens", [1, 2, 33, 700])
def test_heads_and_tokens(gpu_lib, tokens, heads, kv):
    import torch
    if heads and kv:
        _run(tokens=tokens, heads=heads, kv=kv, dim=64, rot=64, scaling="bands")
        return
    shape, turns, freq, qkv, w, pos = _case(tokens, max(heads, 1), max(kv, 1), 64, 64)
    q, k, _ = _views(qkv, shape)
    shape.num_q_heads, shape.num_k_heads = heads, kv
    args = [x.cuda() if n else None for x, n in ((q, heads), (k, kv))]
    outs = [torch.empty(tokens, n, 64, dtype=qkv.dtype, device="cuda") if n else None for n in (heads, kv)]
    binding.rgd_qk_rope(shape, *args, pos.cuda(), turns.cuda(), w[0].cuda(), w[1].cuda(), *outs)
    torch.cuda.synchronize()
    x, got, i = (q, outs[0], 0) if heads else (k, outs[1], 1)
    _agrees(got, x, pos, shape, freq, w[i], "half", "bf16")


@pytest.mark.parametrize("kw", [dict(norm=False), dict(weights=None), dict(weights="f32"), dict(dtype="f32", weights="f32"),
                                dict(scaling="ramp"), dict(scaling="ramp", norm=False, layout="pairs"), dict(scaling="linear"),
                                dict(scaling="base"), dict(pad=1), dict(pad=3, layout="pairs"), dict(pad=4), dict(pad=8), dict(pad=2, dtype="f32")])
def test_kinds(gpu_lib, kw):
    _run(**{**dict(tokens=50, heads=6, kv=2, dim=128, rot=128), **kw})
    _run(**{**dict(tokens=9, heads=3, kv=1, dim=80, rot=20), **kw})


def test_far_positions_are_exact(gpu_lib):
    """At positions up to the last int the angle is what 64 bits give: in fp32 it would be off by whole turns."""
    import torch
    shape, turns, freq, qkv, _, _ = _case(4, 2, 1, 128, 128, norm=False, dtype="f32")
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 1000003, 77777777], dtype=torch.int32)
    q, k, _ = _views(qkv.cuda(), shape)
    outs = [torch.empty(4, n, 128, device="cuda") for n in (2, 1)]
    binding.rgd_qk_rope(shape, q, k, pos.cuda(), turns.cuda(), None, None, *outs)
    # the oracle's angles in whole numbers: fp64 would lose 2^31 2^-53 of a turn as well
    t = np.array([[(int(p) * (int(f) % 2 ** 64)) % 2 ** 64 / 2 ** 64 for f in turns] for p in pos])
    x = _views(qkv, shape)[0].double().numpy()
    z = (x[..., :64] + 1j * x[..., 64:]) * np.exp(2j * np.pi * t)[:, None, :]
    want = np.concatenate([z.real, z.imag], -1)
    size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    assert (np.abs(outs[0].double().cpu().numpy() - want) <= 4e-6 * np.concatenate([size, size], -1)).all()


@pytest.mark.parametrize("dim, rot", [(128, 128), (80, 20), (37, 30)])
def test_in_place_gives_the_same(gpu_lib, dim, rot):
    import torch
    shape, turns, freq, qkv, w, pos = _case(40, 8, 2, dim, rot)
    dev = qkv.cuda()
    q, k, v = _views(dev, shape)
    outs = [torch.empty(40, n, dim, dtype=qkv.dtype, device="cuda") for n in (8, 2)]
    args = (pos.cuda(), turns.cuda(), w[0].cuda(), w[1].cuda())
    binding.rgd_qk_rope(shape, q, k, *args, *outs)
    values = v.clone()
    binding.rgd_qk_rope(shape, q, k, *args, q, k)
    assert torch.equal(q, outs[0]) and torch.equal(k, outs[1]) and torch.equal(v, values)


def test_infinities_and_nan_stay_with_their_pair(gpu_lib):
    import torch
    for dim, rot, layout in ((128, 64, "half"), (128, 64, "pairs"), (80, 20, "half"), (80, 20, "pairs"), (37, 10, "half")):
        shape, turns, freq, qkv, _, pos = _case(3, 2, 1, dim, rot, layout, norm=False)
        inf, nan = float("inf"), float("nan")
        q = _views(qkv, shape)[0]
        q[0, 0, rot], q[1, 1, dim - 1], q[2, 0, 0] = inf, nan, inf  # behind the rotated part twice, and in it
        dev = qkv.cuda()
        out, kout = torch.empty(3, 2, dim, dtype=qkv.dtype, device="cuda"), torch.empty(3, 1, dim, dtype=qkv.dtype, device="cuda")
        binding.rgd_qk_rope(shape, *_views(dev, shape)[:2], pos.cuda(), turns.cuda(), None, None, out, kout)
        odd = ~torch.isfinite(out.cpu().float())
        want = torch.zeros_like(odd)
        want[0, 0, rot] = want[1, 1, dim - 1] = want[2, 0, 0] = True
        want[2, 0, rot // 2 if layout == "half" else 1] = True
        assert torch.equal(odd, want) and out[0, 0, rot] == inf and bool(out[1, 1, dim - 1].isnan())


def test_stream_graph_and_strided_output(gpu_lib):
    import torch
    side = torch.cuda.Stream()
    a = _run(tokens=60, heads=4, kv=2, dim=64, rot=32, stream=side)
    b = _run(tokens=60, heads=4, kv=2, dim=64, rot=32)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    shape, turns, _, qkv, w, pos = _case(60, 4, 2, 64, 32)
    dev, t, p, wq, wk = qkv.cuda(), turns.cuda(), pos.cuda(), w[0].cuda(), w[1].cuda()
    wide = torch.full((60, 9, 64), 3.0, dtype=qkv.dtype, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.rgd_qk_rope(shape, *_views(dev, shape)[:2], p, t, wq, wk, wide[:, 1:5], wide[:, 6:8], stream=side)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 1:5], b[0]) and torch.equal(wide[:, 6:8], b[1]) and bool((wide[:, [0, 5, 8]] == 3).all())


# ---------------------------------------------------------------------------
# into pages
# ---------------------------------------------------------------------------
def _paged(rows, new, heads, kv, dim, rot, seed=0, layers=2, **kw):
    import torch
    shape, turns, freq, qkv, w, _ = _case(rows * new, heads, kv, dim, rot, seed=seed, **kw)
    rng = np.random.default_rng(seed)
    length = rng.integers(0, 60, rows).astype(np.int32)
    n_new = rng.integers(0, new + 1, rows).astype(np.int32)
    n_new[0] = new
    counts = (length + n_new + 15) // 16
    pages, cols = int(counts.sum()) + 3, int(counts.max()) + 1
    order, at = rng.permutation(pages).astype(np.int32), 0
    table = np.full((rows, cols), -1, np.int32)
    for r in range(rows):
        table[r, :counts[r]] = order[at:at + counts[r]]
        at += counts[r]
    dev = {k: torch.from_numpy(v).cuda() for k, v in dict(length=length, n_new=n_new, table=table,
                                                         first=rng.integers(-5, 3000, rows).astype(np.int32),
                                                         active=(rng.random(rows) < 0.8).astype(np.uint8)).items()}
    cache = binding.CacheShape(num_layers=layers, num_pages=pages, num_kv_heads=kv, page_size=16, head_dim=dim)
    pools = [torch.randn(layers, pages, kv, 16, dim, device="cuda").bfloat16() for _ in range(2)]
    return shape, turns.cuda(), qkv.view(rows, new, -1).cuda(), w, dev, cache, pools


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows, new, heads, kv, dim, rot", [(1, 1, 4, 1, 64, 64), (7, 3, 8, 2, 128, 128), (20, 8, 3, 3, 80, 20), (5, 40, 4, 2, 96, 24),
                                                            (3, 2, 1, 1, 1024, 1000), (40, 1, 32, 8, 128, 64), (4, 5, 0, 2, 64, 64)])
def test_pages_are_as_rotated_then_written(gpu_lib, rows, new, heads, kv, dim, rot, layout):
    """The same bits as rgd_qk_rope on every token's position and rgd_cache_write of its keys; nothing else changes."""
    import torch
    shape, turns, qkv, w, d, cache, pools = _paged(rows, new, max(heads, 1), kv, dim, rot, layout=layout)
    q, k, v = _views(qkv, shape)
    shape.num_q_heads = heads
    wq, wk = (x.cuda() for x in w)
    pos = (d["first"] + d["length"])[:, None] + torch.arange(new, device="cuda", dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    turned = [torch.empty(rows * new, n, dim, dtype=torch.bfloat16, device="cuda") if n else None for n in (heads, kv)]
    binding.rgd_qk_rope(shape, q.reshape(rows * new, -1, dim) if heads else None, k.reshape(rows * new, -1, dim),
                        pos.reshape(-1).contiguous(), turns, wq, wk, *turned)
    want = [p.clone() for p in pools]
    binding.rgd_cache_write(cache, 1, turned[1].view(rows, new, kv, dim), v.contiguous(), d["n_new"], d["table"], d["length"], d["active"],
                            *want, dev_status=status)
    q_out = torch.full((rows, new, heads, dim), 5.0, dtype=torch.bfloat16, device="cuda") if heads else None
    binding.rgd_qk_rope_cache(shape, cache, 1, q if heads else None, k, v, d["first"], turns, wq, wk, d["n_new"], d["table"], d["length"],
                              d["active"], q_out, *pools, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
    if heads:
        on = (torch.arange(new, device="cuda") < d["n_new"][:, None]) & (d["active"] != 0)[:, None]
        assert torch.equal(q_out[on], turned[0].view(rows, new, heads, dim)[on]) and bool((q_out[~on] == 5).all())


def test_pages_that_are_not_listed(gpu_lib):
    import torch
    shape, turns, qkv, w, d, cache, pools = _paged(6, 4, 2, 1, 64, 64, seed=3)
    q, k, v = _views(qkv, shape)
    d["active"].fill_(1)
    d["n_new"].copy_(torch.tensor([4, 4, 4, -1, 9, 4]))
    d["length"].copy_(torch.tensor([-3, 2, 30, 0, 0, 10 ** 6]))
    d["table"].fill_(0)
    d["table"][1, 0], d["table"][2, 1:] = cache.num_pages, -1
    d["table"][2, 2:] = 2
    d["table"][4, 0] = 1
    before = [p.clone() for p in pools]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full((6, 4, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.rgd_qk_rope_cache(shape, cache, 0, q, k, v, None, turns, None, None, d["n_new"], d["table"], d["length"], None, q_out, *pools,
                              dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == binding.RGD_DEV_BAD_PAGE
    done = (q_out != 5).any(-1).any(-1).cpu()
    # row 2: tokens 30 and 31 have no page, 32 and 33 page 2; row 4: the first max_new; row 0: token 3 - 3 = 0
    want = torch.zeros(6, 4, dtype=torch.bool)
    want[2, 2:] = want[4] = want[0, 3] = True
    assert torch.equal(done, want)
    changed = [(a != b).any(-1).any(2)[0] for a, b in zip(pools, before)]  # [page, slot]
    for c in changed:
        slots = sorted((int(p), int(s)) for p, s in c.nonzero())
        assert slots == [(0, 0)] + [(1, s) for s in range(4)] + [(2, 0), (2, 1)]


def test_offsets_past_32_bits(gpu_lib):
    """Pages that start past 2^32 bytes, and a layer's pool past 2^31 elements, are written where they are."""
    import torch
    pages = 2 ** 31 // (16 * 128 * 8) + 40
    cache = binding.CacheShape(num_layers=2, num_pages=pages, num_kv_heads=8, page_size=16, head_dim=128)
    pools = [torch.zeros(2, pages, 8, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shape, turns, _, qkv, w, _ = _case(3, 4, 8, 128, 128)
    q, k, v = _views(qkv.view(3, 1, -1).cuda(), shape)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.tensor([[pages - 1], [0], [pages // 2]], **i32)
    q_out = torch.empty(3, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([5, 6, 7], **i32)
    args = (turns.cuda(), w[0].cuda(), w[1].cuda())
    binding.rgd_qk_rope_cache(shape, cache, 1, q, k, v, pos, *args, torch.ones(3, **i32), table, torch.zeros(3, **i32), None, q_out, *pools)
    turned = [torch.empty(3, n, 128, dtype=torch.bfloat16, device="cuda") for n in (4, 8)]
    binding.rgd_qk_rope(shape, q[:, 0], k[:, 0], pos, *args, *turned)
    torch.cuda.synchronize()
    for r in range(3):
        assert torch.equal(pools[0][1, table[r, 0], :, 0], turned[1][r]) and torch.equal(pools[1][1, table[r, 0], :, 0], v[r, 0])
    assert torch.equal(q_out[:, 0], turned[0])
    assert int(torch.count_nonzero(pools[1][0, :10])) == 0 and int(torch.count_nonzero(pools[1][1, 1:10])) == 0
