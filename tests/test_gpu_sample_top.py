"""Sampling with temperature, top-k, top-p and min-p on the GPU vs the fp64 oracle.

Tokens and counts are equal but where a cut or the draw lies within rounding of its threshold.  A weight 2^x: x is a
product and a quotient (three roundings, 3 * 2^-24 of x, |x| < 33 where the weight counts: 2^-17.3 at most), the power
2^-22; so 33 * 3 * 2^-24 ln 2 + 2^-22 < 5e-6 of itself, and half a unit of 2^-31 of the largest weight more.  The
sum of V weights, at least 1, is off by 5e-6 + V 2^-32 of itself; a threshold and the sum up to it by twice that."""
import numpy as np
import pytest

from conftest import report
from oracle import dense
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _call(logits, temp, top_k, top_p, min_p, u, probe=None, active=None, vocab=None, stream=None):
    import torch
    rows = logits.shape[0]
    dev = [None if a is None else a if isinstance(a, torch.Tensor) else torch.as_tensor(np.asarray(a), dtype=d, device="cuda")
           for a, d in ((probe, torch.uint8), (temp, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32),
                        (u, torch.float32), (active, torch.uint8))]
    token, kept = (torch.full((rows,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    prob, status = torch.full((rows,), -9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    binding.rgd_sample_top(logits, dev[0], dev[1], dev[2], dev[3], dev[4], dev[5], dev[6], token, kept, prob, vocab=vocab, dev_status=status,
                           stream=stream)
    torch.cuda.synchronize()
    return token.cpu().numpy(), kept.cpu().numpy(), prob.cpu().numpy(), int(status.item())


def _check(logits, temp, top_k, top_p, min_p, u, vocab=None, name="", **kw):
    vocab = vocab or logits.shape[1]
    rows = logits[:, :vocab].float().cpu().numpy()
    token, kept, prob, status = _call(logits, temp, top_k, top_p, min_p, u, vocab=vocab, **kw)
    assert status == 0
    band, near = 2 * (5e-6 + vocab * 2.0 ** -32), 0
    for r in range(len(rows)):
        want = dense.sample(rows[r], float(temp[r]), int(top_k[r]), float(top_p[r]), float(min_p[r]), float(u[r]), band)
        near += want.near
        if not want.near:
            assert (token[r], kept[r]) == (want.token, want.kept), (r, temp[r], top_k[r], top_p[r], min_p[r], u[r], token[r], kept[r], want)
            # (weights below 2^-20 of the largest have few of the 2^-31)
            assert abs(prob[r] - want.prob) <= band * want.prob + 2.0 ** -31
    if name:
        report(f"sampling {name}: {near} of {len(rows)} rows near a threshold")
    # (where the tokens about a threshold weigh less than the band each, as in a long tail at top_p 0.999, or where
    # the threshold is an edge, as 0.8 of 50 equal ones, no arithmetic in fp32 decides)
    assert near <= 2 + len(rows) // 2


def _params(rows, rng):
    t = rng.choice([0.0, 0.3, 0.7, 1.0, 2.0, 5.0], rows)
    k = rng.choice([0, 0, 1, 5, 50, 1000, 3000, 10 ** 6], rows)
    p = rng.choice([1.0, 1.0, 0.999, 0.95, 0.8, 0.3, 0.01], rows)
    m = rng.choice([0.0, 0.0, 0.02, 0.2], rows)
    return t.astype(np.float32), k, p.astype(np.float32), m.astype(np.float32), rng.random(rows).astype(np.float32)


def _logits(rows, vocab, kind, dtype, seed, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed + vocab)
    x = torch.zeros(rows, vocab + pad)
    if kind == "zipf":
        for r in range(rows):
            x[r, :vocab] = -1.1 * torch.log(torch.arange(1, vocab + 1.0))[torch.randperm(vocab, generator=g)]
    elif kind == "sorted":
        x[:, :vocab] = -torch.linspace(0, 25, vocab)
    elif kind == "steps":  # few values, many ties
        x[:, :vocab] = (2 * torch.randn(rows, vocab, generator=g)).round() / 2
    elif kind == "zeros":  # -0 and 0 are the same
        x[:, :vocab] = torch.where(torch.rand(rows, vocab, generator=g) < 0.5, -0.0, 0.0)
    elif kind == "junk":  # most of the row is never drawn
        x[:, :vocab] = 3 * torch.randn(rows, vocab, generator=g)
        x[:, vocab // 5:vocab] -= 60
    elif kind == "few":  # a mask of -inf, or of the type's lowest value
        x[:, :vocab] = torch.randn(rows, vocab, generator=g)
        x[:, :vocab][torch.rand(rows, vocab, generator=g) < 0.99] = -float("inf") if seed % 2 else torch.finfo(torch.bfloat16).min
        x[:, vocab // 2] = 1.0
    else:
        x[:, :vocab] = {"normal": 3.0, "flat": 0.01, "wide": 1e4}[kind] * torch.randn(rows, vocab, generator=g)
    if pad:
        x[:, vocab:] = 1e5  # (behind a row's end: not read as logits)
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 32, 33, 100, 255, 256, 257, 1000, 2047, 2049, 5000])
def test_small_vocabularies(gpu_lib, vocab, dtype):
    rng = np.random.default_rng(vocab)
    for pad in (0, 1, 8):
        _check(_logits(24, vocab, "normal", dtype, pad, pad).cuda(), *_params(24, rng), vocab=vocab)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["zipf", "sorted", "steps", "zeros", "junk", "few", "normal", "flat", "wide"])
@pytest.mark.parametrize("rows, vocab, pad", [(16, 3001, 0), (12, 32000, 0), (10, 32001, 2), (6, 128256, 0)])
def test_distributions(gpu_lib, rows, vocab, pad, kind, dtype):
    rng = np.random.default_rng(vocab + len(kind))
    _check(_logits(rows, vocab, kind, dtype, rows, pad).cuda(), *_params(rows, rng), vocab=vocab, name=f"{rows} x {vocab} {dtype} {kind}")


@pytest.mark.parametrize("rows, vocab, dtype", [(300, 5931, "bf16"), (700, 1000, "f32"), (150, 20000, "bf16"), (3, 500000, "f32"), (2, 1 << 20, "bf16"),
                                                (2, 1 << 20, "f32"), (310, 70001, "bf16")])
def test_batches(gpu_lib, rows, vocab, dtype):
    rng = np.random.default_rng(rows)
    _check(_logits(rows, vocab, "zipf", dtype, 1).cuda(), *_params(rows, rng), name=f"{rows} x {vocab} {dtype}")


@pytest.mark.parametrize("top_k", [1, 2, 31, 33, 255, 256, 257, 511, 1023, 1024, 1025, 2048, 2049, 4095, 20000, 39999, 40000])
def test_counts(gpu_lib, top_k):
    """Every kept token by its place: few values, so that the cut lies among equal ones."""
    for kind, dtype in (("steps", "bf16"), ("zipf", "f32"), ("flat", "f32"), ("flat", "bf16")):
        x = _logits(4, 40000, kind, dtype, top_k).cuda()
        u = np.array([0.0, 0.37, 0.9999999, 0.73], np.float32)
        _check(x, np.full(4, 1.7), np.full(4, top_k), np.array([1, 1, 1, 0.9], np.float32), np.zeros(4), u)


def test_draws_reach_every_kept_token_and_no_other(gpu_lib):
    """A row's 40 kept tokens among 9000, by 4000 uniforms: as often as their weights say, exactly."""
    import torch
    row = _logits(1, 9000, "zipf", "f32", 3)
    n = 4000
    x = row.expand(n, -1).contiguous().cuda()
    u = (np.arange(n) + 0.5) / n
    token, kept, prob, status = _call(x, np.full(n, 1.3), np.full(n, 40), None, None, u)
    assert status == 0 and (kept == 40).all()
    top = torch.topk(row[0], 40).indices.numpy()
    w = np.exp((row[0, top].double().numpy() - float(row.max())) / np.float64(np.float32(1.3)))
    p = dict(zip(top.tolist(), w / w.sum()))
    assert set(token.tolist()) <= set(top.tolist()) and (np.diff(token) >= 0).all()
    for t, q in p.items():
        assert abs((token == t).sum() - n * q) <= 1 + 1e-4 * n
        assert np.allclose(prob[token == t], q, rtol=2e-5)


def test_greedy_inactive_and_null_arguments(gpu_lib):
    import torch
    x = _logits(6, 1001, "steps", "f32", 4)
    x[2, 5] = float("nan")
    probe, active = [1, 0, 1, 0, 0, 1], [1, 1, 1, 0, 1, 0]
    # (greedy rows read no other parameter)
    token, kept, prob, status = _call(x.cuda(), [5.0, 0.0, float("nan"), 1.0, 1.0, 1.0], [3] * 6, [2.0, -1.0, 0.5, 0.5, 1.0, 0.5],
                                      [7.0] * 4 + [0.0] * 2, [2.0, -1.0, 0.5, 0.5, 0.0, 0.0], probe, active)
    assert status == 0
    best = [int(np.argmax(np.where(np.isnan(r), -np.inf, r))) for r in x.numpy()]
    first = int(np.sort(np.argsort(-x[4].numpy(), kind="stable")[:3])[0])
    assert token.tolist() == [best[0], best[1], best[2], -1, first, -1]
    assert kept.tolist() == [1, 1, 1, 0, 3, 0] and prob.tolist()[:4] == [1, 1, 1, 0]
    # all filters absent: every token, as by rgd_sample_head's draw of the same uniform in order of the indices
    u = np.array([0.0, 0.2, 0.5, 0.8, 0.99, 0.999999], np.float32)
    y = _logits(6, 1001, "normal", "f32", 5)
    a = _call(y.cuda(), np.ones(6), None, None, None, u)
    b = _call(y.cuda(), np.ones(6), np.zeros(6), np.ones(6), np.zeros(6), u)
    assert all(np.array_equal(p, q) for p, q in zip(a, b)) and (a[1] == 1001).all()
    token = torch.full((6,), -9, dtype=torch.int32, device="cuda")
    binding.rgd_sample_top(y.cuda(), None, torch.ones(6, device="cuda"), None, None, None, torch.from_numpy(u).cuda(), None, token)
    assert np.array_equal(token.cpu().numpy(), a[0])


@pytest.mark.parametrize("kw", [dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")), dict(top_p=-0.1), dict(top_p=1.1),
                                dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan")), dict(u=1.0), dict(u=-0.1),
                                dict(u=float("nan")), dict(logit=float("inf")), dict(logit=None)])
def test_rejected_rows(gpu_lib, kw):
    for vocab in (70, 50000):
        x = _logits(3, vocab, "normal", "f32", 6)
        if "logit" in kw:
            if kw["logit"] is None:
                x[1] = -float("inf")
            else:
                x[1, 60] = kw["logit"]
        a = {n: np.full(3, v, np.float32) for n, v in dict(temp=1.0, top_p=0.9, min_p=0.0, u=0.5).items()}
        for n, v in kw.items():
            if n != "logit":
                a[n][1] = v
        token, kept, prob, status = _call(x.cuda(), a["temp"], [0, 5, 7], a["top_p"], a["min_p"], a["u"])
        assert status == binding.RGD_DEV_BAD_PARAM and (token[1], kept[1], prob[1]) == (-1, 0, 0)
        good = _call(x[[0, 2]].cuda(), [1.0, 1.0], [0, 7], [0.9, 0.9], [0.0, 0.0], [0.5, 0.5])
        assert good[3] == 0 and np.array_equal(token[[0, 2]], good[0]) and np.array_equal(kept[[0, 2]], good[1])


def test_parameters_at_their_ends(gpu_lib):
    x = _logits(8, 6000, "normal", "f32", 7).cuda()
    z = np.zeros(8)
    u = np.linspace(0, 0.999, 8).astype(np.float32)
    best = x.argmax(-1).cpu().numpy()
    for kw in (dict(t=1e-38), dict(t=1e-30), dict(k=1), dict(p=0.0), dict(p=1e-30), dict(m=1.0)):
        token, kept, _, status = _call(x, np.full(8, kw.get("t", 1.0)), np.full(8, kw.get("k", 0)), np.full(8, kw.get("p", 0.9)), np.full(8, kw.get("m", 0.0)), u)
        assert status == 0 and np.array_equal(token, best) and (kept == 1).all(), kw
    token, kept, prob, status = _call(x, np.full(8, 3e38), z, z + 1, z, u)  # as good as uniform
    assert status == 0 and (kept == 6000).all() and np.array_equal(token, (u.astype(np.float64) * 6000).astype(int))
    token, kept, _, status = _call(x, np.full(8, 3e38), z, z + 0.5, z, u)
    assert status == 0 and (kept == 3000).all()
    token, kept, _, status = _call(x, np.full(8, 3e38), z + 4000, z + 0.5, z, u)
    assert status == 0 and (kept == 2000).all()


@pytest.mark.parametrize("rows, vocab, dtype", [(80, 128256, "bf16"), (5, 32001, "f32"), (300, 5931, "bf16")])
def test_same_result_every_time(gpu_lib, rows, vocab, dtype):
    """Back to back, so that calls overlap: what a block reads of another is read before it is written again."""
    import torch
    rng = np.random.default_rng(9)
    x = _logits(rows, vocab, "zipf", dtype, 8).cuda()
    t, k, p, m, u = (torch.as_tensor(a, device="cuda") for a in _params(rows, rng))
    out = [torch.zeros(rows, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    first, wrong = None, torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        binding.rgd_sample_top(x, None, t, k.int(), p, m, u, None, *out)
        if first is None:
            first = [o.clone() for o in out]
        wrong += sum((a != b).sum() for a, b in zip(out, first))
    assert int(wrong.item()) == 0


def test_two_calls_at_once(gpu_lib):
    """On streams of their own, beside a product whose blocks want the same SMs."""
    import torch
    sides = [torch.cuda.Stream() for _ in range(3)]
    rng = np.random.default_rng(21)
    cases = []
    for rows, vocab, dtype in ((80, 128256, "bf16"), (200, 5931, "f32")):
        t, k, p, m, u = (torch.as_tensor(a, device="cuda") for a in _params(rows, rng))
        out = [torch.zeros(rows, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
        cases.append((_logits(rows, vocab, "zipf", dtype, rows).cuda(), None, t, k.int(), p, m, u, None, *out))
    x, w = (torch.randint(0, 0x70, (r, 1024), device="cuda", dtype=torch.uint8) for r in (1000, 4000))
    product = (x, torch.rand(1000, 8, device="cuda"), w, torch.rand(32, 8, device="cuda"), torch.empty(1000, 4000, device="cuda"))
    calls = [(binding.rgd_sample_top, c, c[-3:]) for c in cases] + [(binding.rgd_fp8_matmul, product, product[-1:])]
    alone = []
    for call, args, out in calls:
        call(*args)
        alone.append([o.clone() for o in out])
        for o in out:
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for side, (call, args, _) in zip(sides, calls):
            call(*args, stream=side)
    torch.cuda.synchronize()
    for (_, _, out), want in zip(calls, alone):
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_strided_rows_stream_and_graph(gpu_lib):
    import torch
    side = torch.cuda.Stream()
    wide = _logits(20, 4096, "zipf", "bf16", 11).cuda()
    x = wide[::2, 8:3008]  # (every other row, from 16 bytes on)
    rng = np.random.default_rng(12)
    args = _params(10, rng)
    a = _call(x.contiguous(), *args)
    b = _call(x, *args, stream=side)
    assert all(np.array_equal(p, q) for p, q in zip(a, b))
    t, k, p, m, u = (torch.as_tensor(v, device="cuda") for v in args)
    k = k.int()
    token = torch.zeros(10, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.rgd_sample_top(x, None, t, k, p, m, u, None, token, stream=side)
    token.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(token.cpu().numpy(), a[0])


def test_offsets_past_32_bits(gpu_lib):
    """Rows that start past 2^32 bytes."""
    import torch
    rows, vocab = 9000, 262144
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(rows, device="cuda") * 7919) % vocab
    x[torch.arange(rows, device="cuda"), at] = 20.0
    ones = torch.ones(rows, device="cuda")
    token, kept = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    binding.rgd_sample_top(x, None, ones, (50 * ones).int(), 0.9 * ones, None, 0.5 * ones, None, token, kept)
    torch.cuda.synchronize()
    assert torch.equal(token.long(), at) and bool((kept == 1).all())
