"""The drafting operators where offsets pass 32 bits: logits, weights and pools of more than 2^31 elements or bytes."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


def _free(gigabytes):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30:
        pytest.skip(f"needs {gigabytes} GB free")


@pytest.mark.parametrize("vocab", [128256, 128257])
def test_verification_of_the_last_rows(gpu_lib, vocab):
    """Rows far into a batch of more than 2^31 logits give what they give alone, bit for bit."""
    import torch
    _free(16)
    rows, draft, few = 3500, 4, 5
    g = torch.Generator(device="cuda").manual_seed(vocab)
    t = torch.zeros(rows, draft + 1, vocab, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(rows, draft, vocab, dtype=torch.bfloat16, device="cuda")
    assert t.numel() > 2 ** 31
    for r in range(rows - few, rows):
        t[r] = 2.0 * torch.randn(draft + 1, vocab, generator=g, device="cuda")
        q[r] = t[r, :draft].float() + 0.5 * torch.randn(draft, vocab, generator=g, device="cuda")
    tokens = q.argmax(-1).int()
    temp, min_p = torch.ones(rows, device="cuda"), torch.full((rows,), 0.01, device="cuda")
    temp[-1] = 0.0
    active = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    active[-few:] = 1
    au, du = torch.rand(rows, draft, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    got = []
    for s in (slice(0, rows), slice(rows - few, rows)):
        n = s.stop - s.start
        out, acc = torch.zeros(n, draft + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        prob, status = torch.zeros(n, draft, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.zeros(binding.rgd_verify_draft_workspace_size(n, draft), dtype=torch.uint8, device="cuda")
        args = [a[s] for a in (t, q, tokens, temp, min_p, au, du, active)]
        if n == few:
            args = [a.clone() for a in args]  # (on 16 bytes)
        t_, q_, tokens_, temp_, min_p_, au_, du_, active_ = args
        binding.rgd_verify_draft(t_, q_, tokens_, None, None, temp_, min_p_, au_, du_, active_, out, acc, prob, ws, dev_status=status)
        assert int(status.item()) == 0
        got.append((out[-few:], acc[-few:], prob[-few:]))
    assert bool((got[0][0][:, 0] >= 0).all())
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("m, n, k, group", [(5, 270000, 16384, 128), (12, 270000, 16385, 32)])
def test_products_with_the_last_rows_of_weights(gpu_lib, m, n, k, group):
    """Rows far into more than 2^31 bytes of weights, against the formula in fp64 (the bound: at most K / 32 + 80
    roundings of 2^-24 over the groups, warps and blocks of k, and 129 of 2^-23 within a group)."""
    import torch
    _free(12)
    g = torch.Generator(device="cuda").manual_seed(n + k)
    x = torch.randn(m, k, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand(n, -(-k // group), generator=g, device="cuda") + 0.1
    z = torch.randint(0, 16, s.shape, generator=g, device="cuda", dtype=torch.uint8)
    assert w.numel() > 2 ** 31
    y = torch.zeros(m, n, device="cuda")
    binding.rgd_w4_matvec(x, w, s, z, group, y)
    of, xd = torch.arange(k, device="cuda") // group, x.double()
    for a in (0, 100001, n - 300):
        b = slice(a, a + 300)
        wide = (torch.stack((w[b] & 15, w[b] >> 4), -1).flatten(1)[:, :k].double() - z[b][:, of].double()) * s[b][:, of].double()
        tol = (169 + k / 64) * 2.0 ** -23 * (xd.abs() @ wide.abs().T)
        assert bool(((y[:, b].double() - xd @ wide.T).abs() <= tol).all()), a


def test_pages_and_layers_at_the_end_of_a_large_pool(gpu_lib):
    """A shared page near the end of a pool of more than 2^31 elements a layer: copied, written, copied on and
    moved to the front, in a second layer that starts past 2^32."""
    import torch
    _free(40)
    pages, heads, dim = 140000, 8, 128
    pool = pages * heads * 16 * dim
    stride = 2 ** 32 + 64
    assert pool > 2 ** 31 and stride > pool
    shape = binding.CacheShape(num_layers=2, num_pages=pages, num_kv_heads=heads, page_size=16, head_dim=dim, layer_stride=stride)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.zeros(stride + pool, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    view = lambda p, layer: p[layer * stride:layer * stride + pool].view(pages, heads, 16, dim)
    old, new, other = pages - 10, pages - 5, pages - 1
    for p in (k, v):
        for layer in range(2):
            view(p, layer)[old] = torch.randn(heads, 16, dim, generator=g, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[old], refs[new:] = 2, 0
    table, length = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), i32(5, 5)
    table[:, 0] = old
    ws = torch.empty(binding.rgd_cache_workspace_size(shape, 2), dtype=torch.uint8, device="cuda")
    ok, status, live = torch.zeros(2, dtype=torch.uint8, device="cuda"), i32(0), i32(0)
    n = i32(1, 0)
    binding.rgd_cache_reserve(shape, table, length, n, None, refs, k, v, ok, ws, dev_status=status)
    fresh = torch.randn(2, 2, 1, heads, dim, generator=g, device="cuda").bfloat16()
    for layer in range(2):
        binding.rgd_cache_write(shape, layer, fresh[0], fresh[1], n, table, length, ok, k, v, dev_status=status)
    binding.rgd_cache_copy(shape, i32(new), i32(other), k, v, dev_status=status)
    assert table[:, 0].tolist() == [new, old] and ok.tolist() == [1, 1] and refs[[old, new]].tolist() == [1, 1]
    for p, x in ((k, fresh[0]), (v, fresh[1])):
        for layer in range(2):
            of = view(p, layer)
            for at in (new, other):
                assert torch.equal(of[at, :, :5], of[old, :, :5]) and torch.equal(of[at, :, 5], x[0, 0]) and not bool(of[at, :, 6:].any())
    refs[:] = 0
    refs[old], refs[new] = 1, 1
    want = [[view(p, layer)[at].clone() for at in (old, new)] for p in (k, v) for layer in range(2)]
    binding.rgd_cache_compact(shape, table, None, refs, k, v, live, ws, dev_status=status)
    assert int(status.item()) == 0 and int(live.item()) == 2 and table[:, 0].tolist() == [1, 0] and refs[:3].tolist() == [1, 1, 0]
    got = [[view(p, layer)[at] for at in (0, 1)] for p in (k, v) for layer in range(2)]
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
