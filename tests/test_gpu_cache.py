"""Cache pages on the GPU vs the oracle, exactly: tables, counts, lengths and every value of the pools."""
import numpy as np
import pytest

from oracle import drafting
from paper_2607_20791_gb300 import binding

pytestmark = pytest.mark.gpu


class Cache:
    """The same cache on both sides; pools hold random 16-bit patterns (also those of NaN and infinity)."""

    def __init__(self, rows, cols, pages, layers=2, heads=2, dim=64, seed=0, gap=0):
        import torch
        self.torch, self.rng = torch, np.random.default_rng(seed)
        self.rows, self.cols, self.pages, self.layers, self.heads, self.dim = rows, cols, pages, layers, heads, dim
        pool = pages * heads * 16 * dim
        self.stride = pool + gap
        self.shape = binding.CacheShape(num_layers=layers, num_pages=pages, num_kv_heads=heads, page_size=16, head_dim=dim,
                                        layer_stride=self.stride if gap else 0)
        host = self.rng.integers(0, 1 << 16, (2, layers, self.stride)).astype(np.uint16)
        self.k, self.v = (torch.from_numpy(h.view(np.int16).copy()).cuda().view(torch.bfloat16) for h in host)
        self.gap = host[:, :, pool:]
        # the oracle's pools: [page, slot, everything else]
        data = host[:, :, :pool].reshape(2, layers, pages, heads, 16, dim).transpose(2, 4, 0, 1, 3, 5)
        self.ref = drafting.Pages(np.full((rows, cols), -1), np.zeros(rows, int), np.zeros(pages, int), data)
        i32 = torch.int32
        self.table = torch.full((rows, cols), -1, dtype=i32, device="cuda")
        self.length, self.refs = torch.zeros(rows, dtype=i32, device="cuda"), torch.zeros(pages, dtype=i32, device="cuda")
        self.ws = torch.empty(binding.rgd_cache_workspace_size(self.shape, rows), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=i32, device="cuda")
        self.live = torch.zeros(1, dtype=i32, device="cuda")

    def dev(self, a, kind):
        return self.torch.from_numpy(np.ascontiguousarray(a)).to("cuda", kind)

    def grow(self, n, active=None, most=None):
        """Reserves and writes n tokens a row, raises the lengths where there was room; returns row_ok."""
        t = self.torch
        n, act = np.asarray(n), None if active is None else self.dev(active, t.uint8)
        ok = t.full((self.rows,), 9, dtype=t.uint8, device="cuda")
        new = self.dev(n, t.int32)
        binding.rgd_cache_reserve(self.shape, self.table, self.length, new, act, self.refs, self.k, self.v, ok, self.ws,
                                  dev_status=self.status)
        want = self.ref.reserve(n, active)
        assert np.array_equal(ok.cpu().numpy(), want)
        most = max(1, int(n.max())) if most is None else most
        values = self.rng.integers(0, 1 << 16, (2, self.layers, self.rows, most, self.heads, self.dim)).astype(np.uint16)
        dev = self.dev(values.view(np.int16), t.int16).view(t.bfloat16)
        for layer in range(self.layers):
            binding.rgd_cache_write(self.shape, layer, dev[0, layer], dev[1, layer], new, self.table, self.length, ok, self.k,
                                    self.v, dev_status=self.status)
        self.ref.write(values.transpose(2, 3, 0, 1, 4, 5), n, want)
        self.ref.length = self.ref.length + np.where(want, n, 0)
        self.length.copy_(self.dev(self.ref.length, t.int32))
        return want

    def trim(self, length, active=None):
        act = None if active is None else self.dev(active, self.torch.uint8)
        lens = self.dev(length, self.torch.int32)
        binding.rgd_cache_trim(self.table, lens, act, self.refs, dev_status=self.status)
        self.ref.trim(length, active)
        keep = np.ones(self.rows, bool) if active is None else np.asarray(active, bool)
        self.ref.length = np.where(keep, length, self.ref.length)
        self.length.copy_(self.dev(self.ref.length, self.torch.int32))

    def fork(self, parent, child):
        i32 = self.torch.int32
        binding.rgd_cache_fork(self.dev(parent, i32), self.dev(child, i32), self.table, self.length, self.refs,
                               dev_status=self.status)
        self.ref.fork(parent, child)

    def compact(self, second=None):
        binding.rgd_cache_compact(self.shape, self.table, second, self.refs, self.k, self.v, self.live, self.ws,
                                  dev_status=self.status)
        return self.ref.compact()

    def check(self, status=0):
        self.torch.cuda.synchronize()
        assert int(self.status.item()) == status
        assert np.array_equal(self.table.cpu().numpy(), self.ref.table)
        assert np.array_equal(self.refs.cpu().numpy(), self.ref.refs)
        assert np.array_equal(self.length.cpu().numpy(), self.ref.length)
        got = np.stack([p.view(self.torch.int16).cpu().numpy().view(np.uint16) for p in (self.k, self.v)])
        got = got.reshape(2, self.layers, self.stride)
        pool = self.pages * self.heads * 16 * self.dim
        assert np.array_equal(got[:, :, pool:], self.gap)
        got = got[:, :, :pool].reshape(2, self.layers, self.pages, self.heads, 16, self.dim).transpose(2, 4, 0, 1, 3, 5)
        assert np.array_equal(got, self.ref.data)


@pytest.mark.parametrize("layers, heads, dim, gap", [(1, 1, 8, 0), (2, 2, 64, 0), (1, 8, 128, 0), (3, 1, 24, 64), (2, 5, 72, 8)])
def test_random_steps(gpu_lib, layers, heads, dim, gap):
    """Rows grow, fork, roll back, end and are compacted at random; everything is compared after each step."""
    c = Cache(7, 6, 40, layers, heads, dim, seed=dim, gap=gap)
    rng = np.random.default_rng(dim)
    for step in range(60):
        op = rng.integers(5)
        if op <= 1:
            n = np.minimum(rng.integers(0, 20, 7), 6 * 16 - c.ref.length)
            active = rng.integers(0, 4, 7) > 0 if op else None
            if (c.grow(n, active) == 0).any() and active is None:
                c.status.zero_()
            c.status.bitwise_and_(~binding.RGD_DEV_NO_PAGE)  # (a full pool is one of the states)
        elif op == 2:
            c.trim(np.array([rng.integers(0, l + 1) for l in c.ref.length]), rng.integers(0, 2, 7).astype(np.uint8))
        elif op == 3:
            rows = rng.permutation(7)
            parent, child = rows[[0, 0, 1]], rows[2:5]
            c.trim(np.zeros(7, int), np.isin(np.arange(7), child).astype(np.uint8))
            c.fork(parent, child)
        else:
            assert c.compact() == int(c.live.item())
        c.check()


def test_lengths_zero_one_and_page_ends(gpu_lib):
    c = Cache(9, 4, 60, 1, 2, 64, seed=1)
    for n in ([0, 1, 15, 16, 17, 31, 32, 33, 64], [1, 15, 1, 0, 15, 1, 16, 15, 0], [63, 16, 16, 16, 0, 17, 0, 1, 0]):
        assert c.grow(np.array(n)).all()
        c.check()
    c.trim(np.array([0, 1, 15, 16, 17, 32, 33, 48, 63]))
    c.check()
    c.trim(np.zeros(9, int))
    assert (c.ref.refs == 0).all()
    c.check()


def test_forked_rows_copy_before_they_write(gpu_lib):
    """A parent and its children all write into the page they share; whoever rolled back into shared pages and
    writes there again gets a page of its own."""
    c = Cache(6, 5, 40, 2, 2, 64, seed=2)
    c.grow(np.array([37, 0, 0, 0, 0, 0]))
    c.fork([0, 0, 0], [1, 2, 3])
    c.check()
    assert c.ref.refs.max() == 4
    c.grow(np.array([3, 3, 0, 20, 0, 0]))
    c.check()
    c.fork([2, 2], [4, 5])
    c.trim(np.array([40, 40, 5, 57, 5, 33]))
    c.grow(np.array([1, 1, 1, 1, 30, 1]))  # (rows 2 and 4 are back inside the first, shared page)
    c.check()


def test_full_pool_serves_rows_in_order(gpu_lib):
    """Rows whose pages and those before them exceed the free ones are left as they were."""
    c = Cache(5, 4, 6, 1, 1, 8, seed=3)
    ok = c.grow(np.array([32, 16, 64, 16, 0]))
    assert ok.tolist() == [1, 1, 0, 0, 0]  # 2 + 1 pages, then 4 do not fit the 3 left, nor those after them
    c.check(status=binding.RGD_DEV_NO_PAGE)
    c.status.zero_()
    assert c.grow(np.array([0, 0, 0, 16, 16])).all()
    c.check()


def test_wrong_rows_are_left_alone(gpu_lib):
    c = Cache(6, 2, 20, 1, 1, 8, seed=4)
    c.grow(np.array([5, 5, 5, 5, 5, 5]))
    t = c.torch
    before = c.table.clone(), c.refs.clone()
    lens = c.dev([5, -1, 30, 5, 5, 5], t.int32)
    new = c.dev([-1, 1, 3, 0, 0, 0], t.int32)
    ok = t.full((6,), 9, dtype=t.uint8, device="cuda")
    binding.rgd_cache_reserve(c.shape, c.table, lens, new, None, c.refs, c.k, c.v, ok, c.ws, dev_status=c.status)
    t.cuda.synchronize()
    assert ok.tolist() == [0, 0, 0, 1, 1, 1] and int(c.status.item()) == binding.RGD_DEV_BAD_PAGE
    assert t.equal(c.table, before[0]) and t.equal(c.refs, before[1])
    # entries outside the pool, pairs outside the rows, a token without a page
    for call in ("reserve", "write", "fork", "copy", "trim"):
        c.status.zero_()
        table = c.table.clone()
        if call == "reserve":
            table[0, 0] = 20
            binding.rgd_cache_reserve(c.shape, table, c.length, c.dev([1, 0, 0, 0, 0, 0], t.int32), None, c.refs, c.k, c.v, ok,
                                      c.ws, dev_status=c.status)
        elif call == "write":
            table[0, 0] = -1
            x = t.zeros(6, 1, 1, 8, dtype=t.bfloat16, device="cuda")
            binding.rgd_cache_write(c.shape, 0, x, x, c.dev([1, 0, 0, 0, 0, 0], t.int32), table, c.length, None, c.k, c.v,
                                    dev_status=c.status)
        elif call == "fork":
            binding.rgd_cache_fork(c.dev([0, 9], t.int32), c.dev([6, 1], t.int32), table, c.length, c.refs, dev_status=c.status)
        elif call == "copy":
            binding.rgd_cache_copy(c.shape, c.dev([0, -1], t.int32), c.dev([20, 1], t.int32), c.k, c.v, dev_status=c.status)
        else:
            table[0, 1] = 20
            binding.rgd_cache_trim(table, c.length, None, c.refs, dev_status=c.status)
        t.cuda.synchronize()
        assert int(c.status.item()) == binding.RGD_DEV_BAD_PAGE, call
    c.status.zero_()
    c.check()


@pytest.mark.parametrize("rows, pages", [(300, 1500), (1024, 4099), (1500, 9000), (3000, 40000), (9000, 20011)])
def test_many_rows_and_pages(gpu_lib, rows, pages):
    """One block or a cluster, one sweep over the counts or several: the pages are the same."""
    c = Cache(rows, 3, pages, 1, 1, 8, seed=5)
    taken = c.rng.permutation(pages)[:pages // 3]  # (pages some other table holds)
    c.ref.refs[taken] = 1
    c.refs.copy_(c.dev(c.ref.refs, c.torch.int32))
    ref = c.ref
    # the oracle's search for the lowest free page, made fast: the free pages in order
    free = iter(np.flatnonzero(ref.refs == 0).tolist())
    ref._take = lambda: next(free)
    c.grow(c.rng.integers(0, 40, rows))
    c.status.bitwise_and_(~binding.RGD_DEV_NO_PAGE)
    c.check()
    c.trim(np.minimum(c.ref.length, c.rng.integers(0, 40, rows)))
    c.ref.refs[taken] = 0  # (that table is gone)
    c.refs.copy_(c.dev(c.ref.refs, c.torch.int32))
    assert c.compact() == int(c.live.item())
    c.check()


def test_copy_and_a_second_table(gpu_lib):
    c = Cache(4, 4, 30, 2, 2, 64, seed=6)
    t = c.torch
    c.grow(np.array([20, 40, 10, 60]))
    binding.rgd_cache_copy(c.shape, c.dev([0, 3], t.int32), c.dev([25, 29], t.int32), c.k, c.v, dev_status=c.status)
    c.ref.data[25], c.ref.data[29] = c.ref.data[0], c.ref.data[3]
    c.check()
    c.trim(np.array([0, 40, 0, 3]))
    second = c.dev([[25, -1, 29]], t.int32)  # pages that another table holds
    c.ref.refs[[25, 29]] = 1
    c.refs.copy_(c.dev(c.ref.refs, t.int32))
    live = c.compact(second)
    t.cuda.synchronize()
    held = second.cpu().numpy()[0]
    assert live == 6 and held[1] == -1 and {int(held[0]), int(held[2])} == set(range(6)) - set(c.ref.table[c.ref.table >= 0])
    c.check()
    # an entry that names a free page past the live ones becomes -1
    stray = c.dev([[28]], t.int32)
    binding.rgd_cache_compact(c.shape, stray, None, c.refs, c.k, c.v, c.live, c.ws, dev_status=c.status)
    t.cuda.synchronize()
    assert stray.item() == -1 and int(c.status.item()) == binding.RGD_DEV_BAD_PAGE


def test_write_takes_views_of_a_fused_projection(gpu_lib):
    c = Cache(3, 2, 10, 1, 2, 64, seed=7)
    t = c.torch
    n = c.dev([2, 3, 0], t.int32)
    ok = t.zeros(3, dtype=t.uint8, device="cuda")
    binding.rgd_cache_reserve(c.shape, c.table, c.length, n, None, c.refs, c.k, c.v, ok, c.ws)
    qkv = t.randn(3, 3, 10, 64, device="cuda").bfloat16()  # 6 query heads, then keys, then values
    binding.rgd_cache_write(c.shape, 0, qkv[:, :, 6:8], qkv[:, :, 8:10], n, c.table, c.length, ok, c.k, c.v, dev_status=c.status)
    t.cuda.synchronize()
    assert int(c.status.item()) == 0
    for r, count in ((0, 2), (1, 3)):
        page = int(c.table[r, 0])
        k = c.k.view(10, 2, 16, 64)[page, :, :count].transpose(0, 1)
        assert t.equal(k, qkv[r, :count, 6:8]) and t.equal(c.v.view(10, 2, 16, 64)[page, :, :count].transpose(0, 1), qkv[r, :count, 8:10])


def test_side_stream_and_graph(gpu_lib):
    """A reserve, a write and a trim as one graph on a side stream, replayed."""
    c = Cache(5, 4, 30, 1, 2, 64, seed=8)
    t = c.torch
    c.grow(np.array([3, 16, 20, 0, 31]))
    c.check()
    n = c.dev([4, 4, 4, 4, 4], t.int32)
    x = t.randn(5, 4, 2, 64, device="cuda").bfloat16()
    ok = t.zeros(5, dtype=t.uint8, device="cuda")
    side = t.cuda.Stream()
    t.cuda.synchronize()

    def step():
        binding.rgd_cache_reserve(c.shape, c.table, c.length, n, None, c.refs, c.k, c.v, ok, c.ws, dev_status=c.status, stream=side)
        binding.rgd_cache_write(c.shape, 0, x, x, n, c.table, c.length, ok, c.k, c.v, dev_status=c.status, stream=side)
        binding.rgd_cache_trim(c.table, c.length, None, c.refs, dev_status=c.status, stream=side)
    step()
    t.cuda.synchronize()
    want = c.table.clone(), c.refs.clone(), c.k.clone()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=side):
        step()
        step()
    graph.replay()
    t.cuda.synchronize()
    assert int(c.status.item()) == 0
    assert t.equal(c.table, want[0]) and t.equal(c.refs, want[1]) and t.equal(c.k.view(t.int16), want[2].view(t.int16))
