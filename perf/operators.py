"""Measured cases of the drafting operators: what a decode step with drafted tokens
needs around the attention and the sample head.

Every case is a dict of plain values whose ``kind`` names the operator:

* ``verify``   ``rgd_verify_draft``: drafted tokens against the target's probabilities.
* ``w4``       ``rgd_w4_matvec``: a few rows of activations times 4-bit weights.
* ``extend``   the cache side of a drafted step: what the last step's drafts took rolled
               back, pages reserved, the drafted tokens' keys and values written
               (``rgd_cache_trim``, ``rgd_cache_reserve``, ``rgd_cache_write``).
* ``fork``     the last round's children dropped, rows forked from their parents, the
               shared last page of each copied before it is written (``rgd_cache_trim``,
               ``rgd_cache_fork``, ``rgd_cache_reserve``).
* ``compact``  ``rgd_cache_compact``: the pages in use moved to the front of the pool.

Inputs are drawn on the GPU from the seed; lengths and counts go by the row's index, so
that a case's work is a function of the case alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
LOG2E = 1.4426950408889634
ONE = 2.0 ** 31  # weights are summed as whole multiples of 2^-31


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _verify(rows, rpg, draft, vocab, dtype, sampling, point=False, pad=0):
    """rows of logits groups, the first of every rpg a greedy probe; up to `draft` drafted tokens a row."""
    return {"kind": "verify", "rows": rows, "rpg": rpg, "draft": draft, "vocab": vocab, "pad": pad, "dtype": dtype,
            "sampling": sampling, "point": point}


def _w4(rows, k, n, group, scales, zeros, out):
    return {"kind": "w4", "rows": rows, "k": k, "n": n, "group": group, "scales": scales, "zeros": zeros, "out": out}


def _cache(kind, rows, layers, kv_heads, dim, length, new):
    """rows of up to `length` tokens that grow by up to `new`."""
    return {"kind": kind, "rows": rows, "layers": layers, "kv_heads": kv_heads, "dim": dim, "length": length, "new": new}


def listed():
    return [
        # one prompt of a small model, tokens drafted from a phrase list (no draft logits): latency
        {"name": "verify_tiny", **_verify(3, 3, 3, 4096, "f32", "usual", point=True)},
        # the ordinary serving batch: 16 prompts, 1 probe and 4 samples each, 4 drafted tokens a row
        {"name": "verify_8b", **_verify(80, 5, 4, 128256, "bf16", "usual")},
        # long drafts without truncation over an odd vocabulary in rows of their own length: nothing is aligned,
        # every token has a weight
        {"name": "verify_odd", **_verify(24, 3, 7, 32001, "f32", "open")},
        # the largest batch: 256 prompts of two rows, 3 drafted tokens each
        {"name": "verify_batch", **_verify(512, 2, 3, 152064, "bf16", "sweep")},
        # one row through a square projection of a 4096-wide model: launch and latency
        {"name": "w4_proj", **_w4(1, 4096, 4096, 128, "bf16", False, "bf16")},
        # logits of one prompt's five rows from a 4-bit output matrix
        {"name": "w4_head", **_w4(5, 4096, 128256, 128, "bf16", False, "f32")},
        # ragged sizes, small groups with zero points, as many rows as one prompt's drafts have
        {"name": "w4_odd", **_w4(13, 2730, 20011, 32, "f32", True, "bf16")},
        # one prompt's rows, small heads
        {"name": "extend_tiny", **_cache("extend", 5, 1, 2, 64, 200, 4)},
        # a large batch: 2048 rows, 8 tokens each, one layer's pool
        {"name": "extend_batch", **_cache("extend", 2048, 1, 8, 128, 1000, 8)},
        # a single prompt's samples fork from its probe, a few layers
        {"name": "fork_tiny", **_cache("fork", 8, 4, 2, 64, 100, 1)},
        # 64 probes of 512 tokens fork four samples each, 32 layers
        {"name": "fork_8b", **_cache("fork", 320, 32, 8, 128, 512, 4)},
        # a 32-layer pool after most rows have ended
        {"name": "compact_8b", **_cache("compact", 320, 32, 8, 128, 200, 0)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("verify", "verify", "w4", "w4", "extend", "fork", "compact"))
    if kind == "verify":
        draft, dtype = rng.randint(1, 8), rng.choice(("f32", "bf16"))
        vocab = _log(rng, 500, 262144)
        if rng.random() < 0.6:
            vocab = (vocab + 7) // 8 * 8
        most = (600 << 20) // (vocab * (2 * draft + 1) * (4 if dtype == "f32" else 2))
        rows = _log(rng, 1, max(1, min(512, most)))
        pad = rng.choice((0, 0, 8, 64)) if vocab % 8 == 0 else rng.choice((0, 3))
        return _verify(rows, rng.randint(1, 6), draft, vocab, dtype, rng.choice(("usual", "sweep", "open")),
                       rng.random() < 0.25, pad)
    if kind == "w4":
        k = _log(rng, 64, 16384)
        if rng.random() < 0.7:
            k = (k + 63) // 64 * 64
        n = _log(rng, 16, min(131072, (512 << 20) // k))
        return _w4(_log(rng, 1, 32), k, n, rng.choice((32, 64, 128)), rng.choice(("bf16", "f32")), rng.random() < 0.4,
                   rng.choice(("bf16", "f32")))
    heads, dim = rng.choice(((1, 64), (2, 64), (4, 128), (8, 64), (8, 128), (16, 128)))
    layers = 1 if kind == "extend" else rng.choice((1, 2, 4, 16, 32))
    length = _log(rng, 4, 2000)
    most = (2 << 30) // (layers * heads * dim * 4 * (length + 48))
    rows = _log(rng, 2, max(3, min(2048, most)))
    return _cache(kind, rows, layers, heads, dim, length, 0 if kind == "compact" else rng.randint(1, 16))


# ---------------------------------------------------------------------------
# sizes that go by the row's index
# ---------------------------------------------------------------------------
def _n_draft(c):
    """Drafted tokens of each row: most rows have all of them, some fewer, some none."""
    i = np.arange(c["rows"])
    return np.where(i % 4 == 3, (i * 5) % (c["draft"] + 1), c["draft"]).astype(np.int32)


def _active(rows):
    i = np.arange(rows)
    return ((i % 11 != 7) | (rows < 8)).astype(np.uint8)


def _greedy(c):
    """Rows that take the largest logit: the probes, and temperature 0 in a sweep."""
    i = np.arange(c["rows"])
    return (i % c["rpg"] == 0) | ((c["sampling"] == "sweep") & (i % 5 == 0))


def _lengths(c):
    """Tokens of each row, from 0 to c["length"], the last row the longest."""
    i = np.arange(c["rows"])
    n = (i * 7919 + 13) % (c["length"] + 1)
    n[-1] = c["length"]
    return n.astype(np.int32)


def _news(c):
    """Tokens that each row of a cache case gains: most rows all of them, some fewer, some none."""
    i = np.arange(c["rows"])
    return np.where(i % 5 == 4, i % (c["new"] + 1), c["new"]).astype(np.int32)


def _families(c):
    """Parents and children of a fork: rows 0, 5, 10, ... each have the next four."""
    i = np.arange(c["rows"])
    child = i[i % 5 != 0]
    return (child - child % 5).astype(np.int32), child.astype(np.int32)


def _pages(n):
    return (n + PAGE - 1) // PAGE


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFFFFFF)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _kind(name):
    return torch.float32 if name == "f32" else torch.bfloat16


class State:
    pass


def _sampling(c):
    """Temperatures and min-p by row."""
    i = np.arange(c["rows"])
    if c["sampling"] == "sweep":
        t, p = np.array([0.0, 1.0, 2.0, 5.0, 10.0])[i % 5], np.array([0.0, 0.05, 0.1, 0.3])[(i // 5) % 4]
    elif c["sampling"] == "open":
        t, p = np.array([0.7, 1.0, 1.5])[i % 3], np.zeros(c["rows"])
    else:
        t, p = np.array([1.0, 1.5, 2.0, 3.0])[i % 4], np.array([0.05, 0.1])[i % 2]
    return np.where(i % c["rpg"] == 0, 0.0, t).astype(np.float32), p.astype(np.float32)


def _prepare_verify(s, c, seed):
    R, K, V, gen = c["rows"], c["draft"], c["vocab"], _gen(seed, 1)
    base = -1.1 * torch.log(torch.arange(1, V + 1, dtype=torch.float64))
    base = (base - torch.logsumexp(base, 0)).float().to(DEV)
    s.target = torch.zeros((R, K + 1, V + c["pad"]), dtype=_kind(c["dtype"]), device=DEV)
    s.draft = None if c["point"] else torch.zeros((R, K, V + c["pad"]), dtype=_kind(c["dtype"]), device=DEV)
    s.tokens = torch.zeros((R, K), dtype=torch.int32, device=DEV)
    temp, minp = _sampling(c)
    for r in range(R):
        # a Zipf-ranked target, and a draft model that is off by some noise
        rank = torch.randperm(V, generator=gen, device=DEV)
        t = base[rank] + torch.randn((K + 1, V), generator=gen, device=DEV)
        q = t[:K] + 0.5 * torch.randn((K, V), generator=gen, device=DEV)
        s.target[r, :, :V] = t
        if s.draft is not None:
            s.draft[r, :, :V] = q
            q = s.draft[r, :, :V].float()
        if temp[r] > 0:  # a draw from the draft's own truncated distribution
            noise = -torch.log(-torch.log(torch.rand((K, V), generator=gen, device=DEV).clamp(1e-12, 1 - 1e-7)))
            low = q.amax(-1, keepdim=True) + float(temp[r]) * math.log(max(float(minp[r]), 1e-30))
            q = torch.where(q >= low, q / float(temp[r]) + noise, -torch.inf)
        s.tokens[r] = q.argmax(-1)
    s.count = _dev(_n_draft(c))
    i = np.arange(R)
    s.probe = _dev((i % c["rpg"] == 0).astype(np.uint8))
    s.temp, s.minp, s.active = _dev(temp), _dev(minp), _dev(_active(R))
    s.accept_u = torch.rand((R, K), generator=gen, device=DEV)
    s.draw_u = torch.rand(R, generator=gen, device=DEV)
    s.token_out = torch.zeros((R, K + 1), dtype=torch.int32, device=DEV)
    s.accepted = torch.zeros(R, dtype=torch.int32, device=DEV)
    s.prob = torch.zeros((R, K), dtype=torch.float32, device=DEV)
    s.work = torch.zeros(64 + 4 * R * (K + 3), dtype=torch.uint8, device=DEV)


def _prepare_w4(s, c, seed):
    M, K, N, G, gen = c["rows"], c["k"], c["n"], c["group"], _gen(seed, 2)
    s.x = torch.randn((M, K), generator=gen, device=DEV).to(torch.bfloat16)
    s.weights = torch.randint(0, 256, (N, (K + 1) // 2), generator=gen, device=DEV, dtype=torch.uint8)
    groups = -(-K // G)
    s.scales = (0.002 * torch.rand((N, groups), generator=gen, device=DEV) + 0.001).to(_kind(c["scales"]))
    s.zeros = torch.randint(0, 16, (N, groups), generator=gen, device=DEV, dtype=torch.uint8) if c["zeros"] else None
    s.y = torch.zeros((M, N), dtype=_kind(c["out"]), device=DEV)


def _pool_pages(c):
    """Pages of a case's pool: every row's own, and room for each to grow or to be copied."""
    per = _pages(_lengths(c)) + _pages(np.full(c["rows"], c["new"])) + 1
    return int(per.sum()) + 5


def _prepare_cache(s, c, seed):
    R, L, gen = c["rows"], c["layers"], _gen(seed, 3)
    pages, lens, new = _pool_pages(c), _lengths(c), _news(c)
    cols = int(_pages(lens.max() + c["new"])) + 1
    if c["kind"] == "fork":
        lens[_families(c)[1]] = 0  # (the children's rows are empty)
    if c["kind"] == "compact":
        lens[np.arange(R) % 8 != 0] //= 8  # (most rows have ended or were rolled back)
    counts = _pages(lens)
    order = np.random.default_rng([int(seed) & 0x7FFFFFFF, 4]).permutation(pages).astype(np.int32)
    room = (R * cols + 3) // 4 * 4  # (the counts start on 16 bytes)
    meta = np.zeros(room + pages, np.int32)
    table, refs = meta[:R * cols].reshape(R, cols), meta[room:]
    table[:] = -1
    at = 0
    for r in range(R):
        table[r, :counts[r]] = order[at:at + counts[r]]
        at += counts[r]
    refs[order[:at]] = 1
    s.meta = _dev(meta)
    s.table, s.refs = s.meta[:R * cols].view(R, cols), s.meta[room:]
    s.length, s.new = _dev(lens), _dev(new)
    shape = (L, pages, c["kv_heads"], PAGE, c["dim"])
    s.k = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.v = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.ok = torch.zeros(R, dtype=torch.uint8, device=DEV)
    s.work = torch.zeros(1024 + 4 * (4 * pages + 4 * R), dtype=torch.uint8, device=DEV)
    if c["kind"] == "extend":
        s.active = _dev(_active(R))
        new_shape = (R, c["new"], c["kv_heads"], c["dim"])
        s.k_new = torch.randn(new_shape, generator=gen, device=DEV, dtype=torch.bfloat16)
        s.v_new = torch.randn(new_shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    elif c["kind"] == "fork":
        parent, child = _families(c)
        s.parent, s.child = _dev(parent), _dev(child)
        is_child = np.zeros(R, np.uint8)
        is_child[child] = 1
        s.active = _dev(is_child)
        s.keep = s.length.clone()
    else:
        s.before = s.meta.clone()
        s.live = torch.zeros(1, dtype=torch.int32, device=DEV)


def prepare(c, seed):
    s = State()
    s.kind, s.c = c["kind"], c
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    if s.kind == "verify":
        _prepare_verify(s, c, seed)
    elif s.kind == "w4":
        _prepare_w4(s, c, seed)
    else:
        _prepare_cache(s, c, seed)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_side(l, temp, theta):
    """Weights exp2((l - max) log2(e) / T) of the kept logits, their sum in multiples of 2^-31, and probabilities."""
    top = l.amax(-1, keepdim=True)
    kexp = (torch.full_like(temp, LOG2E) / temp).view(-1, *([1] * (l.dim() - 1)))
    cut = top + theta.view(-1, *([1] * (l.dim() - 1)))
    w = torch.where(l >= cut, torch.exp2((l - top) * kexp), 0.0)
    whole = (w * ONE).round().to(torch.int64)
    total = whole.sum(-1, keepdim=True)
    return top, whole, w * (1.0 / (total.float() / ONE))


def _plain_verify(s):
    c = s.c
    R, K, V = c["rows"], c["draft"], c["vocab"]
    t = s.target[:, :, :V].float()
    at = torch.arange(V, device=DEV)
    greedy = (s.probe != 0) | (s.temp == 0)
    temp = torch.where(greedy, 1.0, s.temp)
    theta = (temp.double() * torch.log(s.minp.double())).float()
    top, whole, p = _plain_side(t, temp, theta)
    best = torch.where(t == top, at, V).amin(-1)  # the lowest index of the largest logit
    d = s.tokens.long()
    pd = p[:, :K].gather(-1, d[..., None])[..., 0]
    if s.draft is not None:
        q = _plain_side(s.draft[:, :, :V].float(), temp, theta)[2]
        qd = q.gather(-1, d[..., None])[..., 0]
    else:
        q, qd = None, torch.ones_like(pd)
    live = (torch.arange(K, device=DEV) < s.count[:, None]) & (s.active[:, None] != 0)
    same = best[:, :K] == d
    take = torch.where(greedy[:, None], same, s.accept_u * qd < pd)
    prob = torch.where(qd > 0, (pd / qd).clamp(max=1.0), (pd > 0).float())
    prob = torch.where(live, torch.where(greedy[:, None], same.float(), prob), 0.0)
    n = (take & live).long().cumprod(-1).sum(-1)  # accepted tokens
    row = torch.arange(R, device=DEV)
    mine, total = p[row, n], whole[row, n]
    k = n.clamp(max=K - 1)
    gone = (at == d[row, k][:, None]).float() if q is None else q[row, k]
    rest = ((mine - gone).clamp(min=0.0) * ONE).round().to(torch.int64)
    use = (n < s.count)[:, None] & (rest.sum(-1, keepdim=True) > 0)
    mass = torch.where(use, rest, total).cumsum(-1)
    mark = (s.draw_u.double() * mass[:, -1].double()).to(torch.int64)
    token = torch.where(greedy, best[row, n], (mass <= mark[:, None]).sum(-1))
    on = s.active != 0
    place = torch.arange(K + 1, device=DEV)
    out = torch.cat([d, torch.full((R, 1), -1, device=DEV)], 1)
    out = torch.where(place < n[:, None], out, torch.where(place == n[:, None], token[:, None], -1))
    return torch.where(on[:, None], out, -1).int(), torch.where(on, n, 0).int(), prob


def _plain_w4(s):
    K, G = s.c["k"], s.c["group"]
    q = torch.stack((s.weights & 15, s.weights >> 4), -1).view(s.weights.shape[0], -1)[:, :K].float()
    wide = torch.arange(K, device=DEV) // G
    q = q - (8.0 if s.zeros is None else s.zeros.float()[:, wide])
    return (s.x.float() @ (q * s.scales.float()[:, wide]).T).to(s.y.dtype)


def _first(on):
    """Indices 0, 1, ... of `on`, those where it is false replaced by one where it is true: writing with them writes the
    same values again."""
    i = torch.arange(on.numel(), device=DEV)
    return torch.where(on, i, on.int().argmax())


def _plain_reserve(s):
    R, P = s.table.shape
    n = torch.where(s.active != 0, s.new, 0)[:, None]
    length, col = s.length[:, None], torch.arange(P, device=DEV)
    first, last = length // PAGE, (length + n + PAGE - 1) // PAGE
    within = (n > 0) & (col >= first) & (col < last)
    held = s.table.clamp(min=0).long()
    shared = within & (col == first) & (length % PAGE > 0) & (s.table >= 0) & (s.refs[held] > 1)
    need = within & ((s.table < 0) | shared)
    order = need.flatten().cumsum(0).view(R, P)
    ok = order[:, -1] <= (s.refs == 0).sum()
    take = need & ok[:, None]
    free = torch.argsort((s.refs > 0).to(torch.uint8), stable=True)  # the free pages first, in order
    fresh = free[(order - 1).clamp(0, free.numel() - 1)]
    copy = take & shared
    row = _first(copy.any(-1))
    at = first[row, 0].clamp(max=P - 1).long()
    src, dst = held[row, at], fresh[row, at]
    slot = torch.arange(PAGE, device=DEV)[None, :] < (length[row] % PAGE)
    slot = (slot & copy.any())[None, :, None, :, None]
    dst = torch.where(copy.any(), dst, src)
    for pool in (s.k, s.v):
        pool[:, dst] = torch.where(slot, pool[:, src], pool[:, dst])
    s.refs.scatter_add_(0, held.flatten(), -copy.flatten().int())
    s.refs.scatter_add_(0, fresh.flatten(), take.flatten().int())
    s.table.copy_(torch.where(take, fresh.int(), s.table))
    s.ok.copy_((s.active != 0) & ok)


def _plain_write(s):
    R, T = s.k_new.shape[:2]
    i = torch.arange(T, device=DEV)
    pos = s.length[:, None].long() + i
    page = s.table.long().gather(1, (pos // PAGE).clamp(max=s.table.shape[1] - 1))
    on = (i < s.new[:, None]) & (s.ok[:, None] != 0) & (page >= 0)
    at = _first(on.flatten())
    page, slot = page.flatten()[at].clamp(min=0), (pos % PAGE).flatten()[at]
    any_on = on.any()
    for pool, new in ((s.k, s.k_new), (s.v, s.v_new)):
        new = new.reshape(R * T, *new.shape[2:])[at]
        pool[0][page, :, slot] = torch.where(any_on, new, pool[0][page, :, slot])


def _plain_trim(s, length):
    past = (torch.arange(s.table.shape[1], device=DEV) >= _pages(length)[:, None]) & (s.table >= 0) & (s.active != 0)[:, None]
    s.refs.scatter_add_(0, s.table.clamp(min=0).flatten().long(), -past.flatten().int())
    s.table.copy_(torch.where(past, -1, s.table))


def _plain_fork(s):
    rows = s.table[s.parent.long()]
    s.table[s.child.long()] = rows
    s.length[s.child.long()] = s.length[s.parent.long()]
    s.refs.scatter_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().int())


def _plain_compact(s):
    used, at = s.refs > 0, torch.arange(s.refs.numel(), device=DEV)
    live = used.sum()
    src, dst = (used & (at >= live)).nonzero()[:, 0], (~used & (at < live)).nonzero()[:, 0]
    for pool in (s.k, s.v):
        pool[:, dst] = pool[:, src]
    place = at.int()
    place[src] = dst.int()
    s.table.copy_(torch.where(s.table >= 0, place[s.table.clamp(min=0).long()], -1))
    s.refs[dst] = s.refs[src]
    s.refs[src] = 0
    s.live.copy_(live.view(1))


def _plain(s):
    if s.kind == "verify":
        return _plain_verify(s)
    if s.kind == "w4":
        return _plain_w4(s)
    if s.kind == "extend":
        _plain_trim(s, s.length)
        _plain_reserve(s)
        _plain_write(s)
        return s.table, s.refs, s.ok, s.k, s.v
    if s.kind == "fork":
        _plain_trim(s, s.keep)
        _plain_fork(s)
        _plain_reserve(s)
        return s.table, s.length, s.refs, s.ok, s.k, s.v
    s.meta.copy_(s.before)  # (the pool as it was, so that every pass has the same pages to move)
    _plain_compact(s)
    return s.table, s.refs, s.live, s.k, s.v


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _shape(s):
    from paper_2607_20791_gb300 import binding
    c = s.c
    return binding.CacheShape(num_layers=c["layers"], num_pages=s.refs.numel(), num_kv_heads=c["kv_heads"],
                              page_size=PAGE, head_dim=c["dim"])


def _run_own(s):
    from paper_2607_20791_gb300 import binding
    c = s.c
    if s.kind == "verify":
        binding.rgd_verify_draft(s.target, s.draft, s.tokens, s.count, s.probe, s.temp, s.minp, s.accept_u, s.draw_u,
                                 s.active, s.token_out, s.accepted, s.prob, s.work, vocab=c["vocab"],
                                 dev_status=s.status)
        return s.token_out, s.accepted, s.prob
    if s.kind == "w4":
        binding.rgd_w4_matvec(s.x, s.weights, s.scales, s.zeros, c["group"], s.y)
        return s.y
    shape = _shape(s)
    if s.kind == "compact":
        s.meta.copy_(s.before)
        binding.rgd_cache_compact(shape, s.table, None, s.refs, s.k, s.v, s.live, s.work, dev_status=s.status)
        return s.table, s.refs, s.live, s.k, s.v
    binding.rgd_cache_trim(s.table, s.length if s.kind == "extend" else s.keep, s.active, s.refs, dev_status=s.status)
    if s.kind == "fork":
        binding.rgd_cache_fork(s.parent, s.child, s.table, s.length, s.refs, dev_status=s.status)
    binding.rgd_cache_reserve(shape, s.table, s.length, s.new, s.active, s.refs, s.k, s.v, s.ok, s.work,
                              dev_status=s.status)
    if s.kind == "fork":
        return s.table, s.length, s.refs, s.ok, s.k, s.v
    binding.rgd_cache_write(shape, 0, s.k_new, s.v_new, s.new, s.table, s.length, s.ok, s.k, s.v, dev_status=s.status)
    return s.table, s.refs, s.ok, s.k, s.v


def run(s):
    return _run_own(s) if own else _plain(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    if c["kind"] == "verify":
        on, greedy, n, size = _active(c["rows"]) != 0, _greedy(c), _n_draft(c), 4 if c["dtype"] == "f32" else 2
        rows = np.where(on, n + 1, 0) + (np.where(on & ~greedy, n, 0) if not c["point"] else 0)
        logits = float(rows.sum()) * c["vocab"]
        return {"bytes": logits * size + c["rows"] * (c["draft"] * 12 + 40.0), "flops": 4 * logits}
    if c["kind"] == "w4":
        M, K, N, groups = c["rows"], c["k"], c["n"], -(-c["k"] // c["group"])
        per = (4 if c["scales"] == "f32" else 2) + (1 if c["zeros"] else 0)
        return {"bytes": N * ((K + 1) // 2) + float(N) * groups * per + 2.0 * M * K + M * N * (4 if c["out"] == "f32" else 2),
                "flops": 2.0 * M * N * K}
    token = 2.0 * 2 * c["kv_heads"] * c["dim"]  # bytes of a token's keys and values in one layer
    R, pages, lens, new = c["rows"], _pool_pages(c), _lengths(c), _news(c)
    table = 4.0 * R * (int(_pages(lens.max() + c["new"])) + 1)
    if c["kind"] == "extend":
        return {"bytes": 2 * token * float((new * (_active(R) != 0)).sum()) + 2 * (table + 4 * pages), "flops": 0}
    if c["kind"] == "fork":
        parent, child = _families(c)
        return {"bytes": 2 * token * c["layers"] * float(((lens[parent] % PAGE) * (new[child] > 0)).sum()) + 2 * (table + 4 * pages),
                "flops": 0}
    lens[np.arange(R) % 8 != 0] //= 8
    live = int(_pages(lens).sum())
    moved = live * (pages - live) / pages  # on average over orders
    return {"bytes": 2 * token * PAGE * c["layers"] * moved + 2 * (table + 4 * pages), "flops": 0}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_probability(l, temp, cut):
    kept = (l >= cut).double()
    e = kept * torch.exp((l.double() - l.double().max()) / temp)
    return e / e.sum()


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "w4":
        K, N, out = c["k"], c["n"], []
        x = s.x.double()
        for a in range(0, N, 8192):
            b = s.weights[a:a + 8192].to(torch.int64)
            q = torch.zeros((b.shape[0], 2 * b.shape[1]), dtype=torch.float64, device=DEV)
            q[:, 0::2], q[:, 1::2] = (b % 16).double(), (b // 16).double()
            y = torch.zeros((x.shape[0], b.shape[0]), dtype=torch.float64, device=DEV)
            for g in range(s.scales.shape[1]):
                lo, hi = g * c["group"], min(K, (g + 1) * c["group"])
                zero = s.zeros[a:a + 8192, g].double() if c["zeros"] else 8.0 * torch.ones(b.shape[0], dtype=torch.float64, device=DEV)
                part = x[:, lo:hi] @ q[:, lo:hi].T - x[:, lo:hi].sum(1, keepdim=True) * zero
                y += part * s.scales[a:a + 8192, g].double()
            out.append(y)
        return torch.cat(out, 1)
    if c["kind"] != "verify" or c["rows"] * c["draft"] > 3000:
        return None
    prob = torch.zeros((c["rows"], c["draft"]), dtype=torch.float64, device=DEV)
    temp, minp = _sampling(c)
    on, greedy, n, V = _active(c["rows"]), _greedy(c), _n_draft(c), c["vocab"]
    for r in range(c["rows"]):
        if not on[r]:
            continue
        low = np.float32(float(temp[r]) * math.log(minp[r])) if minp[r] > 0 and not greedy[r] else np.float32(-np.inf)
        for k in range(n[r]):
            l, d = s.target[r, k, :V].float(), s.tokens[r, k].long()
            top = l.max()
            if greedy[r]:
                prob[r, k] = ((l == top).to(torch.uint8).argmax() == d).double()
                continue
            pd = _exact_probability(l, float(temp[r]), top + float(low))[d]
            qd = torch.ones_like(pd)
            if s.draft is not None:
                q = s.draft[r, k, :V].float()
                qd = _exact_probability(q, float(temp[r]), q.max() + float(low))[d]
            prob[r, k] = torch.where(qd > 0, (pd / qd).clamp(max=1.0), (pd > 0).double())
    return None, None, prob
