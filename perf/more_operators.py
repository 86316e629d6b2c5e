"""Measured cases of the dense operators of a step: what stands between the hidden states and the
attention, and the sampling with more filters than min-p.

Every case is a dict of plain values whose ``kind`` names the operator:

* ``rope``      ``rgd_qk_rope``: norms of queries and keys for each head and their rotation by position.
* ``rope_cache``  ``rgd_qk_rope_cache``: the same for a step's new tokens, the keys and values straight
                  into the pages of the cache.
* ``quantize``  ``rgd_fp8_quantize``: activations (or weights) in 8-bit floating point with a scale
                for every 128 columns.
* ``matmul``    ``rgd_fp8_matmul``: products of such activations and weights.
* ``sample``    ``rgd_sample_top``: temperature, top-k, top-p and min-p from given uniforms.

Inputs are drawn on the GPU from the seed; lengths and counts go by the row's index, so that a
case's work is a function of the case alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
BLOCK = 128  # columns (and rows of weights) that share a scale
DEV = "cuda"
LOG2E = 1.4426950408889634
ONE = 2.0 ** 31  # weights of tokens are summed as whole multiples of 2^-31


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _rope(tokens, heads, kv_heads, dim, rot, layout, norm, scaling, dtype, far):
    """q and k as views of a fused projection; positions up to `far`."""
    return {"kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
            "layout": layout, "norm": norm, "scaling": scaling, "dtype": dtype, "far": far}


def _rope_cache(rows, new, heads, kv_heads, dim, rot, layout, norm, scaling, length, far):
    """rows of up to `length` cached tokens get up to `new` each; prompts of up to `far` tokens lie before them."""
    return {"kind": "rope_cache", "rows": rows, "new": new, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot,
            "layout": layout, "norm": norm, "scaling": scaling, "length": length, "far": far}


def _quantize(rows, cols, dtype, block_rows):
    return {"kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "block_rows": block_rows}


def _matmul(m, n, k, out):
    return {"kind": "matmul", "m": m, "n": n, "k": k, "out": out}


def _sample(rows, rpg, vocab, dtype, filters, pad=0):
    """rows of logits, the first of every rpg a greedy probe."""
    return {"kind": "sample", "rows": rows, "rpg": rpg, "vocab": vocab, "dtype": dtype, "filters": filters, "pad": pad}


def listed():
    return [
        # one prompt's rows of a small model: latency
        {"name": "rope_tiny", **_rope(3, 4, 1, 64, 64, "half", False, "none", "bf16", 300)},
        # the queries and keys of long prompts, normed, positions far past the trained length
        {"name": "rope_prompt", **_rope(16384, 32, 8, 128, 128, "half", True, "bands", "bf16", 500000)},
        # the ordinary serving batch: 16 prompts, 1 probe and 4 samples each, one token a row
        {"name": "cache_step", **_rope_cache(80, 1, 32, 8, 128, 128, "half", True, "bands", 300, 2048)},
        # the largest batch: 2048 rows of 8 drafted tokens, half of each head rotated, pairs side by side
        {"name": "cache_batch", **_rope_cache(2048, 8, 32, 8, 128, 64, "pairs", False, "ramp", 150, 60000)},
        # the ordinary batch's activations
        {"name": "quantize_step", **_quantize(80, 4096, "bf16", 1)},
        # a long prompt's, over the wide side of a feed-forward layer
        {"name": "quantize_prompt", **_quantize(16384, 14336, "bf16", 1)},
        # the ordinary batch through a fused projection to queries, keys and values
        {"name": "matmul_step", **_matmul(80, 6144, 4096, "bf16")},
        # ragged sizes: the last blocks of rows, columns and k are short
        {"name": "matmul_odd", **_matmul(333, 2500, 1000, "f32")},
        # a long prompt through the wide side of a feed-forward layer
        {"name": "matmul_prompt", **_matmul(8192, 14336, 4096, "bf16")},
        # one prompt's rows over an odd vocabulary, top-p alone: every token has a weight
        {"name": "sample_odd", **_sample(5, 5, 32001, "f32", "top_p")},
        # the ordinary serving batch, all filters
        {"name": "sample_8b", **_sample(80, 5, 128256, "bf16", "usual")},
        # the largest batch, filters that differ from row to row
        {"name": "sample_batch", **_sample(512, 2, 152064, "bf16", "sweep")},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


SCALINGS = ("none", "linear", "base", "bands", "ramp")


def draw(rng):
    kind = rng.choice(("rope", "rope_cache", "quantize", "matmul", "matmul", "sample", "sample"))
    if kind in ("rope", "rope_cache"):
        dim, rot = rng.choice(((64, 64), (128, 128), (128, 64), (80, 20), (96, 48), (256, 64), (72, 72), (128, 32)))
        kv = rng.choice((1, 2, 4, 8))
        heads = kv * rng.choice((1, 2, 4, 7))
        how = (heads, kv, dim, rot, rng.choice(("half", "pairs")), rng.random() < 0.6, rng.choice(SCALINGS))
        if kind == "rope":
            most = (80 << 20) // ((heads + 2 * kv) * dim)
            return _rope(_log(rng, 1, min(16384, most)), *how, rng.choice(("bf16", "bf16", "f32")), _log(rng, 100, 1000000))
        new, length = rng.randint(1, 8), _log(rng, 4, 1000)
        most = min((80 << 20) // ((heads + 2 * kv) * dim * new), (1 << 29) // ((length + 32) * kv * dim))
        return _rope_cache(_log(rng, 1, max(1, min(2048, most))), new, *how, length, _log(rng, 16, 100000))
    if kind == "quantize":
        cols = _log(rng, 16, 16384)
        if rng.random() < 0.6:
            cols = (cols + 127) // 128 * 128
        return _quantize(_log(rng, 1, min(16384, (200 << 20) // cols)), cols, rng.choice(("bf16", "f32")), rng.choice((1, 1, 128)))
    if kind == "matmul":
        n, k = _log(rng, 16, 32768), _log(rng, 64, 16384)
        if rng.random() < 0.6:
            n, k = (n + 127) // 128 * 128, (k + 127) // 128 * 128
        most = min((64 << 20) // n, (128 << 20) // k, (400 << 30) // (n * k))
        return _matmul(_log(rng, 1, max(1, min(8192, most))), n, k, rng.choice(("bf16", "f32")))
    dtype, vocab = rng.choice(("f32", "bf16")), _log(rng, 500, 262144)
    if rng.random() < 0.6:
        vocab = (vocab + 7) // 8 * 8
    pad = rng.choice((0, 0, 8, 64)) if vocab % 8 == 0 else rng.choice((0, 3))
    most = (70 << 20) // vocab
    return _sample(_log(rng, 1, max(1, min(512, most))), rng.randint(1, 6), vocab, dtype,
                   rng.choice(("usual", "sweep", "top_p", "top_k")), pad)


# ---------------------------------------------------------------------------
# sizes that go by the row's index
# ---------------------------------------------------------------------------
def _active(rows):
    i = np.arange(rows)
    return ((i % 11 != 7) | (rows < 8)).astype(np.uint8)


def _lengths(c):
    """Cached tokens of each row, from 0 to c["length"], the last row the longest."""
    n = (np.arange(c["rows"]) * 7919 + 13) % (c["length"] + 1)
    n[-1] = c["length"]
    return n.astype(np.int32)


def _news(c):
    """New tokens of each row: most rows all of them, some fewer, some none."""
    i = np.arange(c["rows"])
    return np.where(i % 5 == 4, i % (c["new"] + 1), c["new"]).astype(np.int32)


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _filters(c):
    """Temperature, top-k (0: all), top-p and min-p of each row."""
    i = np.arange(c["rows"])
    t = np.array([1.0, 1.5, 2.0, 0.7])[i % 4]
    k, p, m = np.zeros(c["rows"], int), np.ones(c["rows"]), np.zeros(c["rows"])
    if c["filters"] == "usual":
        k, p, m = np.array([50, 20, 100])[i % 3], np.array([0.9, 0.95])[i % 2], np.array([0.0, 0.02, 0.05])[i % 3]
    elif c["filters"] == "top_p":
        p = np.array([0.9, 0.5, 0.99])[i % 3]
    elif c["filters"] == "top_k":
        k = np.array([1, 40, 1000, 5])[i % 4]
    else:
        t = np.array([0.0, 0.3, 1.0, 2.0, 5.0])[i % 5]
        k, p = np.array([0, 64, 2000, 0])[i % 4], np.array([1.0, 0.8, 0.95])[i % 3]
        m = np.array([0.0, 0.0, 0.1])[(i // 3) % 3]
    t = np.where(i % c["rpg"] == 0, 0.0, t)
    return t.astype(np.float32), k.astype(np.int32), p.astype(np.float32), m.astype(np.float32)


def _frequencies(c):
    """Angle per position of each pair in radians (64 bits), and the factor on the rotated part."""
    rot, kind = c["rot"], c["scaling"]
    factor, trained, base = 8.0, 8192.0, 500000.0 if c["far"] > 100000 else 10000.0
    i = np.arange(rot // 2, dtype=np.float64)
    if kind == "base":
        base *= factor ** (rot / max(rot - 2, 1))
    f = base ** (-2.0 * i / rot)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "bands":  # long waves slowed down, short ones kept, those between blended
        turns = trained * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * (keep + (1 - keep) / factor), 1.0
    if kind == "ramp":  # the same over the pair's index
        at = [rot * math.log(trained / (b * 2 * math.pi)) / (2 * math.log(base)) for b in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * (keep + (1 - keep) / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


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


def _prepare_rotation(s, c, gen):
    """What a model keeps: the norms' weights and the rotation's frequencies."""
    kind = _kind(c.get("dtype", "bf16"))
    f, s.magnitude = _frequencies(c)
    s.freq = _dev(f)
    s.wq = s.wk = None
    if c["norm"]:
        s.wq, s.wk = ((1 + 0.2 * torch.randn(c["dim"], generator=gen, device=DEV)).to(kind) for _ in range(2))
    if own:
        from paper_2607_20791_gb300 import binding
        base = 500000.0 if c["far"] > 100000 else 10000.0
        turns, magnitude = binding.rgd_rope_frequencies(c["rot"], base, c["scaling"], factor=8.0, trained_length=8192.0)
        s.turns = turns.to(DEV)
        s.shape = binding.RopeShape(num_q_heads=c["heads"], num_k_heads=c["kv_heads"], head_dim=c["dim"],
                                    rotary_dim=c["rot"], layout=binding.RGD_ROPE_HALF if c["layout"] == "half" else binding.RGD_ROPE_PAIRS,
                                    norm=int(c["norm"]), eps=1e-6, magnitude=magnitude)


def _fused(s, c, lead, gen):
    """q, k and v as views of one projection's output."""
    h, kv, d = c["heads"], c["kv_heads"], c["dim"]
    s.qkv = (1.5 * torch.randn((*lead, h + 2 * kv, d), generator=gen, device=DEV)).to(_kind(c.get("dtype", "bf16")))
    s.q, s.k, s.v = s.qkv[..., :h, :], s.qkv[..., h:h + kv, :], s.qkv[..., h + kv:, :]


def _prepare_rope(s, c, seed):
    gen, n = _gen(seed, 1), c["tokens"]
    _prepare_rotation(s, c, gen)
    _fused(s, c, (n,), gen)
    s.positions = _dev(((np.arange(n, dtype=np.int64) * 104729 + 17) % (c["far"] + 1)).astype(np.int32))
    s.q_out = torch.zeros((n, c["heads"], c["dim"]), dtype=s.q.dtype, device=DEV)
    s.k_out = torch.zeros((n, c["kv_heads"], c["dim"]), dtype=s.q.dtype, device=DEV)


def _prepare_rope_cache(s, c, seed):
    gen, R = _gen(seed, 2), c["rows"]
    _prepare_rotation(s, c, gen)
    _fused(s, c, (R, c["new"]), gen)
    lens, new = _lengths(c), _news(c)
    counts = _pages(lens + new)
    pages, cols = int(counts.sum()) + 3, int(counts.max()) + 1
    order = np.random.default_rng([int(seed) & 0x7FFFFFFF, 4]).permutation(pages).astype(np.int32)
    table, at = np.full((R, cols), -1, np.int32), 0
    for r in range(R):
        table[r, :counts[r]] = order[at:at + counts[r]]
        at += counts[r]
    s.table, s.length, s.new, s.active = _dev(table), _dev(lens), _dev(new), _dev(_active(R))
    s.first = _dev(((np.arange(R) * 7907 + 5) % (c["far"] + 1)).astype(np.int32))
    shape = (1, pages, c["kv_heads"], PAGE, c["dim"])
    s.k_pages = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.v_pages = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    s.q_out = torch.zeros((R, c["new"], c["heads"], c["dim"]), dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2607_20791_gb300 import binding
        s.cache = binding.CacheShape(num_layers=1, num_pages=pages, num_kv_heads=c["kv_heads"], page_size=PAGE,
                                     head_dim=c["dim"])


def _stride(k):
    """Rows of 8-bit values start on 16 bytes."""
    return (k + 15) // 16 * 16


def _activations(rows, cols, gen):
    """Values whose size differs from column to column and from row to row, a few columns much larger."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    x *= torch.exp(0.7 * torch.randn(cols, generator=gen, device=DEV))
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=DEV))
    x[:, torch.rand(cols, generator=gen, device=DEV) < 0.003] *= 20
    return x


def _prepare_quantize(s, c, seed):
    rows, cols, gen = c["rows"], c["cols"], _gen(seed, 3)
    s.x = _activations(rows, cols, gen).to(_kind(c["dtype"]))
    s.out = torch.zeros((rows, _stride(cols)), dtype=torch.float8_e4m3fn, device=DEV)
    s.scales = torch.zeros((-(-rows // c["block_rows"]), -(-cols // BLOCK)), device=DEV)


def _blocks(x, rows):
    """x padded to whole blocks, as [block of rows, rows, block of columns, BLOCK]."""
    r, n = x.shape
    a, b = -(-r // rows), -(-n // BLOCK)
    full = torch.zeros((a * rows, b * BLOCK), dtype=x.dtype, device=DEV)
    full[:r, :n] = x
    return full.view(a, rows, b, BLOCK)


def _to_8_bits(x, rows):
    """e4m3 values and the scales of blocks of `rows` x BLOCK: the largest of a block becomes 448."""
    r, n = x.shape
    x = _blocks(x.float(), rows)
    most = x.abs().amax((1, 3))
    up = torch.where(most > 0, 448.0 / most, 0.0)
    q = (x * up[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(x.shape[0] * rows, -1)[:r, :n], most / 448.0


def _prepare_matmul(s, c, seed):
    m, n, k, gen = c["m"], c["n"], c["k"], _gen(seed, 5)
    s.x = torch.zeros((m, _stride(k)), dtype=torch.float8_e4m3fn, device=DEV)
    s.w = torch.zeros((n, _stride(k)), dtype=torch.float8_e4m3fn, device=DEV)
    s.x[:, :k], s.sx = _to_8_bits(_activations(m, k, gen), 1)
    s.w[:, :k], s.sw = _to_8_bits(torch.randn((n, k), generator=gen, device=DEV) / math.sqrt(k), BLOCK)
    s.y = torch.zeros((m, n), dtype=_kind(c["out"]), device=DEV)


def _prepare_sample(s, c, seed):
    R, V, gen = c["rows"], c["vocab"], _gen(seed, 6)
    base = -1.1 * torch.log(torch.arange(1, V + 1, dtype=torch.float64))
    base = (base - torch.logsumexp(base, 0)).float().to(DEV)
    s.logits = torch.zeros((R, V + c["pad"]), dtype=_kind(c["dtype"]), device=DEV)
    for r in range(R):  # a Zipf-ranked row, with some noise
        s.logits[r, :V] = base[torch.randperm(V, generator=gen, device=DEV)] + torch.randn(V, generator=gen, device=DEV)
    temp, top_k, top_p, min_p = _filters(c)
    s.temp, s.top_k, s.top_p, s.min_p = _dev(temp), _dev(top_k), _dev(top_p), _dev(min_p)
    s.probe, s.active = _dev((np.arange(R) % c["rpg"] == 0).astype(np.uint8)), _dev(_active(R))
    s.u = torch.rand(R, generator=gen, device=DEV)
    s.token = torch.zeros(R, dtype=torch.int32, device=DEV)
    s.kept = torch.zeros(R, dtype=torch.int32, device=DEV)
    s.prob = torch.zeros(R, device=DEV)


def prepare(c, seed):
    s = State()
    s.kind, s.c = c["kind"], c
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    {"rope": _prepare_rope, "rope_cache": _prepare_rope_cache, "quantize": _prepare_quantize, "matmul": _prepare_matmul,
     "sample": _prepare_sample}[s.kind](s, c, seed)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_turn(s, x, weight, positions):
    """x [..., heads, D] normed (where the case norms) and rotated by its positions [...]."""
    c, y = s.c, x.float()
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    angle = positions.double()[..., None, None] * s.freq  # (64 bits: far positions)
    cos, sin = (torch.cos(angle) * s.magnitude).float(), (torch.sin(angle) * s.magnitude).float()
    rot, half = c["rot"], c["rot"] // 2
    out = y.clone()
    if c["layout"] == "half":
        a, b = y[..., :half], y[..., half:rot]
        out[..., :half], out[..., half:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _places(s):
    """Which new tokens are written, and the page and the slot of each (those that are not: of one that is)."""
    R, T = s.q.shape[:2]
    i = torch.arange(T, device=DEV)
    pos = s.length[:, None].long() + i
    page = s.table.long().gather(1, (pos // PAGE).clamp(max=s.table.shape[1] - 1))
    on = (i < s.new[:, None]) & (s.active[:, None] != 0)
    flat = on.flatten()
    at = torch.where(flat, torch.arange(R * T, device=DEV), flat.int().argmax())
    return on, pos, at, page.flatten()[at].clamp(min=0), (pos % PAGE).flatten()[at]


def _plain_rope_cache(s):
    R, T = s.q.shape[:2]
    on, pos, at, page, slot = _places(s)
    pos = pos + s.first[:, None]
    q, k = _plain_turn(s, s.q, s.wq, pos), _plain_turn(s, s.k, s.wk, pos)
    s.q_out.copy_(torch.where(on[..., None, None], q, s.q_out))
    for pool, new in ((s.k_pages, k), (s.v_pages, s.v)):
        pool[0][page, :, slot] = torch.where(on.any(), new.reshape(R * T, *new.shape[2:])[at], pool[0][page, :, slot])
    return s.q_out, s.k_pages, s.v_pages


def _plain_matmul(s):
    k, n = s.c["k"], s.c["n"]
    by = torch.arange(k, device=DEV) // BLOCK
    x = s.x[:, :k].float() * s.sx[:, by]
    w = s.w[:, :k].float() * s.sw[(torch.arange(n, device=DEV) // BLOCK)[:, None], by]
    return (x @ w.T).to(s.y.dtype)


def _plain_sample(s):
    V = s.c["vocab"]
    l = s.logits[:, :V].float()
    greedy = (s.probe != 0) | (s.temp == 0)
    temp = torch.where(greedy, 1.0, s.temp)
    value, token = torch.sort(l, dim=-1, descending=True, stable=True)  # (equal logits: the lower index first)
    top = value[:, :1]
    cut = top + (temp.double() * torch.log(s.min_p.double())).float()[:, None]
    place = torch.arange(V, device=DEV)
    keep = (value >= cut) & ((s.top_k <= 0)[:, None] | (place < s.top_k[:, None]))
    w = torch.exp2((value - top) * (torch.full_like(temp, LOG2E) / temp)[:, None])
    whole = torch.where(keep, (w * ONE).round().to(torch.int64), 0)
    upto = whole.cumsum(-1)
    need = torch.ceil(s.top_p.double() * upto[:, -1].double()).to(torch.int64)
    keep &= (upto - whole < need[:, None]) | (s.top_p >= 1)[:, None]
    keep = torch.where(greedy[:, None], place == 0, keep)
    whole = torch.where(keep, whole, 0)
    mass = torch.zeros_like(whole).scatter(1, token, whole).cumsum(-1)
    total = mass[:, -1]
    mark = (s.u.double() * total.double()).to(torch.int64)
    picked = torch.where(greedy, token[:, 0], (mass <= mark[:, None]).sum(-1))
    mine = torch.where(token == picked[:, None], whole, 0).sum(-1)
    on = s.active != 0
    return (torch.where(on, picked, -1).int(), torch.where(on, keep.sum(-1), 0).int(),
            torch.where(on, torch.where(greedy, 1.0, mine.float() / total.float()), 0.0))


def _plain(s):
    if s.kind == "rope":
        return _plain_turn(s, s.q, s.wq, s.positions), _plain_turn(s, s.k, s.wk, s.positions)
    if s.kind == "rope_cache":
        return _plain_rope_cache(s)
    if s.kind == "quantize":
        s.out[:, :s.c["cols"]], s.scales = _to_8_bits(s.x, s.c["block_rows"])
        return s.out, s.scales
    if s.kind == "matmul":
        return _plain_matmul(s)
    return _plain_sample(s)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _run_own(s):
    from paper_2607_20791_gb300 import binding
    c = s.c
    if s.kind == "rope":
        binding.rgd_qk_rope(s.shape, s.q, s.k, s.positions, s.turns, s.wq, s.wk, s.q_out, s.k_out, dev_status=s.status)
        return s.q_out, s.k_out
    if s.kind == "rope_cache":
        binding.rgd_qk_rope_cache(s.shape, s.cache, 0, s.q, s.k, s.v, s.first, s.turns, s.wq, s.wk, s.new, s.table,
                                  s.length, s.active, s.q_out, s.k_pages, s.v_pages, dev_status=s.status)
        return s.q_out, s.k_pages, s.v_pages
    if s.kind == "quantize":
        binding.rgd_fp8_quantize(s.x, s.out, s.scales, block_rows=c["block_rows"], dev_status=s.status)
        return s.out, s.scales
    if s.kind == "matmul":
        binding.rgd_fp8_matmul(s.x, s.sx, s.w, s.sw, s.y, k=c["k"], dev_status=s.status)
        return s.y
    binding.rgd_sample_top(s.logits, s.probe, s.temp, s.top_k, s.top_p, s.min_p, s.u, s.active, s.token, s.kept, s.prob,
                           vocab=c["vocab"], dev_status=s.status)
    return s.token, s.kept, s.prob


def run(s):
    return _run_own(s) if own else _plain(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    if c["kind"] == "rope":
        each = (c["heads"] + c["kv_heads"]) * c["dim"]
        return {"bytes": c["tokens"] * (2.0 * each * (4 if c["dtype"] == "f32" else 2) + 4), "flops": 6.0 * each * c["tokens"]}
    if c["kind"] == "rope_cache":
        tokens = float((_news(c) * (_active(c["rows"]) != 0)).sum())
        each = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": tokens * (4.0 * each + 4) + 16.0 * c["rows"], "flops": 6.0 * each * tokens}
    if c["kind"] == "quantize":
        n = float(c["rows"]) * c["cols"]
        scales = 4.0 * -(-c["rows"] // c["block_rows"]) * -(-c["cols"] // BLOCK)
        return {"bytes": n * (5 if c["dtype"] == "f32" else 3) + scales, "flops": 3 * n}
    if c["kind"] == "matmul":
        m, n, k = float(c["m"]), float(c["n"]), c["k"]
        scales = 4.0 * -(-k // BLOCK) * (m + -(-c["n"] // BLOCK))
        return {"bytes": (m + n) * k + scales + m * n * (4 if c["out"] == "f32" else 2), "flops": 2 * m * n * k}
    logits = float((_active(c["rows"]) != 0).sum()) * c["vocab"]
    return {"bytes": logits * (4 if c["dtype"] == "f32" else 2) + 37.0 * c["rows"], "flops": 4 * logits}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_turn(c, x, weight, positions):
    """As complex numbers: each pair times m e^(i t)."""
    f, magnitude = _frequencies(c)
    rot = c["rot"]
    x = x.double()
    if c["norm"]:
        x = weight.double() * (x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + 1e-6))
    t = torch.outer(positions.double().flatten(), torch.from_numpy(f).to(DEV)).view(*positions.shape, 1, rot // 2)
    by = torch.polar(torch.full_like(t, magnitude), t)
    if c["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * by
        return torch.cat([z.real, z.imag, x[..., rot:]], -1)
    z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * by
    return torch.cat([torch.view_as_real(z).flatten(-2), x[..., rot:]], -1)


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "rope":
        return _exact_turn(c, s.q, s.wq, s.positions), _exact_turn(c, s.k, s.wk, s.positions)
    if c["kind"] == "rope_cache":
        lens, new, on, first = _lengths(c), _news(c), _active(c["rows"]), s.first.cpu().numpy()
        table = s.table.cpu().numpy()
        where = [(r, i) for r in range(c["rows"]) if on[r] for i in range(new[r])]
        q, k = torch.zeros(s.q.shape, dtype=torch.float64, device=DEV), s.k_pages.double()
        if where:
            r, i = (torch.tensor(v, device=DEV) for v in zip(*where))
            pos = torch.tensor([int(first[a]) + int(lens[a]) + b for a, b in where], device=DEV)
            page = torch.tensor([int(table[a, (lens[a] + b) // PAGE]) for a, b in where], device=DEV)
            slot = torch.tensor([int(lens[a] + b) % PAGE for a, b in where], device=DEV)
            q[r, i] = _exact_turn(c, s.q[r, i], s.wq, pos)
            k[0][page, :, slot] = _exact_turn(c, s.k[r, i], s.wk, pos)
        return q, k, None
    if c["kind"] == "quantize":
        x, R, B = s.x.double().abs(), c["block_rows"], BLOCK
        out = torch.zeros(s.scales.shape, dtype=torch.float64, device=DEV)
        if R == 1:
            for b in range(out.shape[1]):
                out[:, b] = x[:, b * B:(b + 1) * B].amax(1) / 448
        else:
            for a in range(out.shape[0]):
                for b in range(out.shape[1]):
                    out[a, b] = x[a * R:(a + 1) * R, b * B:(b + 1) * B].max() / 448
        return None, out
    if c["kind"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        if float(m) * n * k > 6e11:
            return None
        y = torch.zeros((m, n), dtype=torch.float64, device=DEV)
        for b in range(-(-k // BLOCK)):
            at = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
            part = s.x[:, at].double() @ s.w[:, at].double().T
            y += part * s.sx[:, b, None].double() * s.sw[:, b].double().repeat_interleave(BLOCK)[:n]
        return y
    prob = torch.zeros(c["rows"], dtype=torch.float64, device=DEV)
    temp, top_k, top_p, min_p = _filters(c)
    on, u = _active(c["rows"]), s.u.cpu().numpy()
    for r in range(c["rows"]):
        if not on[r]:
            continue
        if r % c["rpg"] == 0 or temp[r] == 0:
            prob[r] = 1.0
            continue
        l = s.logits[r, :c["vocab"]].double()
        e = torch.exp((l - l.max()) / float(temp[r]))
        order = torch.argsort(l, descending=True, stable=True)
        if min_p[r] > 0:
            order = order[e[order] >= float(min_p[r])]
        if top_k[r] > 0:
            order = order[:int(top_k[r])]
        if top_p[r] < 1:
            upto = e[order].cumsum(0)
            order = order[:int((upto < float(top_p[r]) * upto[-1]).sum()) + 1]
        order = order.sort().values
        upto = e[order].cumsum(0)
        i = min(int((upto <= float(u[r]) * upto[-1]).sum()), order.numel() - 1)
        prob[r] = e[order[i]] / upto[-1]
    return None, None, prob
