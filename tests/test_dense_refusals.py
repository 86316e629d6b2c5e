"""Arguments that the dense operators' entry points refuse, on the host, before any launch."""
import ctypes

import pytest

from paper_2607_20791_gb300 import binding
from paper_2607_20791_gb300.build import build

P = 1 << 12  # any non-NULL, 16-byte aligned stand-in pointer
BAD, UNSUPPORTED = binding.RGD_ERR_INVALID_ARG, binding.RGD_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return binding.load_library(build())


def _refused(lib, rc, code, word):
    assert rc == code and word in lib.rgd_last_error_string(), (rc, lib.rgd_last_error_string())


@pytest.mark.parametrize("kw, word", [
    (dict(rot=3), b"rotary_dim"), (dict(rot=-2), b"rotary_dim"), (dict(base=0.5), b"base"), (dict(base=float("inf")), b"base"),
    (dict(base=float("nan")), b"base"), (dict(kind=5), b"scaling"), (dict(kind=1, factor=0.5), b"factor"),
    (dict(kind=3, factor=float("nan")), b"factor"), (dict(kind=3, trained=0.0), b"trained_length"),
    (dict(kind=4, low=4.0, high=4.0), b"low and high"), (dict(kind=4, base=1.0), b"RAMP"), (dict(turns=None), b"turns"),
    (dict(magnitude=False), b"magnitude"),
])
def test_frequency_refusals(lib, kw, word):
    a = {**dict(rot=8, base=1e4, kind=0, factor=2.0, trained=100.0, low=1.0, high=4.0, turns=(ctypes.c_uint64 * 4)(), magnitude=True), **kw}
    out = ctypes.byref(ctypes.c_double()) if a["magnitude"] else None
    turns = None if a["turns"] is None else ctypes.addressof(a["turns"])
    _refused(lib, lib.rgd_rope_frequencies(a["rot"], a["base"], a["kind"], a["factor"], a["trained"], a["low"], a["high"], turns, out),
             BAD, word)


def _rope(**kw):
    return binding.RopeShape(**{**dict(num_q_heads=4, num_k_heads=2, head_dim=64, rotary_dim=64, layout=0, norm=1, eps=1e-6,
                                       magnitude=1.0), **kw})


SHAPES = [(dict(num_q_heads=-1), BAD, b"heads"), (dict(head_dim=0), BAD, b"head_dim"), (dict(rotary_dim=66), BAD, b"rotary_dim"),
          (dict(rotary_dim=5), BAD, b"rotary_dim"), (dict(layout=2), BAD, b"layout"), (dict(norm=2), BAD, b"norm"),
          (dict(eps=-1.0), BAD, b"eps"), (dict(eps=float("nan")), BAD, b"eps"), (dict(magnitude=float("inf")), BAD, b"magnitude"),
          (dict(num_k_heads=4097), UNSUPPORTED, b"heads"), (dict(head_dim=1026, rotary_dim=2), UNSUPPORTED, b"head_dim")]


def _qk(lib, shape, tokens=3, dtype=1, q=P, qs=256, k=P, ks=128, pos=P, turns=P, wt=0, wq=None, wk=None, qo=P, qos=256, ko=P, kos=128):
    s = None if shape is None else ctypes.byref(shape)
    return lib.rgd_qk_rope(s, tokens, dtype, q, qs, k, ks, pos, turns, wt, wq, wk, qo, qos, ko, kos, None, None)


@pytest.mark.parametrize("kw, code, word", SHAPES)
def test_rope_shape_refusals(lib, kw, code, word):
    _refused(lib, _qk(lib, _rope(**kw)), code, word)


@pytest.mark.parametrize("kw, word", [
    (dict(tokens=-1), b"tokens"), (dict(dtype=2), b"dtype"), (dict(qs=-8), b"q_stride"), (dict(qos=255), b"q_out_stride"),
    (dict(kos=127), b"k_out_stride"), (dict(pos=None), b"positions"), (dict(q=None), b"non-NULL"), (dict(ko=None), b"non-NULL"),
    (dict(turns=None), b"turns"), (dict(turns=P + 4), b"turns"), (dict(wt=7), b"weight_dtype"), (dict(q=P + 1), b"aligned"),
    (dict(dtype=0, k=P + 2), b"aligned"), (dict(wq=P + 2), b"aligned"), (dict(wt=1, wk=P + 1), b"aligned"),
])
def test_rope_refusals(lib, kw, word):
    _refused(lib, _qk(lib, _rope(), **kw), BAD, word)


def test_rope_nothing_to_do(lib):
    _refused(lib, _qk(lib, None), BAD, b"shape")
    assert _qk(lib, _rope(), tokens=0, q=None, k=None, pos=None) == 0
    assert _qk(lib, _rope(num_q_heads=0, num_k_heads=0), q=None, k=None, qo=None, ko=None) == 0


def _cache(**kw):
    return binding.CacheShape(**{**dict(num_layers=2, num_pages=10, num_kv_heads=2, page_size=16, head_dim=64), **kw})


def _qkc(lib, shape=None, cache=None, layer=0, rows=2, new=1, q=P, k=P, v=P, rs=512, ts=512, first=None, turns=P, wt=0, n=P, cols=4,
         table=P, length=P, qo=P, kp=P, vp=P):
    shape, cache = shape or _rope(), cache or _cache()
    return lib.rgd_qk_rope_cache(ctypes.byref(shape), ctypes.byref(cache), layer, rows, new, q, k, v, rs, ts, first, turns, wt, None,
                                 None, n, cols, table, length, None, qo, kp, vp, None, None)


@pytest.mark.parametrize("kw, code, word", [
    (dict(cache=_cache(num_pages=0)), BAD, b"num_pages"), (dict(cache=_cache(page_size=8)), UNSUPPORTED, b"page_size"),
    (dict(shape=_rope(layout=9)), BAD, b"layout"), (dict(shape=_rope(num_k_heads=3)), BAD, b"differ"),
    (dict(shape=_rope(head_dim=128)), BAD, b"differ"), (dict(layer=2), BAD, b"layer"), (dict(rows=-1), BAD, b"rows"),
    (dict(cols=0), BAD, b"max_pages"), (dict(rs=-8), BAD, b"strides"), (dict(q=None), BAD, b"non-NULL"), (dict(v=None), BAD, b"non-NULL"),
    (dict(qo=None), BAD, b"non-NULL"), (dict(table=None), BAD, b"non-NULL"), (dict(k=P + 1), BAD, b"aligned"), (dict(kp=P + 8), BAD, b"pools"),
    (dict(rows=1 << 20, new=1 << 12), BAD, b"too many"),
])
def test_rope_cache_refusals(lib, kw, code, word):
    _refused(lib, _qkc(lib, **kw), code, word)


def test_rope_cache_nothing_to_do(lib):
    assert _qkc(lib, rows=0, q=None, k=None, table=None) == 0 and _qkc(lib, new=0, v=None) == 0


def _quant(lib, rows=2, cols=200, dtype=1, x=P, xs=200, each=1, q=P, qs=208, s=P):
    return lib.rgd_fp8_quantize(rows, cols, dtype, x, xs, each, q, qs, s, None, None)


@pytest.mark.parametrize("kw, code, word", [
    (dict(rows=-1), BAD, b"rows"), (dict(cols=-1), BAD, b"cols"), (dict(dtype=3), BAD, b"dtype"), (dict(each=2), BAD, b"block_rows"),
    (dict(xs=199), BAD, b"stride"), (dict(qs=199), BAD, b"stride"), (dict(x=None), BAD, b"non-NULL"), (dict(s=None), BAD, b"non-NULL"),
    (dict(x=P + 1), BAD, b"aligned"), (dict(s=P + 2), BAD, b"aligned"),
    (dict(rows=1 << 30, cols=1 << 20, xs=1 << 20, qs=1 << 20), UNSUPPORTED, b"too many"),
])
def test_quantize_refusals(lib, kw, code, word):
    _refused(lib, _quant(lib, **kw), code, word)
    assert _quant(lib, rows=0, x=None) == 0 and _quant(lib, cols=0, xs=0, qs=0, q=None) == 0


def _mm(lib, m=2, n=8, k=100, x=P, xs=112, sx=P, w=P, ws=112, sw=P, ot=0, y=P, ys=8):
    return lib.rgd_fp8_matmul(m, n, k, x, xs, sx, w, ws, sw, ot, y, ys, None, None)


@pytest.mark.parametrize("kw, code, word", [
    (dict(m=-1), BAD, b"m/n/k"), (dict(k=0), BAD, b"m/n/k"), (dict(k=(1 << 24) + 1, xs=1 << 25, ws=1 << 25), BAD, b"k too large"),
    (dict(ot=2), BAD, b"out_dtype"), (dict(xs=96), BAD, b"x_stride"), (dict(ws=96), BAD, b"w_stride"), (dict(ys=7), BAD, b"y_stride"),
    (dict(xs=104), BAD, b"multiples of 16"), (dict(ws=120), BAD, b"multiples of 16"), (dict(x=None), BAD, b"non-NULL"),
    (dict(sw=None), BAD, b"non-NULL"), (dict(x=P + 8), BAD, b"aligned"), (dict(w=P + 4), BAD, b"aligned"), (dict(y=P + 8), BAD, b"aligned"),
    (dict(sx=P + 2), BAD, b"scales"), (dict(m=(1 << 30) + 1), UNSUPPORTED, b"2^30"), (dict(xs=1 << 40), BAD, b"2^40"),
])
def test_matmul_refusals(lib, kw, code, word):
    _refused(lib, _mm(lib, **kw), code, word)
    assert _mm(lib, m=0, x=None) == 0 and _mm(lib, n=0, w=None, ys=0) == 0


def _sample(lib, rows=2, vocab=100, dtype=0, logits=P, stride=100, temp=P, u=P, token=P):
    return lib.rgd_sample_top(rows, vocab, dtype, logits, stride, None, temp, None, None, None, u, None, token, None, None, None, None)


@pytest.mark.parametrize("kw, code, word", [
    (dict(rows=-1), BAD, b"rows"), (dict(vocab=0), BAD, b"vocab"), (dict(dtype=2), BAD, b"dtype"), (dict(stride=99), BAD, b"stride"),
    (dict(logits=None), BAD, b"logits"), (dict(temp=None), BAD, b"temperature"), (dict(u=None), BAD, b"draw_u"),
    (dict(token=None), BAD, b"token_out"), (dict(logits=P + 8), BAD, b"aligned"),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED, b"vocab"), (dict(rows=1 << 28), UNSUPPORTED, b"rows"),
])
def test_sample_refusals(lib, kw, code, word):
    _refused(lib, _sample(lib, **kw), code, word)
    assert _sample(lib, rows=0, logits=None, temp=None) == 0


def test_binding_refuses_wrong_tensors(lib):
    torch = pytest.importorskip("torch")
    i32, i64, bf, f8 = torch.int32, torch.int64, torch.bfloat16, torch.float8_e4m3fn
    shape = _rope()
    good = dict(shape=shape, q=torch.empty(3, 4, 64, dtype=bf), k=torch.empty(3, 2, 64, dtype=bf), positions=torch.empty(3, dtype=i32),
                turns=torch.empty(32, dtype=i64), q_weight=torch.empty(64), k_weight=torch.empty(64),
                q_out=torch.empty(3, 4, 64, dtype=bf), k_out=torch.empty(3, 2, 64, dtype=bf))
    for name, t in (("q", torch.empty(2, 4, 64, dtype=bf)), ("k", torch.empty(3, 2, 32, dtype=bf)), ("turns", torch.empty(31, dtype=i64)),
                    ("q_weight", torch.empty(63)), ("q_out", torch.empty(3, 64, 4, dtype=bf).transpose(1, 2))):
        with pytest.raises(ValueError, match=name):
            binding.rgd_qk_rope(**{**good, name: t})
    for name, t in (("k", torch.empty(3, 2, 64)), ("q", torch.empty(3, 4, 64, dtype=torch.float16)), ("q", None),
                    ("k_weight", torch.empty(64, dtype=bf)), ("positions", torch.empty(3, dtype=i64)), ("positions", None)):
        with pytest.raises(TypeError, match=name):
            binding.rgd_qk_rope(**{**good, name: t})
    with pytest.raises(ValueError, match="CUDA"):
        binding.rgd_qk_rope(**good)
    cache, per_row, table = _cache(), torch.empty(2, dtype=i32), torch.empty(2, 4, dtype=i32)
    pool = torch.empty(2 * 10 * 2 * 16 * 64, dtype=bf)
    qkv = torch.empty(2, 3, 8, 64, dtype=bf)
    good = dict(shape=shape, cache=cache, layer=0, q=qkv[:, :, :4], k=qkv[:, :, 4:6], v=qkv[:, :, 6:], first_position=None,
                turns=torch.empty(32, dtype=i64), q_weight=None, k_weight=None, n_new=per_row, block_table=table, length=per_row,
                row_active=None, q_out=torch.empty(2, 3, 4, 64, dtype=bf), k_pages=pool, v_pages=pool)
    for name, t, word in (("v", qkv[:, :2, 6:], "leading"), ("q", qkv[:1, :, :4], "leading"), ("k", qkv[..., 4:6, :].contiguous(), "strides"),
                          ("q_out", torch.empty(2, 3, 4, 63, dtype=bf), "q_out"), ("k_pages", pool[:-1], "k_pages"),
                          ("n_new", per_row[:1], "n_new"), ("first_position", per_row[:1], "first_position")):
        with pytest.raises(ValueError, match=word):
            binding.rgd_qk_rope_cache(**{**good, name: t})
    with pytest.raises(ValueError, match="CUDA"):
        binding.rgd_qk_rope_cache(**good)
    x, q = torch.empty(5, 200, dtype=bf), torch.empty(5, 208, dtype=f8)
    for args, word in (((x, q[:4], torch.empty(10)), "q must"), ((x, q[:, :199], torch.empty(10)), "q must"), ((x, q, torch.empty(9)), "scales"),
                       ((x.t(), q, torch.empty(10)), "columns"), ((x, q, torch.empty(10)), "CUDA")):
        with pytest.raises(ValueError, match=word):
            binding.rgd_fp8_quantize(*args)
    with pytest.raises(TypeError, match="q must"):
        binding.rgd_fp8_quantize(x, q.view(torch.int8), torch.empty(10))
    w, y = torch.empty(7, 208, dtype=f8), torch.empty(5, 7)
    good = dict(x=q, x_scales=torch.empty(10), weights=w, w_scales=torch.empty(2), y=y, k=200)
    for name, t, word in (("x_scales", torch.empty(9), "x_scales"), ("w_scales", torch.empty(1), "w_scales"), ("y", y[:4], "y must"),
                          ("y", y[:, :6], "y must"), ("k", 209, "columns"), ("weights", w[:, :199], "columns")):
        with pytest.raises(ValueError, match=word):
            binding.rgd_fp8_matmul(**{**good, name: t})
    with pytest.raises(ValueError, match="CUDA"):
        binding.rgd_fp8_matmul(**good)
    rows = torch.empty(3)
    good = dict(logits=torch.empty(3, 50), is_probe=None, temperature=rows, top_k=rows.int(), top_p=rows, min_p=rows, draw_u=rows,
                row_active=None, token_out=rows.int(), kept_count=rows.int(), prob_out=rows, vocab=40)
    for name in ("temperature", "top_k", "top_p", "min_p", "draw_u", "token_out", "kept_count", "prob_out"):
        with pytest.raises(ValueError, match=name):
            binding.rgd_sample_top(**{**good, name: good[name][:2]})
    with pytest.raises(ValueError, match="rows of 50"):
        binding.rgd_sample_top(**{**good, "vocab": 51})
    with pytest.raises(ValueError, match="CUDA"):
        binding.rgd_sample_top(**good)
    with pytest.raises(ValueError, match="scaling"):
        binding.rgd_rope_frequencies(8, 1e4, "other")
