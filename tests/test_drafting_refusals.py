"""Arguments that the drafting entry points refuse, on the host, before any launch."""
import ctypes

import pytest

from paper_2607_20791_gb300 import binding
from paper_2607_20791_gb300.build import build

P = 1 << 12  # any non-NULL, 16-byte aligned stand-in pointer
BAD = binding.RGD_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    return binding.load_library(build())


def _verify(lib, rows=2, draft=3, vocab=100, dtype=0, target=P, tstride=100, dlogits=P, dstride=100, tokens=P, n=None,
            probe=None, temp=P, minp=P, au=P, du=P, active=None, out=P, acc=P, prob=None, ws=P, wsb=1 << 20):
    return lib.rgd_verify_draft(rows, draft, vocab, dtype, target, tstride, dlogits, dstride, tokens, n, probe, temp, minp,
                                au, du, active, out, acc, prob, ws, wsb, None, None)


@pytest.mark.parametrize("bad, word", [
    (dict(rows=-1), b"rows"), (dict(draft=-1), b"max_draft"), (dict(vocab=0), b"vocab"), (dict(dtype=5), b"dtype"),
    (dict(tstride=99), b"stride"), (dict(dstride=99), b"stride"), (dict(target=None), b"target_logits"),
    (dict(target=P + 8), b"aligned"), (dict(dlogits=P + 2), b"aligned"), (dict(tokens=None), b"draft_tokens"),
    (dict(au=None), b"accept_u"), (dict(du=None), b"draw_u"), (dict(temp=None), b"temperature"),
    (dict(minp=None), b"min_p"), (dict(out=None), b"token_out"), (dict(acc=None), b"accepted_out"),
    (dict(ws=None), b"workspace"), (dict(ws=P + 2), b"workspace"), (dict(wsb=2 * 5 * 4 - 1), b"workspace too small"),
])
def test_verify_refusals(lib, bad, word):
    assert _verify(lib, **bad) == BAD
    assert word in lib.rgd_last_error_string()


def test_verify_limits_and_empty_batch(lib):
    assert _verify(lib, vocab=(1 << 20) + 1, tstride=1 << 21, dstride=1 << 21) == binding.RGD_ERR_UNSUPPORTED
    assert _verify(lib, rows=1 << 27, draft=15, wsb=1 << 60) == binding.RGD_ERR_UNSUPPORTED
    assert _verify(lib, rows=0, target=None, temp=None) == 0
    assert lib.rgd_verify_draft_workspace_size(-1, 2) == 0
    assert lib.rgd_verify_draft_workspace_size(7, 4) == 7 * 6 * 4
    with pytest.raises(binding.RgdError):
        binding.rgd_verify_draft_workspace_size(1, -1)


def _w4(lib, m=2, n=8, k=64, g=32, x=P, w=P, st=0, s=P, z=None, ot=0, y=P, ys=8):
    return lib.rgd_w4_matvec(m, n, k, g, x, w, st, s, z, ot, y, ys, None, None)


@pytest.mark.parametrize("bad, word", [
    (dict(m=-1), b"m/n/k"), (dict(n=-1), b"m/n/k"), (dict(k=0), b"m/n/k"), (dict(k=(1 << 24) + 1), b"k too large"),
    (dict(g=16), b"group_size"), (dict(g=0), b"group_size"), (dict(st=2), b"scale_dtype"), (dict(ot=-1), b"out_dtype"),
    (dict(ys=7), b"y_stride"), (dict(x=None), b"x/weights"), (dict(w=None), b"weights"), (dict(s=None), b"scales"),
    (dict(y=None), b"y must"), (dict(w=P + 4), b"aligned"), (dict(z=P + 1), b"aligned"),
])
def test_w4_refusals(lib, bad, word):
    assert _w4(lib, **bad) == BAD
    assert word in lib.rgd_last_error_string()


def test_w4_empty(lib):
    assert _w4(lib, m=0, x=None) == 0 and _w4(lib, n=0, w=None, ys=0) == 0


def _shape(**kw):
    return binding.CacheShape(**{**dict(num_layers=2, num_pages=10, num_kv_heads=2, page_size=16, head_dim=64), **kw})


@pytest.mark.parametrize("kw, code, word", [
    (dict(num_layers=0), BAD, b"num_layers"), (dict(num_pages=0), BAD, b"num_pages"), (dict(reserved=1), BAD, b"reserved"),
    (dict(layer_stride=100), BAD, b"layer_stride"), (dict(layer_stride=10 * 2 * 16 * 64 + 4), BAD, b"layer_stride"),
    (dict(page_size=32), binding.RGD_ERR_UNSUPPORTED, b"page_size"), (dict(head_dim=60), binding.RGD_ERR_UNSUPPORTED, b"head_dim"),
    (dict(head_dim=2048), binding.RGD_ERR_UNSUPPORTED, b"head_dim"), (dict(num_kv_heads=5000), binding.RGD_ERR_UNSUPPORTED, b"heads"),
])
def test_cache_shape_refusals(lib, kw, code, word):
    s = ctypes.byref(_shape(**kw))
    assert lib.rgd_cache_workspace_size(s, 4) == 0 and word in lib.rgd_last_error_string()
    assert lib.rgd_cache_reserve(s, 2, 4, P, P, P, None, P, P, P, None, P, 1 << 20, None, None) == code
    assert lib.rgd_cache_write(s, 0, 2, 1, P, P, 128, 128, P, 4, P, P, None, P, P, None, None) == code
    assert lib.rgd_cache_copy(s, 1, P, P, P, P, None, None) == code
    assert lib.rgd_cache_compact(s, 2, 4, P, 0, 0, None, P, P, P, P, P, 1 << 20, None, None) == code


def test_cache_refusals(lib):
    s, need = ctypes.byref(_shape()), lib.rgd_cache_workspace_size(ctypes.byref(_shape()), 2)
    assert need == 256 + 4 * (40 + 2)

    def refused(rc, word):
        assert rc == BAD and word in lib.rgd_last_error_string()
    refused(lib.rgd_cache_reserve(s, -1, 4, P, P, P, None, P, P, P, None, P, need, None, None), b"rows")
    refused(lib.rgd_cache_reserve(s, 2, 0, P, P, P, None, P, P, P, None, P, need, None, None), b"max_pages")
    refused(lib.rgd_cache_reserve(s, 2, 4, None, P, P, None, P, P, P, None, P, need, None, None), b"block_table")
    refused(lib.rgd_cache_reserve(s, 2, 4, P, P, P, None, P, P + 2, P, None, P, need, None, None), b"aligned")
    refused(lib.rgd_cache_reserve(s, 2, 4, P, P, P, None, P, P, P, None, P, need - 1, None, None), b"too small")
    refused(lib.rgd_cache_write(s, 2, 2, 1, P, P, 128, 128, P, 4, P, P, None, P, P, None, None), b"layer")
    refused(lib.rgd_cache_write(s, 0, 2, 1, P, P, 128, 4, P, 4, P, P, None, P, P, None, None), b"strides")
    refused(lib.rgd_cache_write(s, 0, 2, 1, P, P, -8, 128, P, 4, P, P, None, P, P, None, None), b"strides")
    refused(lib.rgd_cache_write(s, 0, 2, 1, None, P, 128, 128, P, 4, P, P, None, P, P, None, None), b"k_new")
    refused(lib.rgd_cache_trim(2, 4, 0, P, P, None, P, None, None), b"num_pages")
    refused(lib.rgd_cache_trim(2, 4, 10, P, None, None, P, None, None), b"length")
    refused(lib.rgd_cache_fork(-1, P, P, 2, 4, 10, P, P, P, None, None), b"pairs")
    refused(lib.rgd_cache_fork(1, None, P, 2, 4, 10, P, P, P, None, None), b"parent")
    refused(lib.rgd_cache_copy(s, -1, P, P, P, P, None, None), b"n < 0")
    refused(lib.rgd_cache_copy(s, 1, None, P, P, P, None, None), b"src")
    refused(lib.rgd_cache_compact(s, 2, 4, P, 0, 0, None, P, P, P, None, P, need, None, None), b"num_live")
    # nothing to do is not an error
    assert lib.rgd_cache_reserve(s, 0, 4, None, None, None, None, None, None, None, None, None, 0, None, None) == 0
    assert lib.rgd_cache_write(s, 0, 2, 0, None, None, 0, 0, None, 4, None, None, None, None, None, None, None) == 0
    assert lib.rgd_cache_trim(0, 4, 10, None, None, None, None, None, None) == 0
    assert lib.rgd_cache_fork(0, None, None, 2, 4, 10, None, None, None, None, None) == 0
    assert lib.rgd_cache_copy(s, 0, None, None, None, None, None, None) == 0


def test_binding_refuses_wrong_tensors(lib):
    torch = pytest.importorskip("torch")
    i32, u8, f32, bf = torch.int32, torch.uint8, torch.float32, torch.bfloat16
    R, K, V = 3, 2, 40
    good = dict(target_logits=torch.empty(R, K + 1, V), draft_logits=torch.empty(R, K, V),
                draft_tokens=torch.empty(R * K, dtype=i32), n_draft=torch.empty(R, dtype=i32),
                is_probe=torch.empty(R, dtype=u8), temperature=torch.empty(R), min_p=torch.empty(R),
                accept_u=torch.empty(R * K), draw_u=torch.empty(R), row_active=torch.empty(R, dtype=u8),
                token_out=torch.empty(R * (K + 1), dtype=i32), accepted_out=torch.empty(R, dtype=i32),
                accept_prob=torch.empty(R * K), workspace=torch.empty(1024, dtype=u8))
    for name in ("draft_tokens", "n_draft", "is_probe", "temperature", "min_p", "accept_u", "draw_u", "row_active",
                 "token_out", "accepted_out", "accept_prob"):
        with pytest.raises(ValueError, match=name):
            binding.rgd_verify_draft(**{**good, name: good[name][:-1]})
    for name, t in (("draft_logits", torch.empty(R, K + 1, V)), ("target_logits", torch.empty(R, V))):
        with pytest.raises(ValueError, match=name):
            binding.rgd_verify_draft(**{**good, name: t})
    with pytest.raises(TypeError, match="draft_logits"):
        binding.rgd_verify_draft(**{**good, "draft_logits": torch.empty(R, K, V, dtype=bf)})
    with pytest.raises(ValueError, match="CUDA"):
        binding.rgd_verify_draft(**good)
    w4 = dict(x=torch.empty(2, 64, dtype=bf), weights=torch.empty(8, 32, dtype=u8), scales=torch.empty(16),
              zeros=torch.empty(16, dtype=u8), group_size=32, y=torch.empty(2, 8))
    for name, t in (("weights", torch.empty(8, 31, dtype=u8)), ("scales", torch.empty(15)),
                    ("zeros", torch.empty(15, dtype=u8)), ("y", torch.empty(2, 7)), ("y", torch.empty(1, 8))):
        with pytest.raises(ValueError, match=name):
            binding.rgd_w4_matvec(**{**w4, name: t})
    with pytest.raises(TypeError, match="x"):
        binding.rgd_w4_matvec(**{**w4, "x": torch.empty(2, 64)})
    shape = _shape()
    pool = torch.empty(2 * 10 * 2 * 16 * 64, dtype=bf)
    table, per_row = torch.empty(2, 4, dtype=i32), torch.empty(2, dtype=i32)
    with pytest.raises(ValueError, match="k_pages"):
        binding.rgd_cache_reserve(shape, table, per_row, per_row, None, torch.empty(10, dtype=i32), pool[:-1], pool, None,
                                  torch.empty(1024, dtype=u8))
    with pytest.raises(ValueError, match="page_refs"):
        binding.rgd_cache_reserve(shape, table, per_row, per_row, None, torch.empty(9, dtype=i32), pool, pool, None,
                                  torch.empty(1024, dtype=u8))
    new = torch.empty(2, 3, 2, 64, dtype=bf)
    with pytest.raises(ValueError, match="k_new"):
        binding.rgd_cache_write(shape, 0, new[..., :32], new, per_row, table, per_row, None, pool, pool)
    with pytest.raises(ValueError, match="dense"):
        binding.rgd_cache_write(shape, 0, new.transpose(2, 3).contiguous().transpose(2, 3), new, per_row, table, per_row,
                                None, pool, pool)
    with pytest.raises(ValueError, match="strides"):
        binding.rgd_cache_write(shape, 0, new, new[:, :2], per_row, table, per_row, None, pool, pool)
    with pytest.raises(ValueError, match="length"):
        binding.rgd_cache_trim(table, per_row[:1], None, torch.empty(10, dtype=i32))
    with pytest.raises(ValueError, match="block_table"):
        binding.rgd_cache_trim(per_row, per_row, None, torch.empty(10, dtype=i32))
