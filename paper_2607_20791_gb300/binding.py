"""Thin ctypes binding of the C ABI in ``include/rgd.h`` (argument marshalling only).

Every function here has the name of the C entry point it calls and does nothing
but check and convert arguments: torch CUDA tensors become device pointers, the
current torch CUDA stream becomes the stream argument, and a non-zero status is
raised as :class:`RgdError`.  All computation happens in the CUDA kernels of
``librgd.so``; there is no fallback.  If the library has not been built the first
call raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librgd.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "rgd.h")

RGD_OK, RGD_ERR_INVALID_ARG, RGD_ERR_CUDA, RGD_ERR_UNSUPPORTED = 0, 1, 2, 3
RGD_DEV_BAD_PAGE, RGD_DEV_BAD_TOKEN, RGD_DEV_WAIT_TIMEOUT, RGD_DEV_BAD_PARAM, RGD_DEV_NO_PAGE = 1, 2, 4, 8, 16
RGD_F32, RGD_BF16 = 0, 1
RGD_ROPE_HALF, RGD_ROPE_PAIRS = 0, 1
RGD_ROPE_PLAIN, RGD_ROPE_LINEAR, RGD_ROPE_BASE, RGD_ROPE_BANDS, RGD_ROPE_RAMP = 0, 1, 2, 3, 4
RGD_PENDING, RGD_REFUSAL, RGD_NON_REFUSAL = 0, 1, 2


class RgdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"rgd error {code}: {msg}")
        self.code = code


class AttnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_groups", "rows_per_group", "num_q_heads", "num_kv_heads", "head_dim", "page_size",
        "num_pages", "max_prompt_pages", "max_suffix_pages", "num_ctas", "reserved")]


class CacheShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_layers", "num_pages", "num_kv_heads", "page_size", "head_dim", "reserved")] + [
            ("layer_stride", ctypes.c_int64)]


class RopeShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_q_heads", "num_k_heads", "head_dim", "rotary_dim", "layout", "norm")] + [
            ("eps", ctypes.c_float), ("magnitude", ctypes.c_float)]


class GateState(ctypes.Structure):
    _fields_ = [("node", ctypes.c_int32), ("length", ctypes.c_int32), ("steps", ctypes.c_int32),
                ("decisive_step", ctypes.c_int32), ("decision", ctypes.c_uint8),
                ("confirmed", ctypes.c_uint8), ("done", ctypes.c_uint8), ("reserved", ctypes.c_uint8)]


GATE_STATE_BYTES = ctypes.sizeof(GateState)  # 20

_lib = None
_P = ctypes.c_void_p
_I32, _I64, _U64, _SZ, _F = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_float
_D = ctypes.c_double

_SIGNATURES = {
    "rgd_last_error_string": (ctypes.c_char_p, []),
    "rgd_version": (ctypes.c_char_p, []),
    "rgd_set_wait_limit_ns": (ctypes.c_int, [_U64]),
    "rgd_prefix_decode_attn_workspace_size": (_SZ, [ctypes.POINTER(AttnShape)]),
    "rgd_prefix_decode_attn": (ctypes.c_int, [ctypes.POINTER(AttnShape), _P, _P, _P, _P, _P, _P, _P, _P, _F,
                                               _P, _P, _P, _SZ, _P, _P]),
    "rgd_prefix_decode_attn_noalloc": (ctypes.c_int, [ctypes.POINTER(AttnShape), _P, _P, _P, _P, _P, _P, _P,
                                                       _P, _F, _P, _P, _P, _P]),
    "rgd_sample_head": (ctypes.c_int, [_I32, _I32, _I32, _P, _P, _P, _P, _P, _U64, _P, _P, _P, _P, _P, _P]),
    "rgd_sample_head_gated": (ctypes.c_int, [_I32, _I32, _I32, _P, _P, _P, _P, _P, _U64, _P, _P, _P, _P, _I32,
                                             _I32, _I32, _P, _P, _P]),
    "rgd_decode_step": (ctypes.c_int, [ctypes.POINTER(AttnShape), _P, _P, _P, _P, _P, _P, _P, _F, _P, _P, _P,
                                       _SZ, _I32, _I32, _P, _P, _P, _P, _P, _U64, _P, _P, _P, _P, _I32, _I32,
                                       _P, _P, _P]),
    "rgd_trie_create": (ctypes.c_int, [_P, _P, _I32, _I32, ctypes.POINTER(_P)]),
    "rgd_trie_destroy": (ctypes.c_int, [_P]),
    "rgd_trie_info": (ctypes.c_int, [_P, ctypes.POINTER(_I32), ctypes.POINTER(_I32)]),
    "rgd_gate_state_init": (ctypes.c_int, [_P, _I32, _P]),
    "rgd_probe_gate": (ctypes.c_int, [_P, _I32, _I32, _P, _I32, _I64, _I32, _I32, _P, _P, _P, _P]),
    "rgd_residual_precheck": (ctypes.c_int, [_I32, _I32, _I32, _P, _P, _F, _F, _I32, _P, _P, _P, _P, _P]),
    "rgd_soft_gate": (ctypes.c_int, [_P, _I32, _I32, _I32, _I32, _P, _I64, _I32, _F, _I32, _I32, _I32, _P, _P,
                                     _P, _P, _P, _P]),
    "rgd_verify_draft_workspace_size": (_SZ, [_I32, _I32]),
    "rgd_verify_draft": (ctypes.c_int, [_I32, _I32, _I32, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P,
                                        _P, _P, _P, _P, _SZ, _P, _P]),
    "rgd_w4_matvec": (ctypes.c_int, [_I32, _I32, _I32, _I32, _P, _P, _I32, _P, _P, _I32, _P, _I64, _P, _P]),
    "rgd_cache_workspace_size": (_SZ, [ctypes.POINTER(CacheShape), _I32]),
    "rgd_cache_reserve": (ctypes.c_int, [ctypes.POINTER(CacheShape), _I32, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                         _SZ, _P, _P]),
    "rgd_cache_write": (ctypes.c_int, [ctypes.POINTER(CacheShape), _I32, _I32, _I32, _P, _P, _I64, _I64, _P, _I32, _P,
                                       _P, _P, _P, _P, _P, _P]),
    "rgd_cache_trim": (ctypes.c_int, [_I32, _I32, _I32, _P, _P, _P, _P, _P, _P]),
    "rgd_cache_fork": (ctypes.c_int, [_I32, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]),
    "rgd_cache_copy": (ctypes.c_int, [ctypes.POINTER(CacheShape), _I32, _P, _P, _P, _P, _P, _P]),
    "rgd_cache_compact": (ctypes.c_int, [ctypes.POINTER(CacheShape), _I32, _I32, _P, _I32, _I32, _P, _P, _P, _P, _P,
                                         _P, _SZ, _P, _P]),
    "rgd_rope_frequencies": (ctypes.c_int, [_I32, _D, _I32, _D, _D, _D, _D, _P, ctypes.POINTER(_D)]),
    "rgd_qk_rope": (ctypes.c_int, [ctypes.POINTER(RopeShape), _I32, _I32, _P, _I64, _P, _I64, _P, _P, _I32, _P, _P, _P, _I64,
                                   _P, _I64, _P, _P]),
    "rgd_qk_rope_cache": (ctypes.c_int, [ctypes.POINTER(RopeShape), ctypes.POINTER(CacheShape), _I32, _I32, _I32, _P, _P, _P,
                                         _I64, _I64, _P, _P, _I32, _P, _P, _P, _I32, _P, _P, _P, _P, _P, _P, _P, _P]),
    "rgd_fp8_quantize": (ctypes.c_int, [_I32, _I32, _I32, _P, _I64, _I32, _P, _I64, _P, _P, _P]),
    "rgd_sample_top": (ctypes.c_int, [_I32, _I32, _I32, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "rgd_fp8_matmul": (ctypes.c_int, [_I32, _I32, _I32, _P, _I64, _P, _P, _I64, _P, _I32, _P, _I64, _P, _P]),
}


def header_symbols(path: str = HEADER):
    """Function names declared in the C header."""
    text = open(path).read()
    return sorted(set(re.findall(r"^\s*(?:[A-Za-z_][\w\s\*]*?)\b(rgd_\w+)\s*\(", text, re.M)))


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load ``librgd.so`` (once) and declare the signatures; raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(python -m paper_2607_20791_gb300.build)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != RGD_OK:
        raise RgdError(rc, load_library().rgd_last_error_string().decode())


class _HostTensor:
    """Stands in for the pointer of a tensor that is not on the GPU; :func:`_call`
    refuses the call once every other argument has been checked."""

    def __init__(self, name: str):
        self.name = name


def _call(fn, *args):
    """Call a C entry point unless an argument is a host tensor (which ctypes
    refuses to convert: the arguments are looked through only then)."""
    try:
        return fn(*args)
    except ctypes.ArgumentError:
        for a in args:
            if isinstance(a, _HostTensor):
                raise ValueError(f"{a.name} must be a CUDA tensor") from None
        raise


_Tensor = None  # torch.Tensor, once an argument has been checked (importing this module does not import torch)


def _ptr(t, name: str, dtype=None, optional: bool = False, numel: Optional[int] = None):
    """Device pointer of a contiguous CUDA tensor (or a raw int pointer, passed
    through unchecked).  ``numel`` is the number of elements the call will
    touch: a smaller tensor is refused here, since the C side sees only the
    pointer.  A host tensor gives a :class:`_HostTensor`, refused by
    :func:`_call`, so that every argument's type and size is checked first."""
    global _Tensor
    # A call has up to 22 tensors and its launch takes about as long as checking
    # them: one that passes every check returns here (0.45 us; 0.84 us with the
    # checks below for each), any other goes on to the check that it fails.
    if type(t) is _Tensor and (dtype is None or t.dtype is dtype) and t.is_contiguous() and t.is_cuda and (
            numel is None or t.numel() >= numel):
        return t.data_ptr()
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if isinstance(t, int):
        return t
    import torch
    _Tensor = torch.Tensor
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor or an int pointer")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{name}: dtype {t.dtype} not accepted")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, the call needs {numel}")
    if not t.is_cuda:
        return _HostTensor(name)
    return t.data_ptr()


_raw_stream = None  # (current device, its current stream), once asked for: without a Stream object 2 us less


def _stream(stream) -> Optional[int]:
    global _raw_stream
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream[1](_raw_stream[0]())
        import torch
        try:
            torch.cuda.current_device()  # (initialises CUDA)
            raw = (getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None))
            if None not in raw:
                _raw_stream = raw
                return raw[1](raw[0]())
            return torch.cuda.current_stream().cuda_stream
        except (RuntimeError, AssertionError):  # no CUDA device: the call is refused or fails in CUDA
            return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def rgd_version() -> str:
    return load_library().rgd_version().decode()


def rgd_set_wait_limit_ns(limit_ns: int) -> None:
    """Limit of the attention kernel's waits for later calls (0: the default, 2 s)."""
    _check(load_library().rgd_set_wait_limit_ns(int(limit_ns)))


def rgd_prefix_decode_attn_workspace_size(shape: AttnShape) -> int:
    n = load_library().rgd_prefix_decode_attn_workspace_size(ctypes.byref(shape))
    if n == 0:
        raise RgdError(RGD_ERR_INVALID_ARG, load_library().rgd_last_error_string().decode())
    return int(n)


def _attn_sizes(shape: AttnShape) -> dict:
    """Elements each attention argument must hold for ``shape``."""
    R = shape.num_groups * shape.rows_per_group
    return {"q": R * shape.num_q_heads * shape.head_dim,
            "kv": shape.num_pages * shape.num_kv_heads * shape.page_size * shape.head_dim,
            "pbt": shape.num_groups * shape.max_prompt_pages, "plen": shape.num_groups,
            "sbt": R * shape.max_suffix_pages, "rows": R, "lse": R * shape.num_q_heads}


def rgd_prefix_decode_attn(shape: AttnShape, q, k_pages, v_pages, prompt_block_table, prompt_len,
                           suffix_block_table, suffix_len, row_active, softmax_scale: float, out, lse,
                           workspace, dev_status=None, stream=None) -> None:
    import torch
    lib = load_library()
    n = _attn_sizes(shape)
    ws_bytes = workspace.numel() * workspace.element_size() if isinstance(workspace, torch.Tensor) else 0
    _check(_call(lib.rgd_prefix_decode_attn,
        ctypes.byref(shape), _ptr(q, "q", torch.bfloat16, numel=n["q"]),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=n["kv"]), _ptr(v_pages, "v_pages", torch.bfloat16, numel=n["kv"]),
        _ptr(prompt_block_table, "prompt_block_table", torch.int32, numel=n["pbt"]),
        _ptr(prompt_len, "prompt_len", torch.int32, numel=n["plen"]),
        _ptr(suffix_block_table, "suffix_block_table", torch.int32, numel=n["sbt"]),
        _ptr(suffix_len, "suffix_len", torch.int32, numel=n["rows"]),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=n["rows"]), float(softmax_scale),
        _ptr(out, "out", torch.bfloat16, numel=n["q"]), _ptr(lse, "lse", torch.float32, optional=True, numel=n["lse"]),
        _ptr(workspace, "workspace"), ws_bytes, _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1),
        _stream(stream)))


def rgd_prefix_decode_attn_noalloc(shape: AttnShape, q, k_pages, v_pages, prompt_block_table, prompt_len,
                                   suffix_block_table, suffix_len, row_active, softmax_scale: float, out,
                                   lse, dev_status=None, stream=None) -> None:
    """Same as :func:`rgd_prefix_decode_attn` without a workspace: the library's
    fixed device scratch is used (for callers that cannot allocate device memory)."""
    import torch
    n = _attn_sizes(shape)
    _check(_call(load_library().rgd_prefix_decode_attn_noalloc,
        ctypes.byref(shape), _ptr(q, "q", torch.bfloat16, numel=n["q"]),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=n["kv"]), _ptr(v_pages, "v_pages", torch.bfloat16, numel=n["kv"]),
        _ptr(prompt_block_table, "prompt_block_table", torch.int32, numel=n["pbt"]),
        _ptr(prompt_len, "prompt_len", torch.int32, numel=n["plen"]),
        _ptr(suffix_block_table, "suffix_block_table", torch.int32, numel=n["sbt"]),
        _ptr(suffix_len, "suffix_len", torch.int32, numel=n["rows"]),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=n["rows"]), float(softmax_scale),
        _ptr(out, "out", torch.bfloat16, numel=n["q"]), _ptr(lse, "lse", torch.float32, optional=True, numel=n["lse"]),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_sample_head(logits, is_probe, temperature, min_p, seed, step: int, row_active, token_out,
                    kept_count=None, kept_mask=None, dev_status=None, stream=None) -> None:
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    dtype = {torch.float32: RGD_F32, torch.bfloat16: RGD_BF16}.get(logits.dtype)
    if dtype is None:
        raise TypeError("logits must be float32 or bfloat16")
    rows, vocab = logits.shape
    _check(_call(load_library().rgd_sample_head,
        rows, vocab, dtype, _ptr(logits, "logits"),
        _ptr(is_probe, "is_probe", torch.uint8, optional=True, numel=rows),
        _ptr(temperature, "temperature", torch.float32, numel=rows), _ptr(min_p, "min_p", torch.float32, numel=rows),
        _ptr(seed, "seed", (torch.int64, torch.uint64), numel=rows), int(step) & 0xFFFFFFFFFFFFFFFF,
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows),
        _ptr(token_out, "token_out", torch.int32, numel=rows),
        _ptr(kept_count, "kept_count", torch.int32, optional=True, numel=rows),
        _ptr(kept_mask, "kept_mask", torch.uint8, optional=True, numel=rows * vocab),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def _logits_dtype(logits):
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    dtype = {torch.float32: RGD_F32, torch.bfloat16: RGD_BF16}.get(logits.dtype)
    if dtype is None:
        raise TypeError("logits must be float32 or bfloat16")
    return dtype


def rgd_sample_head_gated(logits, is_probe, temperature, min_p, seed, step: int, row_active, token_out,
                          kept_count, trie: "Trie", rows_per_group: int, eos_token: int, max_len: int, state,
                          dev_status=None, stream=None) -> None:
    """The sample head and the hard gate of one step in one kernel (see the C header)."""
    import torch
    dtype = _logits_dtype(logits)
    rows, vocab = logits.shape
    rpg = int(rows_per_group)
    groups = rows // rpg if rpg > 0 else 0
    _check(_call(load_library().rgd_sample_head_gated,
        rows, vocab, dtype, _ptr(logits, "logits"),
        _ptr(is_probe, "is_probe", torch.uint8, optional=True, numel=rows),
        _ptr(temperature, "temperature", torch.float32, numel=rows), _ptr(min_p, "min_p", torch.float32, numel=rows),
        _ptr(seed, "seed", (torch.int64, torch.uint64), numel=rows), int(step) & 0xFFFFFFFFFFFFFFFF,
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows),
        _ptr(token_out, "token_out", torch.int32, numel=rows),
        _ptr(kept_count, "kept_count", torch.int32, optional=True, numel=rows),
        trie.handle, rpg, int(eos_token), int(max_len), _state_ptr(state, groups),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_decode_step(shape: AttnShape, q, k_pages, v_pages, prompt_block_table, prompt_len, suffix_block_table,
                    suffix_len, softmax_scale: float, out, lse, workspace, logits, is_probe, temperature, min_p,
                    seed, step: int, row_active, token_out, kept_count, trie: "Trie", eos_token: int,
                    max_len: int, state, dev_status=None, stream=None) -> None:
    """One whole decode step: attention, then the gated sample head (see the C header)."""
    import torch
    n = _attn_sizes(shape)
    dtype = _logits_dtype(logits)
    rows, vocab = logits.shape
    if rows != n["rows"]:
        raise ValueError(f"logits has {rows} rows, the attention shape {n['rows']}")
    ws_bytes = workspace.numel() * workspace.element_size() if isinstance(workspace, torch.Tensor) else 0
    _check(_call(load_library().rgd_decode_step,
        ctypes.byref(shape), _ptr(q, "q", torch.bfloat16, numel=n["q"]),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=n["kv"]), _ptr(v_pages, "v_pages", torch.bfloat16, numel=n["kv"]),
        _ptr(prompt_block_table, "prompt_block_table", torch.int32, numel=n["pbt"]),
        _ptr(prompt_len, "prompt_len", torch.int32, numel=n["plen"]),
        _ptr(suffix_block_table, "suffix_block_table", torch.int32, numel=n["sbt"]),
        _ptr(suffix_len, "suffix_len", torch.int32, numel=n["rows"]), float(softmax_scale),
        _ptr(out, "out", torch.bfloat16, numel=n["q"]), _ptr(lse, "lse", torch.float32, optional=True, numel=n["lse"]),
        _ptr(workspace, "workspace"), ws_bytes, vocab, dtype, _ptr(logits, "logits"),
        _ptr(is_probe, "is_probe", torch.uint8, optional=True, numel=rows),
        _ptr(temperature, "temperature", torch.float32, numel=rows), _ptr(min_p, "min_p", torch.float32, numel=rows),
        _ptr(seed, "seed", (torch.int64, torch.uint64), numel=rows), int(step) & 0xFFFFFFFFFFFFFFFF,
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows),
        _ptr(token_out, "token_out", torch.int32, numel=rows),
        _ptr(kept_count, "kept_count", torch.int32, optional=True, numel=rows),
        trie.handle, int(eos_token), int(max_len), _state_ptr(state, shape.num_groups),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


class Trie:
    """Owner of an ``rgd_trie`` handle built from host token sequences."""

    def __init__(self, sequences, min_confirm: int = 2):
        import numpy as np
        lib = load_library()
        seqs = [np.asarray(s, dtype=np.int32).reshape(-1) for s in sequences]
        toks = np.concatenate(seqs) if seqs else np.zeros(1, np.int32)
        offs = np.zeros(len(seqs) + 1, dtype=np.int64)
        for i, s in enumerate(seqs):
            offs[i + 1] = offs[i] + s.size
        toks = np.ascontiguousarray(toks)
        h = _P()
        _check(lib.rgd_trie_create(toks.ctypes.data, offs.ctypes.data, len(seqs), int(min_confirm),
                                   ctypes.byref(h)))
        self.handle = h
        self._lib = lib

    def info(self):
        n, e = _I32(), _I32()
        _check(self._lib.rgd_trie_info(self.handle, ctypes.byref(n), ctypes.byref(e)))
        return n.value, e.value

    def close(self):
        if getattr(self, "handle", None):
            self._lib.rgd_trie_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rgd_trie_create(sequences, min_confirm: int = 2) -> Trie:
    return Trie(sequences, min_confirm)


def _state_ptr(state, groups: int) -> Optional[int]:
    """A gate-state buffer must hold ``groups`` states of GATE_STATE_BYTES each."""
    import torch
    return _ptr(state, "state", torch.uint8, numel=max(int(groups), 0) * GATE_STATE_BYTES)


def rgd_gate_state_init(state, groups: int, stream=None) -> None:
    _check(_call(load_library().rgd_gate_state_init, _state_ptr(state, groups), int(groups), _stream(stream)))


def rgd_probe_gate(trie: Trie, groups: int, rows_per_group: int, probe_tokens, n_tokens: int,
                   token_stride: int, eos_token: int, max_len: int, state, row_active=None,
                   dev_status=None, stream=None) -> None:
    import torch
    G, rpg = int(groups), int(rows_per_group)
    tok_n = (G - 1) * int(token_stride) + int(n_tokens) if G > 0 else 0
    _check(_call(load_library().rgd_probe_gate,
        trie.handle, G, rpg, _ptr(probe_tokens, "probe_tokens", torch.int32, numel=tok_n),
        int(n_tokens), int(token_stride), int(eos_token), int(max_len), _state_ptr(state, G),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=G * rpg),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_residual_precheck(h, w, bias: float, theta: float, rows_per_group: int, state, row_active=None,
                          prob_out=None, dev_status=None, stream=None) -> None:
    import torch
    if h.dim() != 2:
        raise ValueError("h must be [groups, d]")
    dtype = {torch.float32: RGD_F32, torch.bfloat16: RGD_BF16}.get(h.dtype)
    if dtype is None:
        raise TypeError("h must be float32 or bfloat16")
    groups, d = h.shape
    rpg = int(rows_per_group)
    _check(_call(load_library().rgd_residual_precheck,
        int(groups), int(d), dtype, _ptr(h, "h"), _ptr(w, "w", torch.float32, numel=d), float(bias), float(theta),
        rpg, _ptr(prob_out, "prob_out", torch.float32, optional=True, numel=groups), _state_ptr(state, groups),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=groups * rpg),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_soft_gate(trie: Trie, groups: int, rows_per_group: int, logits, row_stride: int, top_k: int, rho: float,
                  c: int, eos_token: int, max_len: int, state, token_out, row_active=None, mass_out=None,
                  dev_status=None, stream=None) -> None:
    """``logits`` is the step's [rows, vocab] tensor (or any tensor whose rows
    g * row_stride / vocab hold group g's probe logits)."""
    import torch
    dtype = {torch.float32: RGD_F32, torch.bfloat16: RGD_BF16}.get(logits.dtype)
    if dtype is None:
        raise TypeError("logits must be float32 or bfloat16")
    vocab = logits.shape[-1]
    G, rpg = int(groups), int(rows_per_group)
    log_n = (G - 1) * int(row_stride) + int(vocab) if G > 0 else 0
    _check(_call(load_library().rgd_soft_gate,
        trie.handle, G, rpg, int(vocab), dtype, _ptr(logits, "logits", numel=log_n), int(row_stride),
        int(top_k), float(rho), int(c), int(eos_token), int(max_len), _state_ptr(state, G),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=G * rpg),
        _ptr(token_out, "token_out", torch.int32, numel=G),
        _ptr(mass_out, "mass_out", torch.float32, optional=True, numel=G),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


_DTYPE = None  # torch dtype -> RGD_F32 / RGD_BF16, once torch is needed


def _dtype_of(t, name: str) -> int:
    global _DTYPE
    if _DTYPE is None:
        import torch
        _DTYPE = {torch.float32: RGD_F32, torch.bfloat16: RGD_BF16}
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16")
    return code


def rgd_verify_draft_workspace_size(rows: int, max_draft: int) -> int:
    n = load_library().rgd_verify_draft_workspace_size(int(rows), int(max_draft))
    if n == 0:
        raise RgdError(RGD_ERR_INVALID_ARG, load_library().rgd_last_error_string().decode())
    return int(n)


def _bytes_of(workspace) -> int:
    return workspace.numel() * workspace.element_size() if hasattr(workspace, "numel") else 0


def rgd_verify_draft(target_logits, draft_logits, draft_tokens, n_draft, is_probe, temperature, min_p, accept_u, draw_u,
                     row_active, token_out, accepted_out, accept_prob, workspace, vocab: Optional[int] = None,
                     dev_status=None, stream=None) -> None:
    """``target_logits`` [rows, max_draft + 1, W] and ``draft_logits`` [rows, max_draft, W'] (or None: certain
    drafts), of which the first ``vocab`` of every row are logits (default: W)."""
    import torch
    if target_logits.dim() != 3 or target_logits.shape[1] < 1:
        raise ValueError("target_logits must be [rows, max_draft + 1, vocab]")
    rows, positions, width = target_logits.shape
    draft = positions - 1
    dtype = _dtype_of(target_logits, "target_logits")
    draft_width = width
    if draft_logits is not None:
        if draft_logits.dim() != 3 or draft_logits.shape[0] != rows or draft_logits.shape[1] != draft:
            raise ValueError("draft_logits must be [rows, max_draft, vocab]")
        draft_width = draft_logits.shape[2]
    i32, f32, u8 = torch.int32, torch.float32, torch.uint8
    _check(_call(load_library().rgd_verify_draft,
        rows, draft, width if vocab is None else int(vocab), dtype, _ptr(target_logits, "target_logits"), width,
        _ptr(draft_logits, "draft_logits", target_logits.dtype, optional=True), draft_width,
        _ptr(draft_tokens, "draft_tokens", i32, optional=draft == 0, numel=rows * draft),
        _ptr(n_draft, "n_draft", i32, optional=True, numel=rows),
        _ptr(is_probe, "is_probe", u8, optional=True, numel=rows),
        _ptr(temperature, "temperature", f32, numel=rows), _ptr(min_p, "min_p", f32, numel=rows),
        _ptr(accept_u, "accept_u", f32, optional=draft == 0, numel=rows * draft),
        _ptr(draw_u, "draw_u", f32, numel=rows), _ptr(row_active, "row_active", u8, optional=True, numel=rows),
        _ptr(token_out, "token_out", i32, numel=rows * positions), _ptr(accepted_out, "accepted_out", i32, numel=rows),
        _ptr(accept_prob, "accept_prob", f32, optional=True, numel=rows * draft),
        _ptr(workspace, "workspace"), _bytes_of(workspace),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def rgd_w4_matvec(x, weights, scales, zeros, group_size: int, y, dev_status=None, stream=None) -> None:
    """``y`` [m, W >= n] gets ``x`` [m, k] times the 4-bit ``weights`` [n, ceil(k / 2)] in its first n columns."""
    import torch
    if x.dim() != 2 or weights.dim() != 2 or y.dim() != 2:
        raise ValueError("x must be [m, k], weights [n, ceil(k / 2)] and y [m, n]")
    m, k = x.shape
    n, group = weights.shape[0], int(group_size)
    if weights.shape[1] != (k + 1) // 2:
        raise ValueError(f"weights holds rows of {weights.shape[1]} bytes, {k} weights take {(k + 1) // 2}")
    if y.shape[0] != m or y.shape[1] < n:
        raise ValueError(f"y must be [{m}, {n}] (or wider)")
    groups = -(-k // group) if group > 0 else 0
    _check(_call(load_library().rgd_w4_matvec,
        m, n, k, group, _ptr(x, "x", torch.bfloat16), _ptr(weights, "weights", torch.uint8),
        _dtype_of(scales, "scales"), _ptr(scales, "scales", numel=n * groups),
        _ptr(zeros, "zeros", torch.uint8, optional=True, numel=n * groups), _dtype_of(y, "y"), _ptr(y, "y"),
        y.shape[1], _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_cache_workspace_size(shape: CacheShape, rows: int) -> int:
    n = load_library().rgd_cache_workspace_size(ctypes.byref(shape), int(rows))
    if n == 0:
        raise RgdError(RGD_ERR_INVALID_ARG, load_library().rgd_last_error_string().decode())
    return int(n)


def _pool_numel(shape: CacheShape) -> int:
    pool = shape.num_pages * shape.num_kv_heads * shape.page_size * shape.head_dim
    return pool + max(shape.num_layers - 1, 0) * (shape.layer_stride or pool)


def _table_size(block_table, name: str = "block_table"):
    if block_table.dim() != 2:
        raise ValueError(f"{name} must be [rows, max_pages]")
    return block_table.shape


def rgd_cache_reserve(shape: CacheShape, block_table, length, n_new, row_active, page_refs, k_pages, v_pages, row_ok,
                      workspace, dev_status=None, stream=None) -> None:
    import torch
    rows, cols = _table_size(block_table)
    i32, u8, pool = torch.int32, torch.uint8, _pool_numel(shape)
    _check(_call(load_library().rgd_cache_reserve,
        ctypes.byref(shape), rows, cols, _ptr(block_table, "block_table", i32), _ptr(length, "length", i32, numel=rows),
        _ptr(n_new, "n_new", i32, numel=rows), _ptr(row_active, "row_active", u8, optional=True, numel=rows),
        _ptr(page_refs, "page_refs", i32, numel=shape.num_pages),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=pool), _ptr(v_pages, "v_pages", torch.bfloat16, numel=pool),
        _ptr(row_ok, "row_ok", u8, optional=True, numel=rows), _ptr(workspace, "workspace"), _bytes_of(workspace),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def _new_tokens(t, name: str, shape: CacheShape):
    """[rows, max_new, Hkv, D] whose last two dimensions are dense; its rows and tokens may be strided.  Returns the
    pointer and those two strides (0 where there is one element: its stride is never used)."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be a bfloat16 tensor")
    if t.dim() != 4 or t.shape[2] != shape.num_kv_heads or t.shape[3] != shape.head_dim:
        raise ValueError(f"{name} must be [rows, max_new, num_kv_heads, head_dim]")
    rows, tokens, heads, _ = t.shape
    by_row, by_token, by_head, by_element = t.stride()
    if t.numel() and (by_element != 1 or (by_head != shape.head_dim and heads > 1)):
        raise ValueError(f"{name}: heads and head_dim must be dense")
    strides = (by_row if rows > 1 else 0, by_token if tokens > 1 else 0)
    return (t.data_ptr() if t.is_cuda else _HostTensor(name)), strides


def rgd_cache_write(shape: CacheShape, layer: int, k_new, v_new, n_new, block_table, length, row_active, k_pages,
                    v_pages, dev_status=None, stream=None) -> None:
    """``k_new`` and ``v_new`` [rows, max_new, Hkv, D] have the same strides; views of a fused projection do."""
    import torch
    rows, cols = _table_size(block_table)
    (k, strides), (v, v_strides) = _new_tokens(k_new, "k_new", shape), _new_tokens(v_new, "v_new", shape)
    if k_new.shape[0] != rows or v_new.shape != k_new.shape or v_strides != strides:
        raise ValueError("k_new and v_new must have block_table's rows and the same shape and strides")
    i32, pool = torch.int32, _pool_numel(shape)
    _check(_call(load_library().rgd_cache_write,
        ctypes.byref(shape), int(layer), rows, k_new.shape[1], k, v, *strides,
        _ptr(n_new, "n_new", i32, numel=rows), cols, _ptr(block_table, "block_table", i32),
        _ptr(length, "length", i32, numel=rows), _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=pool), _ptr(v_pages, "v_pages", torch.bfloat16, numel=pool),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def rgd_cache_trim(block_table, length, row_active, page_refs, dev_status=None, stream=None) -> None:
    import torch
    rows, cols = _table_size(block_table)
    i32 = torch.int32
    _check(_call(load_library().rgd_cache_trim,
        rows, cols, page_refs.numel(), _ptr(block_table, "block_table", i32), _ptr(length, "length", i32, numel=rows),
        _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows), _ptr(page_refs, "page_refs", i32),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def rgd_cache_fork(parent, child, block_table, length, page_refs, dev_status=None, stream=None) -> None:
    import torch
    rows, cols = _table_size(block_table)
    i32, pairs = torch.int32, parent.numel()
    _check(_call(load_library().rgd_cache_fork,
        pairs, _ptr(parent, "parent", i32), _ptr(child, "child", i32, numel=pairs), rows, cols, page_refs.numel(),
        _ptr(block_table, "block_table", i32), _ptr(length, "length", i32, numel=rows),
        _ptr(page_refs, "page_refs", i32), _ptr(dev_status, "dev_status", i32, optional=True, numel=1),
        _stream(stream)))


def rgd_cache_copy(shape: CacheShape, src, dst, k_pages, v_pages, dev_status=None, stream=None) -> None:
    import torch
    i32, n, pool = torch.int32, src.numel(), _pool_numel(shape)
    _check(_call(load_library().rgd_cache_copy,
        ctypes.byref(shape), n, _ptr(src, "src", i32), _ptr(dst, "dst", i32, numel=n),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=pool), _ptr(v_pages, "v_pages", torch.bfloat16, numel=pool),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def rgd_cache_compact(shape: CacheShape, block_table_a, block_table_b, page_refs, k_pages, v_pages, num_live, workspace,
                      dev_status=None, stream=None) -> None:
    """Both tables may be None; every table of the pool has to be given."""
    import torch
    i32, pool = torch.int32, _pool_numel(shape)
    ra, ca = (0, 0) if block_table_a is None else _table_size(block_table_a, "block_table_a")
    rb, cb = (0, 0) if block_table_b is None else _table_size(block_table_b, "block_table_b")
    _check(_call(load_library().rgd_cache_compact,
        ctypes.byref(shape), ra, ca, _ptr(block_table_a, "block_table_a", i32, optional=True), rb, cb,
        _ptr(block_table_b, "block_table_b", i32, optional=True),
        _ptr(page_refs, "page_refs", i32, numel=shape.num_pages),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=pool), _ptr(v_pages, "v_pages", torch.bfloat16, numel=pool),
        _ptr(num_live, "num_live", i32, numel=1), _ptr(workspace, "workspace"), _bytes_of(workspace),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


_ROPE_SCALINGS = {"none": RGD_ROPE_PLAIN, "linear": RGD_ROPE_LINEAR, "base": RGD_ROPE_BASE, "bands": RGD_ROPE_BANDS,
                  "ramp": RGD_ROPE_RAMP}


def rgd_rope_frequencies(rotary_dim: int, base: float, scaling="none", factor: float = 1.0, trained_length: float = 0.0,
                         low: float = 1.0, high: Optional[float] = None):
    """Frequencies as 64-bit fractions of a turn (an int64 host tensor [rotary_dim / 2], to be moved to the device),
    and the magnitude for :class:`RopeShape`.  ``high`` defaults to 4 for "bands" and 32 for "ramp"."""
    import torch
    kind = _ROPE_SCALINGS.get(scaling, scaling)
    if not isinstance(kind, int):
        raise ValueError(f"scaling must be one of {sorted(_ROPE_SCALINGS)}")
    if high is None:
        high = 32.0 if kind == RGD_ROPE_RAMP else 4.0
    turns, magnitude = torch.zeros(max(int(rotary_dim), 0) // 2, dtype=torch.int64), ctypes.c_double()
    _check(load_library().rgd_rope_frequencies(int(rotary_dim), float(base), kind, float(factor), float(trained_length),
                                               float(low), float(high), turns.data_ptr(), ctypes.byref(magnitude)))
    return turns, magnitude.value


def _heads_of(t, name: str, lead: int, heads: int, dim: int, dtypes):
    """[..., heads, head_dim] with `lead` leading dimensions, whose last two are dense; None where there are no heads.
    Returns the pointer, the leading sizes and their strides (0 where there is one element: never used)."""
    if type(t) is _Tensor and t.dtype in dtypes and t.is_cuda:  # (as in _ptr: what passes every check returns here)
        shape, stride = t.shape, t.stride()
        if len(shape) == lead + 2 and shape[lead] == heads and shape[-1] == dim and stride[-1] == 1 and stride[-2] == dim:
            if lead == 1:
                return t.data_ptr(), (shape[0],), (stride[0] if shape[0] > 1 else 0,)
            return t.data_ptr(), (shape[0], shape[1]), (stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0)
    import torch
    if t is None and heads == 0:
        return None, None, (0,) * lead
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(str(d) for d in dtypes)}")
    if t.dim() != lead + 2 or t.shape[lead] != heads or t.shape[lead + 1] != dim:
        raise ValueError(f"{name} must have {lead} leading dimensions and then [{heads}, {dim}]")
    stride = t.stride()
    if t.numel() and ((stride[-1] != 1 and dim > 1) or (stride[-2] != dim and heads > 1)):
        raise ValueError(f"{name}: heads and head_dim must be dense")
    strides = tuple(stride[i] if t.shape[i] > 1 else 0 for i in range(lead))
    return (t.data_ptr() if t.is_cuda else _HostTensor(name)), tuple(t.shape[:lead]), strides


def _rope_weights(shape: RopeShape, q_weight, k_weight):
    """Pointers of the norms' weights and their dtype code."""
    weights = [w for w in (q_weight, k_weight) if w is not None]
    if not shape.norm or not weights:
        return None, None, RGD_F32
    code = _dtype_of(weights[0], "weights")
    return tuple(_ptr(w, name, weights[0].dtype, optional=True, numel=shape.head_dim)
                 for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight"))) + (code,)


def rgd_qk_rope(shape: RopeShape, q, k, positions, turns, q_weight, k_weight, q_out, k_out, dev_status=None,
                stream=None) -> None:
    """``q`` and ``q_out`` [tokens, Hq, D], ``k`` and ``k_out`` [tokens, Hk, D] (None where the shape has no such heads);
    tokens may be strided."""
    import torch
    first = q if shape.num_q_heads else k
    kinds = (torch.bfloat16, torch.float32) if first is None or not hasattr(first, "dtype") else (
        (first.dtype,) if first.dtype in (torch.bfloat16, torch.float32) else (torch.bfloat16, torch.float32))
    if not isinstance(positions, torch.Tensor):
        raise TypeError("positions must be a tensor")
    hq, hk, d, tokens = shape.num_q_heads, shape.num_k_heads, shape.head_dim, positions.numel()
    args = []
    for t, name, heads in ((q, "q", hq), (k, "k", hk), (q_out, "q_out", hq), (k_out, "k_out", hk)):
        ptr, lead, strides = _heads_of(t, name, 1, heads, d, kinds)
        if heads and lead != (tokens,):
            raise ValueError(f"{name} must have positions' {tokens} tokens")
        if name.endswith("_out") and tokens <= 1:
            strides = (heads * d,)
        args += [ptr, strides[0]]
    wq, wk, code = _rope_weights(shape, q_weight, k_weight)
    _check(_call(load_library().rgd_qk_rope,
        ctypes.byref(shape), tokens, RGD_F32 if kinds[0] is torch.float32 else RGD_BF16, *args[:4],
        _ptr(positions, "positions", torch.int32), _ptr(turns, "turns", torch.int64, optional=shape.rotary_dim == 0,
                                                        numel=shape.rotary_dim // 2),
        code, wq, wk, *args[4:], _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_qk_rope_cache(shape: RopeShape, cache: CacheShape, layer: int, q, k, v, first_position, turns, q_weight, k_weight,
                      n_new, block_table, length, row_active, q_out, k_pages, v_pages, dev_status=None,
                      stream=None) -> None:
    """``q`` [rows, max_new, Hq, D], ``k`` and ``v`` [rows, max_new, Hkv, D] with the same strides of rows and tokens (views
    of a fused projection); ``q_out`` [rows, max_new, Hq, D], contiguous."""
    import torch
    bf, i32, pool = (torch.bfloat16,), torch.int32, _pool_numel(cache)
    rows, cols = _table_size(block_table)
    (kp, lead, strides), (vp, v_lead, v_strides) = (
        _heads_of(t, name, 2, cache.num_kv_heads, cache.head_dim, bf) for t, name in ((k, "k"), (v, "v")))
    qp, q_lead, q_strides = _heads_of(q, "q", 2, shape.num_q_heads, shape.head_dim, bf)
    if lead[0] != rows or v_lead != lead or v_strides != strides or (q_lead is not None and (q_lead, q_strides) != (lead, strides)):
        raise ValueError("q, k and v must have block_table's rows and the same leading sizes and strides")
    wq, wk, code = _rope_weights(shape, q_weight, k_weight)
    _check(_call(load_library().rgd_qk_rope_cache,
        ctypes.byref(shape), ctypes.byref(cache), int(layer), rows, lead[1], qp, kp, vp, *strides,
        _ptr(first_position, "first_position", i32, optional=True, numel=rows),
        _ptr(turns, "turns", torch.int64, optional=shape.rotary_dim == 0, numel=shape.rotary_dim // 2), code, wq, wk,
        _ptr(n_new, "n_new", i32, numel=rows), cols, _ptr(block_table, "block_table", i32),
        _ptr(length, "length", i32, numel=rows), _ptr(row_active, "row_active", torch.uint8, optional=True, numel=rows),
        _ptr(q_out, "q_out", torch.bfloat16, optional=shape.num_q_heads == 0,
             numel=rows * lead[1] * shape.num_q_heads * shape.head_dim),
        _ptr(k_pages, "k_pages", torch.bfloat16, numel=pool), _ptr(v_pages, "v_pages", torch.bfloat16, numel=pool),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def _rows_of(t, name: str, dtypes):
    """[rows, columns] whose columns are dense: the pointer and the stride of its rows (that of one row: its width)."""
    if type(t) is _Tensor and t.dtype in dtypes and t.is_cuda:  # (as in _ptr)
        shape, stride = t.shape, t.stride()
        if len(shape) == 2 and stride[1] == 1:
            return t.data_ptr(), (stride[0] if shape[0] > 1 else max(stride[0], shape[1]))
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(str(d) for d in dtypes)}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    rows, cols = t.shape
    by_row, by_col = t.stride()
    if t.numel() and by_col != 1 and cols > 1:
        raise ValueError(f"{name}: columns must be dense")
    return (t.data_ptr() if t.is_cuda else _HostTensor(name)), (by_row if rows > 1 else max(by_row, cols))


def rgd_fp8_quantize(x, q, scales, block_rows: int = 1, dev_status=None, stream=None) -> None:
    """``x`` [rows, cols] in e4m3 into the first cols columns of ``q`` [rows, W >= cols] (float8_e4m3fn or uint8); rows of
    both may be strided."""
    import torch
    xp, x_stride = _rows_of(x, "x", (torch.float32, torch.bfloat16))
    qp, q_stride = _rows_of(q, "q", (torch.float8_e4m3fn, torch.uint8))
    rows, cols = x.shape
    if q.shape[0] != rows or q.shape[1] < cols:
        raise ValueError(f"q must be [{rows}, {cols}] (or wider)")
    each = int(block_rows)
    numel = -(-rows // each) * -(-cols // 128) if each > 0 else 0
    _check(_call(load_library().rgd_fp8_quantize,
        rows, cols, _dtype_of(x, "x"), xp, x_stride, each, qp, q_stride,
        _ptr(scales, "scales", torch.float32, numel=numel),
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_fp8_matmul(x, x_scales, weights, w_scales, y, k: Optional[int] = None, dev_status=None, stream=None) -> None:
    """``y`` [m, W >= n] gets ``x`` [m, K] times ``weights`` [n, K'] over their first ``k`` columns (default: K) in its first
    n columns.  e4m3 as float8_e4m3fn or uint8; rows of all three may be strided."""
    import torch
    bits = (torch.float8_e4m3fn, torch.uint8)
    xp, x_stride = _rows_of(x, "x", bits)
    wp, w_stride = _rows_of(weights, "weights", bits)
    yp, y_stride = _rows_of(y, "y", (torch.float32, torch.bfloat16))
    m, n = x.shape[0], weights.shape[0]
    k = x.shape[1] if k is None else int(k)
    if x.shape[1] < k or weights.shape[1] < k:
        raise ValueError(f"x and weights must have at least k = {k} columns")
    if y.shape[0] != m or y.shape[1] < n:
        raise ValueError(f"y must be [{m}, {n}] (or wider)")
    blocks = -(-k // 128)
    _check(_call(load_library().rgd_fp8_matmul,
        m, n, k, xp, x_stride, _ptr(x_scales, "x_scales", torch.float32, numel=m * blocks), wp, w_stride,
        _ptr(w_scales, "w_scales", torch.float32, numel=-(-n // 128) * blocks), _dtype_of(y, "y"), yp, y_stride,
        _ptr(dev_status, "dev_status", torch.int32, optional=True, numel=1), _stream(stream)))


def rgd_sample_top(logits, is_probe, temperature, top_k, top_p, min_p, draw_u, row_active, token_out, kept_count=None,
                   prob_out=None, vocab: Optional[int] = None, dev_status=None, stream=None) -> None:
    """``logits`` [rows, W], of which the first ``vocab`` of every row are logits (default: W); rows may be strided."""
    import torch
    lp, stride = _rows_of(logits, "logits", (torch.float32, torch.bfloat16))
    rows, width = logits.shape
    vocab = width if vocab is None else int(vocab)
    if vocab > width:
        raise ValueError(f"logits holds rows of {width}, the call needs {vocab}")
    i32, f32, u8 = torch.int32, torch.float32, torch.uint8
    _check(_call(load_library().rgd_sample_top,
        rows, vocab, _dtype_of(logits, "logits"), lp, stride, _ptr(is_probe, "is_probe", u8, optional=True, numel=rows),
        _ptr(temperature, "temperature", f32, numel=rows), _ptr(top_k, "top_k", i32, optional=True, numel=rows),
        _ptr(top_p, "top_p", f32, optional=True, numel=rows), _ptr(min_p, "min_p", f32, optional=True, numel=rows),
        _ptr(draw_u, "draw_u", f32, numel=rows), _ptr(row_active, "row_active", u8, optional=True, numel=rows),
        _ptr(token_out, "token_out", i32, numel=rows), _ptr(kept_count, "kept_count", i32, optional=True, numel=rows),
        _ptr(prob_out, "prob_out", f32, optional=True, numel=rows),
        _ptr(dev_status, "dev_status", i32, optional=True, numel=1), _stream(stream)))


def new_gate_state(groups: int, device="cuda"):
    """A device buffer holding ``groups`` gate states (uint8 [groups, 20])."""
    import torch
    return torch.empty((groups, GATE_STATE_BYTES), dtype=torch.uint8, device=device)


def decode_gate_state(buf) -> dict:
    """Host view of a gate-state buffer: dict of numpy arrays per field."""
    import numpy as np
    a = buf.cpu().numpy().reshape(-1, GATE_STATE_BYTES)
    i32 = a[:, :16].copy().view(np.int32).reshape(-1, 4)
    return {"node": i32[:, 0], "length": i32[:, 1], "steps": i32[:, 2], "decisive_step": i32[:, 3],
            "decision": a[:, 16].copy(), "confirmed": a[:, 17].copy(), "done": a[:, 18].copy()}
