"""Python binding of libwsr_step: the entry points of include/wsr_step.h under the same names, reachable from
`paper_2608_12114_amd.wsr` too.

Argument marshalling only, as in wsr.py: structures are filled from keywords (pointers as integers, or
objects with a `data_ptr()`; fields left out are 0 or null) and hold no references, so the caller keeps the
tensors alive while they are used.
"""
from __future__ import annotations

import ctypes
import os

from .wsr import WSR_OK, WsrError, _HERE, _ptr, _stream

LIB_PATH = os.path.join(_HERE, "libwsr_step.so")

WSR_NORM_RMS, WSR_NORM_LAYER = range(2)
WSR_BLOCK_POST = 1

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "from the repository root")

_vp, _sz, _i64, _i32, _f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int32, ctypes.c_float


class wsr_block(ctypes.Structure):
    _fields_ = [("kind", _i32), ("fmt", _i32), ("flags", _i32), ("eps", _f32), ("res_scale", _f32), ("reserved", _i32),
                ("n_tokens", _i64), ("d", _i64), ("y", _vp), ("y_tok_stride", _i64), ("post_w", _vp), ("post_b", _vp),
                ("gate", _vp), ("gate_tok_stride", _i64), ("h", _vp), ("h_tok_stride", _i64), ("h_out", _vp),
                ("h_out_tok_stride", _i64), ("pre_w", _vp), ("pre_b", _vp), ("x", _vp), ("x_tok_stride", _i64)]


class wsr_lora(ctypes.Structure):
    _fields_ = [("fmt", _i32), ("rank", _i32), ("M", _i64), ("K", _i64), ("a", _vp), ("a_stride", _i64), ("b", _vp),
                ("b_stride", _i64), ("x", _vp), ("x_tok_stride", _i64), ("y0", _vp), ("y0_tok_stride", _i64), ("y", _vp),
                ("y_tok_stride", _i64)]


class wsr_attn(ctypes.Structure):
    _fields_ = [("fmt", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("n_seqs", _i32),
                ("n_tokens", _i32), ("scale", _f32), ("reserved", _i32), ("q", _vp), ("q_tok_stride", _i64),
                ("q_head_stride", _i64), ("k_prefix", _vp), ("v_prefix", _vp), ("prefix_len", _i64),
                ("prefix_tok_stride", _i64), ("prefix_head_stride", _i64), ("k", _vp), ("v", _vp), ("max_len", _i64),
                ("kv_seq_stride", _i64), ("kv_tok_stride", _i64), ("kv_head_stride", _i64), ("starts", _vp), ("lens", _vp),
                ("out", _vp), ("out_tok_stride", _i64), ("out_head_stride", _i64), ("lse", _vp)]


class wsr_verify(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("n_drafts", _i32), ("vocab", _i64), ("target", _vp), ("target_seq_stride", _i64),
                ("target_row_stride", _i64), ("draft", _vp), ("draft_seq_stride", _i64), ("draft_row_stride", _i64),
                ("tokens", _vp), ("counts", _vp), ("temperature", _vp), ("uniform", _vp), ("noise", _vp),
                ("noise_seq_stride", _i64), ("out", _vp), ("accepted", _vp), ("logp", _vp)]


_L = ctypes.CDLL(LIB_PATH)
_L.wsr_step_last_error.restype = ctypes.c_char_p
_L.wsr_step_last_error.argtypes = []
_L.wsr_block_norm.argtypes = [ctypes.POINTER(wsr_block), _vp]
_L.wsr_lora_workspace_bytes.argtypes = [ctypes.POINTER(wsr_lora), _i32, _i32]
_L.wsr_lora_workspace_bytes.restype = _sz
_L.wsr_lora_sweep.argtypes = [ctypes.POINTER(wsr_lora), _i32, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]
_L.wsr_attn_workspace_bytes.argtypes = [ctypes.POINTER(wsr_attn)]
_L.wsr_attn_workspace_bytes.restype = _sz
_L.wsr_prefix_attention.argtypes = [ctypes.POINTER(wsr_attn), _vp, _sz, _vp]
_L.wsr_verify_workspace_bytes.argtypes = [ctypes.POINTER(wsr_verify)]
_L.wsr_verify_workspace_bytes.restype = _sz
_L.wsr_verify_drafts.argtypes = [ctypes.POINTER(wsr_verify), _vp, _sz, _vp]
for _f in ("wsr_block_norm", "wsr_lora_sweep", "wsr_prefix_attention", "wsr_verify_drafts"):
    getattr(_L, _f).restype = ctypes.c_int


def step_lib() -> ctypes.CDLL:
    return _L


def wsr_step_last_error() -> str:
    return _L.wsr_step_last_error().decode()


def _check(st: int) -> None:
    if st != WSR_OK:
        raise WsrError(st, wsr_step_last_error())


def _fill(cls, fields: dict):
    pointers = {n for n, t in cls._fields_ if t is _vp}
    return cls(**{n: _ptr(v) if n in pointers else v for n, v in fields.items()})


def make_block(**fields) -> wsr_block:
    """A block's structure from keywords (res_scale 1 and eps 1e-5 where left out)."""
    return _fill(wsr_block, {"res_scale": 1.0, "eps": 1e-5, **fields})


def make_loras(specs) -> ctypes.Array:
    """specs: iterable of dicts, one per projection, with the fields of wsr_lora."""
    specs = list(specs)
    arr = (wsr_lora * max(1, len(specs)))(*[_fill(wsr_lora, s) for s in specs])
    arr._n = len(specs)
    return arr


def make_attn(**fields) -> wsr_attn:
    return _fill(wsr_attn, fields)


def make_verify(**fields) -> wsr_verify:
    return _fill(wsr_verify, fields)


def wsr_block_norm(block: wsr_block, stream=None) -> None:
    _check(_L.wsr_block_norm(block, _stream(stream)))


def wsr_lora_workspace_bytes(mods, n_tokens: int) -> int:
    return _L.wsr_lora_workspace_bytes(mods, getattr(mods, "_n", len(mods)), n_tokens)


def wsr_lora_sweep(mods, n_tokens: int, adapter_of, n_adapters: int, ranks, scales, ws, ws_bytes: int, stream=None) -> None:
    _check(_L.wsr_lora_sweep(mods, getattr(mods, "_n", len(mods)), n_tokens, _ptr(adapter_of), n_adapters, _ptr(ranks),
                             _ptr(scales), _ptr(ws), ws_bytes, _stream(stream)))


def wsr_attn_workspace_bytes(attn: wsr_attn) -> int:
    return _L.wsr_attn_workspace_bytes(attn)


def wsr_prefix_attention(attn: wsr_attn, ws, ws_bytes: int, stream=None) -> None:
    _check(_L.wsr_prefix_attention(attn, _ptr(ws), ws_bytes, _stream(stream)))


def wsr_verify_workspace_bytes(verify: wsr_verify) -> int:
    return _L.wsr_verify_workspace_bytes(verify)


def wsr_verify_drafts(verify: wsr_verify, ws, ws_bytes: int, stream=None) -> None:
    _check(_L.wsr_verify_drafts(verify, _ptr(ws), ws_bytes, _stream(stream)))
