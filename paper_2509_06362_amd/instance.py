"""Thin ctypes binding of the instance's operators (include/maaso_instance.h), in the manner of binding.py:
functions carry the names of the C entry points, device buffers are torch tensors, nothing is computed here.

KvPages and KvCache are views that a program makes once of the tensors it keeps; a call marshals its own
arguments only."""
from __future__ import annotations

import ctypes as C
from struct import Struct

from .binding import MaasoError, _check, _stream_handle, _t, load_library

MAASO_BF16, MAASO_FP16, MAASO_FP32, MAASO_E4M3 = 0, 1, 2, 3

BAD_PAGE, BAD_ROW, NO_PAGES, BAD_BOUND, BAD_TOKEN, BAD_POS = 1, 2, 4, 8, 16, 32

EXPORTS = (
    "maaso_instance_create", "maaso_instance_destroy", "maaso_instance_status", "maaso_kv_extend", "maaso_kv_fork",
    "maaso_kv_trim", "maaso_kv_compact", "maaso_kv_copy", "maaso_kv_append", "maaso_kv_attention", "maaso_logits_adjust",
)


class PagesArgs(C.Structure):
    _fields_ = [("n_pages", C.c_uint32), ("page_size", C.c_uint32), ("n_rows", C.c_uint32), ("width", C.c_uint32),
                ("refs", C.c_void_p), ("table", C.c_void_p), ("length", C.c_void_p)]


class CacheArgs(C.Structure):
    _fields_ = [("type", C.c_uint32), ("n_layers", C.c_uint32), ("n_pages", C.c_uint32), ("n_kv_heads", C.c_uint32),
                ("page_size", C.c_uint32), ("head_dim", C.c_uint32), ("page_stride", C.c_uint64),
                ("layer_stride", C.c_uint64), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p)]


class AppendArgs(C.Structure):
    _fields_ = [("type", C.c_uint32), ("n_tok", C.c_uint32), ("n_heads", C.c_uint32), ("rotary", C.c_uint32),
                ("interleaved", C.c_uint32), ("n_pos", C.c_uint32), ("eps", C.c_float), ("q", C.c_void_p),
                ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_uint64), ("k_stride", C.c_uint64),
                ("v_stride", C.c_uint64), ("q_out_stride", C.c_uint64), ("q_out", C.c_void_p),
                ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("cos_sin", C.c_void_p), ("pos", C.c_void_p),
                ("slot", C.c_void_p)]


class AttentionArgs(C.Structure):
    _fields_ = [("type", C.c_uint32), ("n", C.c_uint32), ("n_tok", C.c_uint32), ("n_heads", C.c_uint32),
                ("n_groups", C.c_uint32), ("max_q", C.c_uint32), ("max_len", C.c_uint32), ("max_shared", C.c_uint32),
                ("total_len", C.c_uint64), ("scale", C.c_float), ("q", C.c_void_p), ("out", C.c_void_p),
                ("q_stride", C.c_uint64), ("out_stride", C.c_uint64), ("lse", C.c_void_p), ("q_start", C.c_void_p),
                ("rows", C.c_void_p), ("group_start", C.c_void_p), ("shared", C.c_void_p)]


class LogitsArgs(C.Structure):
    _fields_ = [("type", C.c_uint32), ("out_type", C.c_uint32), ("n", C.c_uint32), ("vocab", C.c_uint32),
                ("stride", C.c_uint64), ("out_stride", C.c_uint64), ("logits", C.c_void_p), ("out", C.c_void_p),
                ("chosen", C.c_void_p), ("repetition", C.c_void_p), ("frequency", C.c_void_p),
                ("presence", C.c_void_p), ("temperature", C.c_void_p), ("history", C.c_void_p),
                ("history_start", C.c_void_p), ("n_history", C.c_uint32), ("n_bias", C.c_uint32),
                ("bias_token", C.c_void_p), ("bias_value", C.c_void_p), ("bias_start", C.c_void_p),
                ("mask", C.c_void_p), ("mask_row", C.c_void_p), ("n_mask", C.c_uint32)]


# The same structures, packed in one go: a ctypes structure of twenty fields takes longer to fill than a kernel to launch.
_codes = {C.c_uint32: "I", C.c_uint64: "Q", C.c_float: "f", C.c_void_p: "P"}


def _packer(structure):
    s = Struct("@" + "".join(_codes[kind] for _, kind in structure._fields_))
    if s.size > C.sizeof(structure):
        raise RuntimeError(f"{structure.__name__} is laid out otherwise than packed")
    pad = b"\0" * (C.sizeof(structure) - s.size)
    return (lambda *v: s.pack(*v) + pad) if pad else s.pack


_pack_append, _pack_attention, _pack_logits = _packer(AppendArgs), _packer(AttentionArgs), _packer(LogitsArgs)

_lib = None


def _library() -> C.CDLL:
    global _lib
    if _lib is None:
        lib = load_library()
        p, u = C.c_void_p, C.c_uint32
        lib.maaso_instance_create.argtypes = [C.c_int, C.c_uint64, C.POINTER(p)]
        lib.maaso_instance_destroy.argtypes = [p]
        lib.maaso_instance_destroy.restype = None
        lib.maaso_instance_status.argtypes = [p, C.POINTER(u)]
        lib.maaso_kv_extend.argtypes = [p, p, p, u, p, u, p, p, p, p]
        lib.maaso_kv_fork.argtypes = [p, p, p, p, u, p]
        lib.maaso_kv_trim.argtypes = [p, p, p, p, u, p]
        lib.maaso_kv_compact.argtypes = [p, p, p, p, p, p, p]
        lib.maaso_kv_copy.argtypes = [p, p, p, u, p]
        lib.maaso_kv_append.argtypes = [p, p, u, p, p]
        lib.maaso_kv_attention.argtypes = [p, p, u, p, p, p]
        lib.maaso_logits_adjust.argtypes = [p, p, p]
        missing = [n for n in EXPORTS if getattr(lib, n).argtypes is None]
        if missing:  # an undeclared signature would pass pointers as C ints
            raise RuntimeError(f"instance.py declares no argument types for {missing}")
        _lib = lib
    return _lib


_types = {}


def _type(t) -> int:
    """maaso_type of a tensor."""
    if not _types:
        torch = _t()
        _types.update({torch.bfloat16: MAASO_BF16, torch.float16: MAASO_FP16, torch.float32: MAASO_FP32,
                       torch.float8_e4m3fn: MAASO_E4M3})
    try:
        return _types[t.dtype]
    except KeyError:
        raise AssertionError(f"{t.dtype} is none of the library's types") from None


def _ptr(t, dtype, size=0):
    """Device pointer of a contiguous tensor of this type, with at least `size` elements; None -> 0.  A call has up to a dozen
    of these, and small calls take no longer than their marshalling: one condition where all is well."""
    if t is None:
        return 0
    if t.dtype is dtype and t.is_cuda and t.is_contiguous() and t.numel() >= size:
        return t.data_ptr()
    if not t.is_cuda or not t.is_contiguous():
        raise AssertionError("device buffers must be contiguous GPU tensors")
    if t.dtype != dtype:
        raise AssertionError(f"expected {dtype}, got {t.dtype}")
    raise AssertionError(f"expected {size} elements, got {t.numel()}")


def _heads(t, shape, dtype):
    """(pointer, elements between tokens) of [tokens, heads, dim], a token's heads side by side."""
    step, heads, side = t.stride() if t.dim() == 3 else (0, 0, 0)
    if t.dtype is dtype and t.is_cuda and t.shape == shape and side == 1 and (heads == shape[2] or shape[1] == 1):
        return t.data_ptr(), step
    if not t.is_cuda or t.dtype != dtype:
        raise AssertionError(f"expected a GPU tensor of {dtype}, got {t.dtype} on {t.device}")
    if t.shape != shape:
        raise AssertionError(f"expected {tuple(shape)}, got {tuple(t.shape)}")
    raise AssertionError("a token's heads must lie side by side")


class Instance:
    """Owns a maaso_instance*."""

    def __init__(self, handle: int, device: int):
        self.handle, self.device = handle, device

    def close(self) -> None:
        if self.handle:
            _library().maaso_instance_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class KvPages:
    """refs [pages], table [rows, width], length [rows]: int32 GPU tensors, changed in place by the calls."""

    def __init__(self, refs, table, length, page_size: int):
        i32 = _t().int32
        rows, width = table.shape
        self.refs, self.table, self.length, self.page_size = refs, table, length, int(page_size)
        self.args = PagesArgs(refs.numel(), int(page_size), rows, width, _ptr(refs, i32), _ptr(table, i32, rows * width),
                              _ptr(length, i32, rows))
        self.ref = C.byref(self.args)


class KvCache:
    """k [layers, pages, key heads, page size, head dim] and v [layers, pages, key heads, head dim, page size], of one
    type, each page whole; scales [key heads] (float32) for a cache of 8 bits."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        layers, pages, heads, page, dim = k.shape
        if tuple(v.shape) != (layers, pages, heads, dim, page) or v.dtype != k.dtype:
            raise AssertionError("v must be [layers, pages, key heads, head dim, page size], of k's type")
        if not (k.is_cuda and v.is_cuda and k[0, 0].is_contiguous() and v[0, 0].is_contiguous()):
            raise AssertionError("pages must be whole, on the GPU")
        if (layers > 1 and k.stride(0) != v.stride(0)) or (pages > 1 and k.stride(1) != v.stride(1)):
            raise AssertionError("k and v must have the same strides of layers and pages")
        f32 = _t().float32
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.heads, self.dim, self.dtype = heads, dim, k.dtype
        self.args = CacheArgs(_type(k), layers, pages, heads, page, dim, k.stride(1), k.stride(0), k.data_ptr(), v.data_ptr(),
                              _ptr(k_scale, f32, heads), _ptr(v_scale, f32, heads))
        self.ref = C.byref(self.args)


def maaso_instance_create(device: int = 0, workspace_bytes: int = 0) -> Instance:
    out = C.c_void_p()
    _check(_library().maaso_instance_create(int(device), int(workspace_bytes), C.byref(out)), "maaso_instance_create")
    return Instance(out.value, int(device))


def maaso_instance_status(inst: Instance) -> int:
    """Synchronises; returns and clears the MAASO_INST_* bits."""
    bits = C.c_uint32(0)
    rc = _library().maaso_instance_status(inst.handle, C.byref(bits))
    if rc not in (0, -1):
        raise MaasoError(rc, "maaso_instance_status")
    return int(bits.value)


def maaso_kv_extend(inst: Instance, pages: KvPages, *, rows, q_start, slot, pos=None, copies, stream=None) -> None:
    torch = _t()
    i32, n, n_tok = torch.int32, rows.numel(), slot.numel()
    _check(_library().maaso_kv_extend(inst.handle, pages.ref, _ptr(rows, i32), n, _ptr(q_start, i32, n + 1), n_tok,
                                      _ptr(slot, torch.int64), _ptr(pos, i32, n_tok), _ptr(copies, i32, 2 * n),
                                      _stream_handle(stream)), "maaso_kv_extend")


def maaso_kv_fork(inst: Instance, pages: KvPages, *, parents, children, stream=None) -> None:
    i32, n = _t().int32, children.numel()
    _check(_library().maaso_kv_fork(inst.handle, pages.ref, _ptr(parents, i32, n), _ptr(children, i32), n,
                                    _stream_handle(stream)), "maaso_kv_fork")


def maaso_kv_trim(inst: Instance, pages: KvPages, *, rows, keep, stream=None) -> None:
    i32, n = _t().int32, rows.numel()
    _check(_library().maaso_kv_trim(inst.handle, pages.ref, _ptr(rows, i32), _ptr(keep, i32, n), n,
                                    _stream_handle(stream)), "maaso_kv_trim")


def maaso_kv_compact(inst: Instance, pages: KvPages, *, refs_out, table_out, moves, n_live, stream=None) -> None:
    i32, a = _t().int32, pages.args
    _check(_library().maaso_kv_compact(inst.handle, pages.ref, _ptr(refs_out, i32, a.n_pages),
                                       _ptr(table_out, i32, a.n_rows * a.width), _ptr(moves, i32, 2 * (a.n_pages // 2)),
                                       _ptr(n_live, i32, 1), _stream_handle(stream)), "maaso_kv_compact")


def maaso_kv_copy(inst: Instance, cache: KvCache, *, pairs, stream=None) -> None:
    _check(_library().maaso_kv_copy(inst.handle, cache.ref, _ptr(pairs, _t().int32), pairs.numel() // 2,
                                    _stream_handle(stream)), "maaso_kv_copy")


def maaso_kv_append(inst: Instance, cache: KvCache, *, layer, q, k, v, q_out, slot, pos=None, cos_sin=None,
                    q_weight=None, k_weight=None, eps=1e-6, interleaved=False, stream=None) -> None:
    """q, q_out [tokens, heads, dim], k, v [tokens, key heads, dim]; cos_sin [positions, rotary] (float32)."""
    torch = _t()
    i32, dtype, shape, dim = torch.int32, q.dtype, q.shape, cache.dim
    if len(shape) != 3 or shape[2] != dim:
        raise AssertionError(f"expected [tokens, heads, {dim}], got {tuple(shape)}")
    tokens, heads, _ = shape
    keys = (tokens, cache.heads, dim)
    qp, qs = _heads(q, shape, dtype)
    op, os = _heads(q_out, shape, dtype)
    kp, ks = _heads(k, keys, dtype)
    vp, vs = _heads(v, keys, dtype)
    n_pos, rotary = cos_sin.shape if cos_sin is not None else (0, 0)
    a = _pack_append(_type(q), tokens, heads, rotary, 1 if interleaved else 0, n_pos, eps, qp, kp, vp, qs, ks, vs, os, op,
                     _ptr(q_weight, dtype, dim), _ptr(k_weight, dtype, dim), _ptr(cos_sin, torch.float32), _ptr(pos, i32, tokens),
                     _ptr(slot, torch.int64, tokens))
    _check(_library().maaso_kv_append(inst.handle, cache.ref, layer, a, _stream_handle(stream)), "maaso_kv_append")


def maaso_kv_attention(inst: Instance, cache: KvCache, pages: KvPages, *, layer, q, out, q_start, scale, max_q, max_len,
                       rows=None, group_start=None, shared=None, max_shared=0, total_len=0, lse=None, stream=None) -> None:
    """q, out [tokens, heads, dim]; lse [tokens, heads] (float32)."""
    torch = _t()
    i32, dtype, shape, dim = torch.int32, q.dtype, q.shape, cache.dim
    if len(shape) != 3 or shape[2] != dim:
        raise AssertionError(f"expected [tokens, heads, {dim}], got {tuple(shape)}")
    tokens, heads, _ = shape
    n = q_start.numel() - 1
    groups = 0 if group_start is None else group_start.numel() - 1
    qp, qs = _heads(q, shape, dtype)
    op, os = _heads(out, shape, dtype)
    a = _pack_attention(_type(q), n, tokens, heads, groups, int(max_q), int(max_len), int(max_shared), int(total_len), scale, qp, op,
                        qs, os, _ptr(lse, torch.float32, tokens * heads), _ptr(q_start, i32), _ptr(rows, i32, n),
                        _ptr(group_start, i32), _ptr(shared, i32, groups))
    _check(_library().maaso_kv_attention(inst.handle, cache.ref, layer, pages.ref, a, _stream_handle(stream)), "maaso_kv_attention")


def maaso_logits_adjust(inst: Instance, *, logits, out=None, chosen=None, repetition=None, frequency=None, presence=None,
                        temperature=None, history=None, history_start=None, bias_token=None, bias_value=None,
                        bias_start=None, mask=None, mask_row=None, stream=None) -> None:
    """logits, out [rows, vocabulary], a row's elements side by side; mask [masks, words] (int32)."""
    torch = _t()
    i32, f32 = torch.int32, torch.float32
    n, vocab = shape = logits.shape
    step, side = logits.stride()
    if side != 1 or not logits.is_cuda:
        raise AssertionError("a row's logits must lie side by side, on the GPU")
    kind, out_kind, out_step, out_at = _type(logits), MAASO_FP32, 0, 0
    if out is not None:
        if not out.is_cuda or out.shape != shape or out.stride(1) != 1:
            raise AssertionError("out must have the logits' shape, a row's elements side by side")
        out_kind, out_step, out_at = _type(out), out.stride(0), out.data_ptr()
    if mask is not None and mask.shape[1] != (vocab + 31) // 32:
        raise AssertionError("a mask has a bit for each token")
    n_bias = bias_token.numel() if bias_token is not None else 0
    a = _pack_logits(kind, out_kind, n, vocab, step, out_step, logits.data_ptr(), out_at, _ptr(chosen, i32, n),
                     _ptr(repetition, f32, n), _ptr(frequency, f32, n), _ptr(presence, f32, n), _ptr(temperature, f32, n),
                     _ptr(history, i32), _ptr(history_start, i32, n + 1), history.numel() if history is not None else 0, n_bias,
                     _ptr(bias_token, i32), _ptr(bias_value, f32, n_bias), _ptr(bias_start, i32, n + 1), _ptr(mask, i32),
                     _ptr(mask_row, i32, n), mask.shape[0] if mask is not None else 0)
    _check(_library().maaso_logits_adjust(inst.handle, a, _stream_handle(stream)), "maaso_logits_adjust")
