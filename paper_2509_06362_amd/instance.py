"""Thin binding of the instance's operators (include/maaso_instance.h), in the manner of binding.py: functions
carry the names of the C entry points, device buffers are torch tensors, nothing is computed here.

KvPages and KvCache are views that a program makes once of the tensors it keeps; a call marshals its own
arguments only.  A decode step's calls take microseconds, so their tensors are looked at and their structures
filled by a small native module (csrc/instance_marshal.cpp) and not by the interpreter: host time of one layer's
write of keys and values 9.7 us a call through ctypes, 4.0 so.  Without it, as without the library, a call raises."""
from __future__ import annotations

import ctypes as C

from .binding import MaasoError, _check, _t, load_library

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


# The three that follow are for callers of the C entry points: the calls below are filled in from the header itself.
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


_native = None


def _load_native():
    """The marshalling module, bound to the library's entry points."""
    global _native
    _t()  # (it needs torch's libraries)
    lib = _library()
    try:
        from . import _marshal
    except ImportError as e:
        raise RuntimeError(f"the marshalling module is missing ({e}): build it first "
                           "(python -m paper_2509_06362_amd.build); there is no fallback path") from e
    calls = (lib.maaso_kv_extend, lib.maaso_kv_fork, lib.maaso_kv_trim, lib.maaso_kv_compact, lib.maaso_kv_copy,
             lib.maaso_kv_append, lib.maaso_kv_attention, lib.maaso_logits_adjust)
    _marshal.bind(*(C.cast(f, C.c_void_p).value for f in calls))
    _native = _marshal
    return _marshal


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
    """Device pointer of a contiguous tensor of this type, with at least `size` elements; None -> NULL."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise AssertionError("device buffers must be contiguous GPU tensors")
    if t.dtype != dtype:
        raise AssertionError(f"expected {dtype}, got {t.dtype}")
    if t.numel() < size:
        raise AssertionError(f"expected {size} elements, got {t.numel()}")
    return t.data_ptr()


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
        self.at = C.addressof(self.args)


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
        self.at = C.addressof(self.args)


def maaso_instance_create(device: int = 0, workspace_bytes: int = 0) -> Instance:
    out = C.c_void_p()
    _check(_library().maaso_instance_create(int(device), int(workspace_bytes), C.byref(out)), "maaso_instance_create")
    return Instance(out.value, int(device))


def maaso_instance_status(inst: Instance) -> int:
    """Synchronises; returns and clears the MAASO_INST_* bits."""
    bits = C.c_uint32(0)
    rc = _library().maaso_instance_status(inst.handle, C.byref(bits))
    if rc not in (0, -1) or (rc == -1 and not bits.value):  # (INVALID_ARG with bits is what they are read by)
        raise MaasoError(rc, "maaso_instance_status")
    return int(bits.value)


def maaso_kv_extend(inst: Instance, pages: KvPages, *, rows, q_start, slot, pos=None, copies, stream=None) -> None:
    _check((_native or _load_native()).extend(inst.handle, pages.at, rows, q_start, slot, pos, copies, stream),
           "maaso_kv_extend")


def maaso_kv_fork(inst: Instance, pages: KvPages, *, parents, children, stream=None) -> None:
    _check((_native or _load_native()).fork(inst.handle, pages.at, parents, children, stream), "maaso_kv_fork")


def maaso_kv_trim(inst: Instance, pages: KvPages, *, rows, keep, stream=None) -> None:
    _check((_native or _load_native()).trim(inst.handle, pages.at, rows, keep, stream), "maaso_kv_trim")


def maaso_kv_compact(inst: Instance, pages: KvPages, *, refs_out, table_out, moves, n_live, stream=None) -> None:
    _check((_native or _load_native()).compact(inst.handle, pages.at, refs_out, table_out, moves, n_live, stream),
           "maaso_kv_compact")


def maaso_kv_copy(inst: Instance, cache: KvCache, *, pairs, stream=None) -> None:
    _check((_native or _load_native()).copy(inst.handle, cache.at, pairs, stream), "maaso_kv_copy")


def maaso_kv_append(inst: Instance, cache: KvCache, *, layer, q, k, v, q_out, slot, pos=None, cos_sin=None,
                    q_weight=None, k_weight=None, eps=1e-6, interleaved=False, stream=None) -> None:
    """q, q_out [tokens, heads, dim], k, v [tokens, key heads, dim]; cos_sin [positions, rotary] (float32)."""
    _check((_native or _load_native()).append(inst.handle, cache.at, layer, q, k, v, q_out, slot, pos, cos_sin, q_weight,
                                              k_weight, eps, interleaved, stream), "maaso_kv_append")


def maaso_kv_attention(inst: Instance, cache: KvCache, pages: KvPages, *, layer, q, out, q_start, scale, max_q, max_len,
                       rows=None, group_start=None, shared=None, max_shared=0, total_len=0, lse=None, stream=None) -> None:
    """q, out [tokens, heads, dim]; lse [tokens, heads] (float32)."""
    _check((_native or _load_native()).attention(inst.handle, cache.at, pages.at, layer, q, out, q_start, scale, max_q,
                                                 max_len, rows, group_start, shared, max_shared, total_len, lse, stream),
           "maaso_kv_attention")


def maaso_logits_adjust(inst: Instance, *, logits, out=None, chosen=None, repetition=None, frequency=None, presence=None,
                        temperature=None, history=None, history_start=None, bias_token=None, bias_value=None,
                        bias_start=None, mask=None, mask_row=None, stream=None) -> None:
    """logits, out [rows, vocabulary], a row's elements side by side; mask [masks, words] (int32)."""
    _check((_native or _load_native()).logits(inst.handle, logits, out, chosen, repetition, frequency, presence, temperature,
                                              history, history_start, bias_token, bias_value, bias_start, mask, mask_row,
                                              stream), "maaso_logits_adjust")
