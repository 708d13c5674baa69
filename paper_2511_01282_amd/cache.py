"""ctypes binding of what a cache goes through around the steps (include/respec_cache.h).

Argument marshalling only: rotary positions (``RotaryPlan``), and the caches of a model's layers whose accepted rows
are kept and whose pages are copied (``CacheLayers``).  Filling an 8-bit cache and attending to it are
``prompt.ChunkPlan.append_q8`` and ``attend_q8``.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from .binding import BF16, F32, OK, VerifyError
from .prompt import _E4M3, _E8M0, _I32, _I64, _P, PagedCache, _Plan, lib as _prompt_lib

HALF, INTERLEAVED = 0, 1
EXPORTS = ("respec_rotary_create", "respec_rotary_destroy", "respec_rotary", "respec_chunk_append_q8", "respec_chunk_attn_q8",
           "respec_cache_keep", "respec_cache_copy")
_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}


class RotaryShape(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "rotary_dim", "layout", "dtype", "max_tokens")] + [
        ("amplitude", ctypes.c_float)]


class RotaryArgs(ctypes.Structure):
    _fields_ = [("tokens", _I32), ("positions", _P), ("batch", _I32), ("new_off", _P), ("kv_len", _P),
                ("q", _P), ("q_token_stride", _I64), ("q_head_stride", _I64),
                ("q_out", _P), ("q_out_token_stride", _I64), ("q_out_head_stride", _I64),
                ("k", _P), ("k_token_stride", _I64), ("k_head_stride", _I64),
                ("k_out", _P), ("k_out_token_stride", _I64), ("k_out_head_stride", _I64), ("seq_status", _P)]


class KeepArgs(ctypes.Structure):
    _fields_ = [("batch", _I32), ("n_layers", _I32), ("n_kv_heads", _I32), ("head_dim", _I32), ("dtype", _I32),
                ("cache", PagedCache), ("layer_stride", _I64), ("kv_len", _P), ("path", _P), ("path_width", _I32),
                ("path_stride", _I64), ("acc_len", _P), ("kv_len_out", _P), ("seq_status", _P)]


class PagePlane(ctypes.Structure):
    _fields_ = [("base", _P), ("page_stride", _I64), ("n_layers", _I32), ("layer_stride", _I64), ("heads", _I32),
                ("head_stride", _I64), ("rows", _I32), ("row_stride", _I64), ("row_bytes", _I64)]


class CopyArgs(ctypes.Structure):
    _fields_ = [("pairs", _I32), ("src", _P), ("dst", _P), ("n_pages", _I32), ("n_planes", _I32), ("planes", _P),
                ("status", _P)]


# the same as one call packs them (native alignment; ctypes takes twice as long to fill such structures)
_ROTARY = struct.Struct("@iPiPP" "PqqPqq" "PqqPqq" "P")
_KEEP = struct.Struct("@iiiii" "PPiiqqqPiq" "qPPiqPPP")
_COPY = struct.Struct("@iPPiiPP")

_READY = False


def lib() -> ctypes.CDLL:
    global _READY
    L = _prompt_lib()
    if not _READY:
        for name, args in (("respec_rotary_create", [_P, _P, _P]), ("respec_rotary", [_P, _P, _P]),
                           ("respec_cache_keep", [_P, _P]), ("respec_cache_copy", [_P, _P])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        L.respec_rotary_destroy.argtypes, L.respec_rotary_destroy.restype = [_P], None
        _READY = True
    return L


def frequencies(rotary_dim, base=10000.0, *, scaling=None, factor=1.0, original_len=None, low=1.0, high=4.0, fast=32.0,
                slow=1.0) -> list:
    """Radians per position of every pair of columns, base^(-2 i / rotary_dim), for contexts ``factor`` times as long
    as those of ``original_len`` that the model was trained on:

    ``"linear"``  every one divided by the factor (positions interpolated)
    ``"bands"``   those of wavelengths above original_len / low divided, those below original_len / high kept, the others
                  blended by how many of their wavelengths original_len holds
    ``"ramp"``    pairs that turn over ``fast`` times in original_len kept, those that turn under ``slow`` times
                  divided, a linear ramp over the pairs between (YaRN, arXiv 2309.00071; its amplitude is
                  ``ramp_amplitude``)
    """
    w = [base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]
    if scaling is None:
        return w
    if scaling not in ("linear", "bands", "ramp"):
        raise ValueError(f"scaling: None, 'linear', 'bands' or 'ramp' expected, got {scaling!r}")
    if not factor >= 1:
        raise ValueError("factor: at least 1 expected")
    if scaling == "linear":
        return [x / factor for x in w]
    if not original_len or original_len < 1:
        raise ValueError("original_len: the length that the model was trained on expected")
    if scaling == "bands":
        if not 0 < low < high:
            raise ValueError("0 < low < high expected")
        keep = [min(1.0, max(0.0, (original_len * x / (2 * math.pi) - low) / (high - low))) for x in w]
    else:
        if not 0 < slow < fast or not base > 1:
            raise ValueError("0 < slow < fast and base > 1 expected")
        at = [rotary_dim * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (fast, slow)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rotary_dim - 1)
        keep = [1.0 - min(1.0, max(0.0, (i - first) / max(last - first, 1e-3))) for i in range(len(w))]
    return [x * k + x / factor * (1 - k) for x, k in zip(w, keep)]


_frequencies = frequencies


def ramp_amplitude(factor) -> float:
    """What the ramp's scaling multiplies cosines and sines by."""
    return 0.1 * math.log(factor) + 1.0


class RotaryPlan(_Plan):
    """A respec_rotary plan: the model's heads, its pairs of columns and their frequencies (radians per position)."""

    def __init__(self, *, n_q_heads, n_kv_heads, head_dim, dtype, rotary_dim=None, layout=HALF, frequencies=None, base=10000.0,
                 amplitude=1.0, max_tokens=1 << 24, device="cuda"):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if frequencies is None:
            frequencies = _frequencies(max(rotary_dim, 1), base)
        if len(frequencies) != rotary_dim // 2:
            raise ValueError(f"frequencies: one for each of {rotary_dim // 2} pairs expected, got {len(frequencies)}")
        if not ctypes.c_float(amplitude).value > 0:   # (0 would mean 1)
            raise ValueError("amplitude: a positive number expected, in float32, too")
        w = (ctypes.c_double * max(len(frequencies), 1))(*frequencies)
        super().__init__("rotary", RotaryShape(n_q_heads, n_kv_heads, head_dim, rotary_dim, layout, dtype, max_tokens, amplitude),
                         device, None, w)

    @staticmethod
    def _lib() -> ctypes.CDLL:
        return lib()

    def _side(self, x, y, name, heads):
        """(tokens, address and strides of x, of y)."""
        if x is None or y is None:
            if x is not None or y is not None:
                raise ValueError(f"{name} and {name}_out: both or neither expected")
            return None, (0, 0, 0, 0, 0, 0)
        dims = (x.shape[0], heads, self.shape.head_dim)
        xp, st = self._rows(x, name, self.dtype, dims)
        yp, y_st = self._rows(y, name + "_out", self.dtype, dims)
        if xp == yp and st != y_st:
            raise ValueError(f"{name}_out is {name}, laid out differently")
        return dims[0], (xp, st[0], st[1], yp, y_st[0], y_st[1])

    def rotate(self, q, k, q_out, k_out, *, positions=None, new_off=None, kv_len=None, status=None, stream=None) -> None:
        """Enqueue respec_rotary: ``q`` [T][Hq][D] into ``q_out`` and ``k`` [T][Hkv][D] into ``k_out`` (each pair, or neither
        of it, given; an output may be its input, and overlaps nothing else), at ``positions`` [T] (negative: left alone), or at a chunk batch's,
        ``kv_len[b]`` + i for token ``new_off[b]`` + i."""
        s, i32 = self.shape, torch.int32
        tq, qs = self._side(q, q_out, "q", s.n_q_heads)
        tk, ks = self._side(k, k_out, "k", s.n_kv_heads)
        tokens = tk if tq is None else tq
        if tokens is None or (tk is not None and tk != tokens):
            raise ValueError("q and k: one of them, or as many tokens in both, expected")
        if positions is not None:
            if new_off is not None or kv_len is not None or status is not None:
                raise ValueError("positions, or new_off and kv_len (and their status), expected")
            a = _ROTARY.pack(tokens, self._flat(positions, "positions", i32, (tokens,)), 0, 0, 0, *qs, *ks, 0)
        else:
            if new_off is None or kv_len is None:
                raise ValueError("positions, or new_off and kv_len, expected")
            batch = kv_len.shape[0]
            a = _ROTARY.pack(tokens, 0, batch, self._flat(new_off, "new_off", i32, (batch + 1,)),
                             self._flat(kv_len, "kv_len", i32, (batch,)), *qs, *ks,
                             0 if status is None else self._flat(status, "status", i32, (batch,)))
        self._call(lib().respec_rotary, "respec_rotary", (a,), stream)


class CacheLayers:
    """The caches of a model's layers, [layers][pages][Hkv][page][D] (or one layer's, without the first dimension):
    ``k_pages`` and ``v_pages``, and for 8-bit caches ``k_scale`` and ``v_scale`` [layers][pages][Hkv][blocks].  The
    tensors are described to the library once; strides are any that respec_cache.h allows."""

    def __init__(self, k_pages, v_pages, k_scale=None, v_scale=None):
        lib()
        if (k_scale is None) != (v_scale is None):
            raise ValueError("k_scale and v_scale: both or neither expected")
        eight = k_scale is not None
        dtype = _E4M3 if eight else k_pages.dtype
        if not eight and dtype not in _DTYPE:
            raise ValueError(f"k_pages: float32 or bfloat16 values, or e4m3 ones with their scales, expected; got {dtype}")
        if k_pages.dim() not in (4, 5):
            raise ValueError(f"k_pages: [layers][pages][heads][rows][columns], or one layer's, expected; got {tuple(k_pages.shape)}")
        self.device, self.tensors = k_pages.device, [k_pages, v_pages] + ([k_scale, v_scale] if eight else [])
        self._index = self.device.index if self.device.type == "cuda" else -1
        one = k_pages.dim() == 4
        shape = ((1,) if one else ()) + tuple(k_pages.shape)
        planes = []
        for name, t in zip(("k_pages", "v_pages", "k_scale", "v_scale"), self.tensors):
            t = t[None] if one else t
            scale = name.endswith("scale")
            want = shape[:3] + t.shape[3:] if scale else shape
            if tuple(t.shape) != want or t.dim() != len(shape) - scale or t.dtype != (_E8M0 if scale else dtype) or t.device != self.device:
                raise ValueError(f"{name}: {_E8M0 if scale else dtype} {want} on {self.device} expected; got {t.dtype} "
                                 f"{tuple(t.shape)} on {t.device}")
            if 0 in t.shape:
                raise ValueError(f"{name}: no elements")
            if t.stride(-1) != 1 and t.shape[-1] > 1:
                raise ValueError(f"{name}: the last dimension contiguous expected; got strides {t.stride()}")
            es, st = t.element_size(), [0 if n == 1 else s for n, s in zip(t.shape, t.stride())]
            rows, row = (1, 0) if scale else (t.shape[3], st[3])
            planes.append(PagePlane(t.data_ptr(), st[1] * es, t.shape[0], st[0] * es, t.shape[2], st[2] * es, rows, row * es,
                                    t.shape[-1] * es))
        if eight and k_scale.shape != v_scale.shape:
            raise ValueError("k_scale and v_scale: of one shape expected")
        self._pages, self._n = (PagePlane * len(planes))(*planes), len(planes)
        self._keep, es = None, k_pages.element_size()
        if not eight and shape[4] in (64, 128):
            k, v = planes
            if [getattr(k, f) for f, _ in PagePlane._fields_[1:]] == [getattr(v, f) for f, _ in PagePlane._fields_[1:]]:
                self._keep = (shape[0], shape[2], shape[4], _DTYPE[dtype])
                self._cache = (k.base, v.base, shape[1], shape[3], k.page_stride // es, k.head_stride // es, k.row_stride // es)
                self._layer = k.layer_stride // es
        self.n_pages = shape[1]

    def _flat(self, t, name, shape):
        if t.shape != shape or t.dtype is not torch.int32 or t.get_device() != self._index or (t.stride(-1) != 1 and shape[-1] > 1) or (
                self._index < 0 and t.device != self.device):
            raise ValueError(f"{name}: {torch.int32} {tuple(shape)} on {self.device}, the last dimension contiguous, expected; got "
                             f"{t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}")
        return t.data_ptr()

    def _call(self, fn, name, args, stream):
        if stream is None:
            raw = torch._C._cuda_getCurrentRawStream(self._index)
        elif stream.device != self.device:
            raise ValueError(f"the stream is of {stream.device}, the cache of {self.device}")
        else:
            raw = stream.cuda_stream
        if torch.cuda.current_device() == self._index:
            status = fn(args, raw)
        else:
            with torch.cuda.device(self.device):
                status = fn(args, raw)
        if status != OK:
            raise VerifyError(status, name)

    def keep_rows(self, page_table, kv_len, path, acc_len, kv_len_out=None, *, status=None, stream=None) -> None:
        """Enqueue respec_cache_keep: the accepted rows of every sequence's verified tree (``path`` [B][width] and ``acc_len`` [B],
        as a verification step leaves them) move behind its ``kv_len`` rows, in every layer, and ``kv_len_out`` (memory of
        its own, not one of the call's other arrays) becomes its new length.  For caches of the step's types, float32 and bfloat16, K and V laid out alike."""
        if self._keep is None:
            raise ValueError("float32 or bfloat16 caches with heads of 64 or 128 columns, K and V laid out alike, expected")
        batch, width = page_table.shape
        if path.dim() != 2:
            raise ValueError(f"path: [sequences][nodes] expected; got {tuple(path.shape)}")
        table = self._flat(page_table, "page_table", (batch, width))
        steps = path.shape[1]
        a = _KEEP.pack(batch, *self._keep, *self._cache, table, width, page_table.stride(0), self._layer,
                       self._flat(kv_len, "kv_len", (batch,)), self._flat(path, "path", (batch, steps)), steps, path.stride(0),
                       self._flat(acc_len, "acc_len", (batch,)),
                       0 if kv_len_out is None else self._flat(kv_len_out, "kv_len_out", (batch,)),
                       0 if status is None else self._flat(status, "status", (batch,)))
        self._call(lib().respec_cache_keep, "respec_cache_keep", a, stream)

    def copy_pages(self, src, dst, *, status=None, stream=None) -> None:
        """Enqueue respec_cache_copy: page ``dst[i]`` becomes a copy of page ``src[i]`` (-1: none), values and scales, in every
        layer."""
        pairs = (src.shape[0],)
        a = _COPY.pack(pairs[0], self._flat(src, "src", pairs), self._flat(dst, "dst", pairs), self.n_pages, self._n,
                       ctypes.addressof(self._pages), 0 if status is None else self._flat(status, "status", pairs))
        self._call(lib().respec_cache_copy, "respec_cache_copy", a, stream)
