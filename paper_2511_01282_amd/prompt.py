"""ctypes binding of the prompt side of librespec_verify.so (include/respec_prompt.h).

Argument marshalling only: a paged cache filled and attended to by chunks of new
tokens (``ChunkPlan``; its 8-bit forms are of include/respec_cache.h), and the scores of given
tokens (``ScorePlan``).  Tensors live on the plan's device; strides are taken from the tensors,
the last dimension is contiguous.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from .binding import BF16, F32, OK, VerifyError, lib as _verify_lib

ERR_PAGE = 11
EXPORTS = ("respec_chunk_create", "respec_chunk_destroy", "respec_chunk_workspace_bytes", "respec_chunk_append",
           "respec_chunk_attn", "respec_score_create", "respec_score_destroy", "respec_score_workspace_bytes",
           "respec_score")
_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_TORCH = {F32: torch.float32, BF16: torch.bfloat16}
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


class ChunkShape(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "max_batch", "max_new",
                                    "max_kv_len")]


class PagedCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("n_pages", _I32), ("page_size", _I32), ("page_stride", _I64),
                ("head_stride", _I64), ("row_stride", _I64), ("page_table", _P), ("table_width", _I32),
                ("table_stride", _I64)]


class ChunkBatch(ctypes.Structure):
    _fields_ = [("batch", _I32), ("total_new", _I32), ("max_new_in_batch", _I32), ("max_kv_len_in_batch", _I32),
                ("new_off", _P), ("kv_len", _P), ("cache", PagedCache), ("seq_status", _P)]


class AppendArgs(ctypes.Structure):
    _fields_ = [("b", ChunkBatch), ("k_new", _P), ("v_new", _P), ("k_token_stride", _I64), ("k_head_stride", _I64),
                ("v_token_stride", _I64), ("v_head_stride", _I64)]


class AttnArgs(ctypes.Structure):
    _fields_ = [("b", ChunkBatch), ("q", _P), ("q_token_stride", _I64), ("q_head_stride", _I64), ("out", _P),
                ("out_token_stride", _I64), ("out_head_stride", _I64), ("scale", ctypes.c_float)]


class Q8Cache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("n_pages", _I32), ("page_size", _I32),
                ("scale_block", _I32), ("page_stride", _I64), ("head_stride", _I64), ("row_stride", _I64),
                ("scale_page_stride", _I64), ("scale_head_stride", _I64), ("page_table", _P), ("table_width", _I32),
                ("table_stride", _I64)]


class Q8Batch(ctypes.Structure):
    _fields_ = [("batch", _I32), ("total_new", _I32), ("max_new_in_batch", _I32), ("max_kv_len_in_batch", _I32),
                ("new_off", _P), ("kv_len", _P), ("cache", Q8Cache), ("seq_status", _P)]


class Q8AppendArgs(ctypes.Structure):
    _fields_ = [("b", Q8Batch), *AppendArgs._fields_[1:]]


class Q8AttnArgs(ctypes.Structure):
    _fields_ = [("b", Q8Batch), *AttnArgs._fields_[1:]]


# the same as one call packs them (native alignment; ctypes takes twice as long to fill such structures)
_Q8_BATCH = "iiiiPP" "PPPPiiiqqqqqPiq" "P"
_Q8_APPEND = struct.Struct("@" + _Q8_BATCH + "PPqqqq")
_Q8_ATTN = struct.Struct("@" + _Q8_BATCH + "PqqPqqf0P")


class ScoreShape(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("vocab", "dtype", "max_rows", "topk_out")]


class ScoreArgs(ctypes.Structure):
    _fields_ = [("rows", _I32), ("logits", _P), ("row_stride", _I64), ("token", _P), ("tok_logprob", _P),
                ("tok_rank", _P), ("lse", _P), ("entropy", _P), ("topk_id", _P), ("topk_logprob", _P)]


_READY = False


def lib() -> ctypes.CDLL:
    global _READY
    L = _verify_lib()
    if not _READY:
        for name, args in (("respec_chunk_create", [_P, _P]), ("respec_chunk_append", [_P, _P, _P]),
                           ("respec_chunk_attn", [_P, _P, _P, _P]), ("respec_chunk_append_q8", [_P, _P, _P]),
                           ("respec_chunk_attn_q8", [_P, _P, _P, _P]), ("respec_score_create", [_P, _P]),
                           ("respec_score", [_P, _P, _P, _P])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        for name in ("respec_chunk_destroy", "respec_score_destroy"):
            f = getattr(L, name)
            f.argtypes, f.restype = [_P], None
        for name in ("respec_chunk_workspace_bytes", "respec_score_workspace_bytes"):
            f = getattr(L, name)
            f.argtypes, f.restype = [_P], ctypes.c_size_t
        _READY = True
    return L


class _Plan:
    """A plan handle, its device and its workspace (of kinds that have one)."""

    def __init__(self, kind: str, shape, device, workspace, *more):
        self._h = None
        L = self._lib()
        self._destroy = getattr(L, f"respec_{kind}_destroy")
        h = ctypes.c_void_p()
        status = getattr(L, f"respec_{kind}_create")(ctypes.byref(shape), *more, ctypes.byref(h))
        if status != OK:
            raise VerifyError(status, f"respec_{kind}_create")
        self._h, self.shape = h, shape
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = _TORCH[shape.dtype]
        self._index = self.device.index if self.device.type == "cuda" else -1
        self._streams = None   # streams that torch's allocator knows the plan's own workspace to be used on
        size = getattr(L, f"respec_{kind}_workspace_bytes", None)
        if size is None:
            return
        self.workspace_bytes = int(size(h))
        if workspace is None:
            if self._index >= 0:
                self._streams = {torch._C._cuda_getCurrentRawStream(self._index)}
            workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
            self.workspace_ptr = workspace.data_ptr() + (-workspace.data_ptr()) % 256
        else:
            if workspace.device != self.device or workspace.numel() * workspace.element_size() < self.workspace_bytes:
                raise ValueError(f"the workspace holds {self.workspace_bytes} bytes on {self.device}")
            self.workspace_ptr = workspace.data_ptr()
        self._ws_buf = workspace

    @staticmethod
    def _lib() -> ctypes.CDLL:
        return lib()

    def close(self):
        if self._h:
            self._destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _refuse(self, t, name, dtype, shape):
        raise ValueError(f"{name}: {dtype} {tuple(shape)} on {self.device}, the last dimension contiguous (every one, of "
                         f"offsets, lengths, tokens and results), expected; got {t.dtype} {tuple(t.shape)}, strides "
                         f"{t.stride()}, on {t.device}")

    def _rows(self, t, name, dtype, shape):
        """Address and strides of a tensor of rows: the last dimension contiguous (where it has more than one), strides
        of dimensions of one element 0."""
        st = t.stride()
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index or (st[-1] != 1 and shape[-1] > 1) or (
                self._index < 0 and t.device != self.device):
            self._refuse(t, name, dtype, shape)
        if 1 in shape:
            st = [0 if n == 1 else s for n, s in zip(shape, st)]
        return t.data_ptr(), st

    def _flat(self, t, name, dtype, shape):
        """Address of a contiguous tensor."""
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index or not t.is_contiguous() or (
                self._index < 0 and t.device != self.device):
            self._refuse(t, name, dtype, shape)
        return t.data_ptr()

    def _call(self, fn, name, args, stream):
        if self._h is None:
            raise ValueError("the plan is closed")
        if stream is None:
            # (of torch's ways to the current stream the one that makes no Python object of it: 0.1 us, not 1.9)
            raw = torch._C._cuda_getCurrentRawStream(self._index)
        elif stream.device != self.device:
            raise ValueError(f"the stream is of {stream.device}, the plan of {self.device}")
        else:
            raw = stream.cuda_stream
        if self._streams is not None and raw not in self._streams:
            # a plan that is dropped while its call waits there: the workspace is nobody else's until the call is done
            self._ws_buf.record_stream(torch.cuda.current_stream(self.device) if stream is None else stream)
            self._streams.add(raw)
        if torch.cuda.current_device() == self._index:
            status = fn(self._h, *args, raw)
        else:
            with torch.cuda.device(self.device):
                status = fn(self._h, *args, raw)
        if status != OK:
            raise VerifyError(status, name)


def _scale(scale) -> float:
    """The scores' scale as float32; 0: the default."""
    scale_f = 0.0 if scale is None else ctypes.c_float(scale).value
    if scale is not None and not scale_f > 0:
        raise ValueError("scale: a positive number expected, in float32, too")
    return scale_f


class ChunkPlan(_Plan):
    """A respec_chunk plan plus its device workspace.

    Calls that may overlap (on several streams) need plans, or workspaces, of their own.  The plan may be dropped
    while its calls are under way, on whatever stream; a captured call, and a workspace of the caller's, need it, or
    theirs, for as long as they are used."""

    def __init__(self, *, n_q_heads, n_kv_heads, head_dim, dtype, max_batch, max_new, max_kv_len, device="cuda",
                 workspace=None):
        super().__init__("chunk", ChunkShape(n_q_heads, n_kv_heads, head_dim, dtype, max_batch, max_new, max_kv_len),
                         device, workspace)

    def _batch(self, k_pages, v_pages, page_table, new_off, kv_len, total_new, max_new, max_kv_len, status):
        s, i32 = self.shape, torch.int32
        n_pages, _, page, _ = k_pages.shape
        batch, width = page_table.shape
        dims = (n_pages, s.n_kv_heads, page, s.head_dim)
        k, st = self._rows(k_pages, "k_pages", self.dtype, dims)
        v, v_st = self._rows(v_pages, "v_pages", self.dtype, dims)
        if st != v_st:
            raise ValueError("k_pages and v_pages are laid out differently")
        table, t_st = self._rows(page_table, "page_table", i32, (batch, width))
        return ChunkBatch(batch, total_new, max_new, max_kv_len, self._flat(new_off, "new_off", i32, (batch + 1,)),
                          self._flat(kv_len, "kv_len", i32, (batch,)),
                          PagedCache(k, v, n_pages, page, st[0], st[1], st[2], table, width, t_st[0]),
                          None if status is None else self._flat(status, "status", i32, (batch,)))

    def append(self, k_new, v_new, k_pages, v_pages, page_table, new_off, kv_len, *, max_new_in_batch, status=None,
               max_kv_len_in_batch=None, stream=None) -> None:
        """Enqueue respec_chunk_append: rows ``k_new``, ``v_new`` [T][Hkv][D] of the new tokens into
        ``k_pages``, ``v_pages`` [pages][Hkv][page][D]."""
        s = self.shape
        dims = (k_new.shape[0], s.n_kv_heads, s.head_dim)
        k, k_st = self._rows(k_new, "k_new", self.dtype, dims)
        v, v_st = self._rows(v_new, "v_new", self.dtype, dims)
        b = self._batch(k_pages, v_pages, page_table, new_off, kv_len, dims[0], max_new_in_batch,
                        s.max_kv_len if max_kv_len_in_batch is None else max_kv_len_in_batch, status)
        a = AppendArgs(b, k, v, k_st[0], k_st[1], v_st[0], v_st[1])
        self._call(lib().respec_chunk_append, "respec_chunk_append", (ctypes.byref(a),), stream)

    def attend(self, q, k_pages, v_pages, page_table, new_off, kv_len, out, *, max_new_in_batch, max_kv_len_in_batch,
               scale=None, status=None, stream=None) -> None:
        """Enqueue respec_chunk_attn: ``out`` [T][Hq][D] for the queries ``q`` [T][Hq][D] of the new
        tokens; ``scale`` defaults to 1 / sqrt(D)."""
        s = self.shape
        dims = (q.shape[0], s.n_q_heads, s.head_dim)
        qp, q_st = self._rows(q, "q", self.dtype, dims)
        op, o_st = self._rows(out, "out", self.dtype, dims)
        scale_f = _scale(scale)
        b = self._batch(k_pages, v_pages, page_table, new_off, kv_len, dims[0], max_new_in_batch, max_kv_len_in_batch,
                        status)
        a = AttnArgs(b, qp, q_st[0], q_st[1], op, o_st[0], o_st[1], scale_f)
        self._call(lib().respec_chunk_attn, "respec_chunk_attn", (ctypes.byref(a), self.workspace_ptr), stream)


    def _batch_q8(self, k_pages, v_pages, k_scale, v_scale, page_table, new_off, kv_len, total_new, max_new, max_kv_len, status):
        """The fields of a respec_q8_batch."""
        s, i32, rows = self.shape, torch.int32, self._rows
        n_pages, _, page, _ = k_pages.shape
        batch, width = page_table.shape
        heads = s.n_kv_heads
        dims = (n_pages, heads, page, s.head_dim)
        k, st = rows(k_pages, "k_pages", _E4M3, dims)
        v, v_st = rows(v_pages, "v_pages", _E4M3, dims)
        blocks = k_scale.shape[-1] if k_scale.dim() == 3 else 0
        if blocks < 1 or page % blocks:
            raise ValueError(f"k_scale: [pages][heads][blocks of a page] expected, {page} rows a page in whole blocks; got "
                             f"{tuple(k_scale.shape)}")
        dims = (n_pages, heads, blocks)
        ks, s_st = rows(k_scale, "k_scale", _E8M0, dims)
        vs, vs_st = rows(v_scale, "v_scale", _E8M0, dims)
        # (the last dimension is contiguous, or of one element)
        if st[:3] != v_st[:3] or s_st[:2] != vs_st[:2]:
            raise ValueError("k_pages and v_pages, or their scales, are laid out differently")
        table, t_st = rows(page_table, "page_table", i32, (batch, width))
        return (batch, total_new, max_new, max_kv_len, self._flat(new_off, "new_off", i32, (batch + 1,)),
                self._flat(kv_len, "kv_len", i32, (batch,)), k, v, ks, vs, n_pages, page, page // blocks, st[0], st[1], st[2], s_st[0],
                s_st[1], table, width, t_st[0], 0 if status is None else self._flat(status, "status", i32, (batch,)))

    def append_q8(self, k_new, v_new, k_pages, v_pages, k_scale, v_scale, page_table, new_off, kv_len, *, max_new_in_batch,
                  status=None, max_kv_len_in_batch=None, stream=None) -> None:
        """Enqueue respec_chunk_append_q8: rows ``k_new``, ``v_new`` [T][Hkv][D] of the new tokens into the e4m3 values
        ``k_pages``, ``v_pages`` [pages][Hkv][page][D] with their blocks' scales ``k_scale``, ``v_scale``
        [pages][Hkv][blocks of a page] (float8_e8m0fnu)."""
        s = self.shape
        dims = (k_new.shape[0], s.n_kv_heads, s.head_dim)
        k, k_st = self._rows(k_new, "k_new", self.dtype, dims)
        v, v_st = self._rows(v_new, "v_new", self.dtype, dims)
        b = self._batch_q8(k_pages, v_pages, k_scale, v_scale, page_table, new_off, kv_len, dims[0], max_new_in_batch,
                           s.max_kv_len if max_kv_len_in_batch is None else max_kv_len_in_batch, status)
        a = _Q8_APPEND.pack(*b, k, v, k_st[0], k_st[1], v_st[0], v_st[1])
        self._call(lib().respec_chunk_append_q8, "respec_chunk_append_q8", (a,), stream)

    def attend_q8(self, q, k_pages, v_pages, k_scale, v_scale, page_table, new_off, kv_len, out, *, max_new_in_batch,
                  max_kv_len_in_batch, scale=None, status=None, stream=None) -> None:
        """Enqueue respec_chunk_attn_q8: ``attend`` over the 8-bit cache that ``append_q8`` fills."""
        s = self.shape
        dims = (q.shape[0], s.n_q_heads, s.head_dim)
        qp, q_st = self._rows(q, "q", self.dtype, dims)
        op, o_st = self._rows(out, "out", self.dtype, dims)
        scale_f = _scale(scale)
        b = self._batch_q8(k_pages, v_pages, k_scale, v_scale, page_table, new_off, kv_len, dims[0], max_new_in_batch,
                           max_kv_len_in_batch, status)
        a = _Q8_ATTN.pack(*b, qp, q_st[0], q_st[1], op, o_st[0], o_st[1], scale_f)
        self._call(lib().respec_chunk_attn_q8, "respec_chunk_attn_q8", (a, self.workspace_ptr), stream)


# outputs of a scoring call: type, and whether they hold the top alternatives' columns
SCORE_OUTPUTS = {"tok_logprob": (torch.float32, False), "tok_rank": (torch.int32, False), "lse": (torch.float32, False),
                 "entropy": (torch.float32, False), "topk_id": (torch.int32, True), "topk_logprob": (torch.float32, True)}


class ScorePlan(_Plan):
    """A respec_score plan plus its device workspace (one call at a time, as ``ChunkPlan``)."""

    def __init__(self, *, vocab, max_rows, topk_out=8, dtype=F32, device="cuda", workspace=None):
        super().__init__("score", ScoreShape(vocab, dtype, max_rows, topk_out), device, workspace)

    def score(self, logits, token, outputs: dict, *, stream=None) -> None:
        """Enqueue respec_score on ``logits`` [R][V] for the tokens ``token`` [R] (-1 or None: none).
        ``outputs``: any of ``SCORE_OUTPUTS`` (``alloc_score_outputs``); missing ones are not written."""
        s = self.shape
        rows = logits.shape[0]
        z, st = self._rows(logits, "logits", self.dtype, (rows, s.vocab))
        tok = None if token is None else self._flat(token, "token", torch.int32, (rows,))
        to = {}
        for name, t in outputs.items():
            dtype, wide = SCORE_OUTPUTS[name]
            to[name] = None if t is None else self._flat(t, name, dtype, (rows, s.topk_out) if wide else (rows,))
        a = ScoreArgs(rows, z, st[0], tok, **to)
        self._call(lib().respec_score, "respec_score", (ctypes.byref(a), self.workspace_ptr), stream)


def alloc_score_outputs(*, rows, topk_out, device="cuda") -> dict:
    """Output tensors of one scoring call."""
    return {name: torch.empty((rows, topk_out) if wide else (rows,), dtype=dtype, device=device)
            for name, (dtype, wide) in SCORE_OUTPUTS.items()}
