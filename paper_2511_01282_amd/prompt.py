"""ctypes binding of the prompt side of librespec_verify.so (include/respec_prompt.h).

Argument marshalling only: a paged cache filled and attended to by chunks of new
tokens (``ChunkPlan``), and the scores of given tokens (``ScorePlan``).  Tensors live
on the plan's device; strides are taken from the tensors, the last dimension is
contiguous.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import BF16, F32, OK, VerifyError, lib as _verify_lib

ERR_PAGE = 11
EXPORTS = ("respec_chunk_create", "respec_chunk_destroy", "respec_chunk_workspace_bytes", "respec_chunk_append",
           "respec_chunk_attn", "respec_score_create", "respec_score_destroy", "respec_score_workspace_bytes",
           "respec_score")
_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_TORCH = {F32: torch.float32, BF16: torch.bfloat16}


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
                           ("respec_chunk_attn", [_P, _P, _P, _P]), ("respec_score_create", [_P, _P]),
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
    """A plan handle, its device and its workspace."""

    def __init__(self, kind: str, shape, device, workspace):
        self._h = None
        L = lib()
        self._destroy = getattr(L, f"respec_{kind}_destroy")
        h = ctypes.c_void_p()
        status = getattr(L, f"respec_{kind}_create")(ctypes.byref(shape), ctypes.byref(h))
        if status != OK:
            raise VerifyError(status, f"respec_{kind}_create")
        self._h, self.shape = h, shape
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = _TORCH[shape.dtype]
        self.workspace_bytes = int(getattr(L, f"respec_{kind}_workspace_bytes")(h))
        if workspace is None:
            workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
            self.workspace_ptr = workspace.data_ptr() + (-workspace.data_ptr()) % 256
        else:
            if workspace.device != self.device or workspace.numel() * workspace.element_size() < self.workspace_bytes:
                raise ValueError(f"the workspace holds {self.workspace_bytes} bytes on {self.device}")
            self.workspace_ptr = workspace.data_ptr()
        self._ws_buf = workspace

    def close(self):
        if self._h:
            self._destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _tensor(self, t, name, dtype, dims):
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the plan on {self.device}")
        if t.dtype != dtype or t.dim() != dims:
            raise ValueError(f"{name}: {dims} dimensions of {dtype} expected, got {tuple(t.shape)} of {t.dtype}")
        return t.data_ptr()

    def _rows(self, t, name, dtype, dims, shape):
        """Address and strides of a tensor of rows: the last dimension contiguous (where it has more than one)."""
        p = self._tensor(t, name, dtype, dims)
        if t.shape != shape:
            raise ValueError(f"{name}: {tuple(shape)} expected, got {tuple(t.shape)}")
        st = t.stride()
        if st[-1] != 1 and shape[-1] > 1:
            raise ValueError(f"{name}: the last dimension is not contiguous")
        return (p, *st[:-1])

    def _flat(self, t, name, dtype, shape):
        """Address of a contiguous tensor."""
        p = self._tensor(t, name, dtype, len(shape))
        if t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous {tuple(shape)} expected, got {tuple(t.shape)}")
        return p

    def _call(self, fn, name, args, stream, *more):
        if self._h is None:
            raise ValueError("the plan is closed")
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        elif stream.device != self.device:
            raise ValueError(f"the stream is of {stream.device}, the plan of {self.device}")
        if torch.cuda.current_device() == self.device.index:
            status = fn(self._h, ctypes.byref(args), *more, stream.cuda_stream)
        else:
            with torch.cuda.device(self.device):
                status = fn(self._h, ctypes.byref(args), *more, stream.cuda_stream)
        if status != OK:
            raise VerifyError(status, name)


class ChunkPlan(_Plan):
    """A respec_chunk plan plus its device workspace.

    Calls that may overlap (on several streams) need plans, or workspaces, of their own."""

    def __init__(self, *, n_q_heads, n_kv_heads, head_dim, dtype, max_batch, max_new, max_kv_len, device="cuda",
                 workspace=None):
        super().__init__("chunk", ChunkShape(n_q_heads, n_kv_heads, head_dim, dtype, max_batch, max_new, max_kv_len),
                         device, workspace)

    def _batch(self, k_pages, v_pages, page_table, new_off, kv_len, total_new, max_new, max_kv_len, status):
        s = self.shape
        n_pages, page = k_pages.shape[0], k_pages.shape[2]
        dims = (n_pages, s.n_kv_heads, page, s.head_dim)
        k, *strides = self._rows(k_pages, "k_pages", self.dtype, 4, dims)
        v, *v_strides = self._rows(v_pages, "v_pages", self.dtype, 4, dims)
        if strides != v_strides:
            raise ValueError("k_pages and v_pages are laid out differently")
        batch = kv_len.shape[0]
        table, stride = self._rows(page_table, "page_table", torch.int32, 2, (batch, page_table.shape[1]))
        return ChunkBatch(batch, total_new, max_new, max_kv_len,
                          self._flat(new_off, "new_off", torch.int32, (batch + 1,)),
                          self._flat(kv_len, "kv_len", torch.int32, (batch,)),
                          PagedCache(k, v, n_pages, page, *strides, table, page_table.shape[1], stride),
                          None if status is None else self._flat(status, "status", torch.int32, (batch,)))

    def append(self, k_new, v_new, k_pages, v_pages, page_table, new_off, kv_len, *, max_new_in_batch, status=None,
               max_kv_len_in_batch=None, stream=None) -> None:
        """Enqueue respec_chunk_append: rows ``k_new``, ``v_new`` [T][Hkv][D] of the new tokens into
        ``k_pages``, ``v_pages`` [pages][Hkv][page][D]."""
        s = self.shape
        dims = (k_new.shape[0], s.n_kv_heads, s.head_dim)
        k, *k_strides = self._rows(k_new, "k_new", self.dtype, 3, dims)
        v, *v_strides = self._rows(v_new, "v_new", self.dtype, 3, dims)
        b = self._batch(k_pages, v_pages, page_table, new_off, kv_len, dims[0], max_new_in_batch,
                        s.max_kv_len if max_kv_len_in_batch is None else max_kv_len_in_batch, status)
        self._call(lib().respec_chunk_append, "respec_chunk_append", AppendArgs(b, k, v, *k_strides, *v_strides), stream)

    def attend(self, q, k_pages, v_pages, page_table, new_off, kv_len, out, *, max_new_in_batch, max_kv_len_in_batch,
               scale=None, status=None, stream=None) -> None:
        """Enqueue respec_chunk_attn: ``out`` [T][Hq][D] for the queries ``q`` [T][Hq][D] of the new
        tokens; ``scale`` defaults to 1 / sqrt(D)."""
        s = self.shape
        dims = (q.shape[0], s.n_q_heads, s.head_dim)
        qp, *q_strides = self._rows(q, "q", self.dtype, 3, dims)
        op, *o_strides = self._rows(out, "out", self.dtype, 3, dims)
        if scale is not None and not scale > 0:
            raise ValueError("scale: a positive number expected")
        b = self._batch(k_pages, v_pages, page_table, new_off, kv_len, dims[0], max_new_in_batch, max_kv_len_in_batch,
                        status)
        self._call(lib().respec_chunk_attn, "respec_chunk_attn",
                   AttnArgs(b, qp, *q_strides, op, *o_strides, scale or 0.0), stream, self.workspace_ptr)


SCORE_OUTPUTS = ("tok_logprob", "tok_rank", "lse", "entropy", "topk_id", "topk_logprob")


class ScorePlan(_Plan):
    """A respec_score plan plus its device workspace (one call at a time, as ``ChunkPlan``)."""

    def __init__(self, *, vocab, max_rows, topk_out=8, dtype=F32, device="cuda", workspace=None):
        super().__init__("score", ScoreShape(vocab, dtype, max_rows, topk_out), device, workspace)

    def score(self, logits, token, outputs: dict, *, stream=None) -> None:
        """Enqueue respec_score on ``logits`` [R][V] for the tokens ``token`` [R] (-1 or None: none).
        ``outputs``: any of ``SCORE_OUTPUTS`` (``alloc_score_outputs``); missing ones are not written."""
        s = self.shape
        rows = logits.shape[0]
        z, stride = self._rows(logits, "logits", self.dtype, 2, (rows, s.vocab))
        a = ScoreArgs(rows, z, stride, None if token is None else self._flat(token, "token", torch.int32, (rows,)))
        for name, t in outputs.items():
            if name not in SCORE_OUTPUTS:
                raise ValueError(f"unknown output {name}")
            if t is not None:
                setattr(a, name, self._flat(t, name, torch.int32 if name in ("tok_rank", "topk_id") else torch.float32,
                                            (rows, s.topk_out) if name[:3] == "top" else (rows,)))
        self._call(lib().respec_score, "respec_score", a, stream, self.workspace_ptr)


def alloc_score_outputs(*, rows, topk_out, device="cuda") -> dict:
    """Output tensors of one scoring call."""
    f32, i32 = dict(dtype=torch.float32, device=device), dict(dtype=torch.int32, device=device)
    return {"tok_logprob": torch.empty(rows, **f32), "tok_rank": torch.empty(rows, **i32),
            "lse": torch.empty(rows, **f32), "entropy": torch.empty(rows, **f32),
            "topk_id": torch.empty(rows, topk_out, **i32), "topk_logprob": torch.empty(rows, topk_out, **f32)}
