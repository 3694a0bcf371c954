"""Python binding of include/hqmq_cache4.h: a paged KV cache held in 4 bits, written token by token, read back and attended
to.  Argument marshalling only, as in binding.py; the same conventions on buffers and streams."""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass

import torch

from . import binding
from .binding import _check, _stream_ptr
from .serving import _on_this_device, _rows_of

HQMQ_CACHE4_FLOAT = 0
HQMQ_CACHE4_INT = 1
_TYPES = {torch.float16: 0, torch.bfloat16: 1}


class Cache4Params(C.Structure):
    """n_pages, page_size (a power of two, 16 or more), H kv heads, D channels of a head, format (HQMQ_CACHE4_*)."""
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("format", C.c_int32)]


class _Buffers(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p)]


class _Batch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("pages_per_seq", C.c_int32), ("max_rows", C.c_int32), ("max_length", C.c_int32),
                ("block_table", C.c_void_p), ("lengths", C.c_void_p), ("starts", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_row", C.c_int64), ("stride_head", C.c_int64)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = binding._load()
        P, B, S, R = C.POINTER(Cache4Params), C.POINTER(_Buffers), C.POINTER(_Batch), C.POINTER(_Rows)
        I, V, U = C.c_int32, C.c_void_p, C.c_uint64
        lib.hqmq_cache4_sizes.restype = I
        lib.hqmq_cache4_sizes.argtypes = [P, C.POINTER(U), C.POINTER(U)]
        for name in ("hqmq_cache4_write", "hqmq_cache4_read"):
            getattr(lib, name).restype = I
            getattr(lib, name).argtypes = [P, B, S, I, I, R, R, V]
        lib.hqmq_cache4_attend.restype = I
        lib.hqmq_cache4_attend.argtypes = [P, B, S, I, I, I, R, C.c_float, I, R, V, V, U, V]
        lib.hqmq_cache4_attend_workspace_bytes.restype = U
        lib.hqmq_cache4_attend_workspace_bytes.argtypes = [P, S, I, I, I]
        _lib = lib
    return _lib


@functools.lru_cache(maxsize=256)
def _sizes(params: bytes) -> tuple:
    codes, scales = C.c_uint64(), C.c_uint64()
    _check(_load().hqmq_cache4_sizes(C.byref(Cache4Params.from_buffer_copy(params)), C.byref(codes), C.byref(scales)), "hqmq_cache4_sizes")
    return codes.value, scales.value


def hqmq_cache4_sizes(params: Cache4Params) -> tuple:
    """(bytes of k_codes and of v_codes, bytes of k_scales and of v_scales)."""
    return _sizes(bytes(params))


@dataclass
class Cache4Buffers:
    """The pages: uint8 tensors of hqmq_cache4_sizes(params) bytes (any shape, contiguous)."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor

    def as_struct(self) -> _Buffers:
        return _Buffers(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(), self.v_scales.data_ptr())


def alloc_cache4(params: Cache4Params, device) -> Cache4Buffers:
    codes, scales = hqmq_cache4_sizes(params)
    return Cache4Buffers(*(torch.empty(n, dtype=torch.uint8, device=device) for n in (codes, scales, codes, scales)))


class Cache4Batch:
    """Which rows a call has and where their tokens lie: block_table (int32 [n_seqs, pages_per_seq]), lengths (int32 [n_seqs], the
    call's rows included), starts (int32 [n_seqs + 1], ascending; None: equal shares).  max_rows and max_length: the largest as
    far as the host knows them, by default all rows (of starts) and all that the table has room for; they shape the launch, not
    the results.  The tensors are read when the calls run, so that one batch serves many steps."""

    def __init__(self, block_table: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor | None = None, max_rows: int | None = None,
                 max_length: int | None = None):
        if block_table.dim() != 2:
            raise ValueError("block_table must be [n_seqs, pages_per_seq]")
        n, pages = block_table.shape
        _rows_of("block_table", block_table, torch.int32, (n, pages))
        _rows_of("lengths", lengths, torch.int32, (n,))
        if starts is not None:
            _rows_of("starts", starts, torch.int32, (n + 1,))
        self.tensors = (block_table, lengths, starts)
        self.struct = _Batch(n, pages, 2 ** 30 if max_rows is None else int(max_rows), 2 ** 30 if max_length is None else int(max_length),
                             block_table.data_ptr(), lengths.data_ptr(), None if starts is None else starts.data_ptr())


def _rows_struct(name: str, x: torch.Tensor, heads: int | None, D: int, like: torch.Tensor | None = None) -> _Rows:
    """x [n_rows, heads, D] with contiguous channels; like: a tensor that has its type and number of rows."""
    if (x.dim() != 3 or x.dtype not in _TYPES or x.shape[2] != D or (heads is not None and x.shape[1] != heads)
            or (D > 1 and x.shape[0] and x.shape[1] and x.stride(2) != 1)):
        raise ValueError(f"{name} must be fp16 or bf16 [n_rows, {'n_q_heads' if heads is None else heads}, {D}] with contiguous channels")
    if like is not None and (x.dtype is not like.dtype or x.shape[0] != like.shape[0]):
        raise ValueError(f"{name} must have the type and the number of rows of the other rows")
    return _Rows(x.data_ptr(), x.stride(0), x.stride(1))


def _hold_cache(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, *rows) -> _Buffers:
    """The buffers are as long as params says, which the library cannot know, and everything is on the current device."""
    codes, scales = hqmq_cache4_sizes(params)
    for t, n in ((cache.k_codes, codes), (cache.v_codes, codes), (cache.k_scales, scales), (cache.v_scales, scales)):
        if t.nbytes < n or not t.is_contiguous():
            raise ValueError(f"the cache's codes must be contiguous and hold {codes} bytes, its scales {scales}")
    _on_this_device(cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales, *batch.tensors, *rows)
    return cache.as_struct()


def _move(name, params, cache, batch, k, v, stream) -> None:
    k_rows = _rows_struct("k", k, params.H, params.D)
    v_rows = _rows_struct("v", v, params.H, params.D, k)
    buffers = _hold_cache(params, cache, batch, k, v)
    rc = getattr(_load(), name)(C.byref(params), C.byref(buffers), C.byref(batch.struct), k.shape[0], _TYPES[k.dtype], C.byref(k_rows),
                                C.byref(v_rows), _stream_ptr(stream))
    _check(rc, name)


def hqmq_cache4_write(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """Enqueue the quantisation of k and v (fp16 or bf16 [n_rows, H, D]) into the pages of the batch's sequences."""
    _move("hqmq_cache4_write", params, cache, batch, k, v, stream)


def hqmq_cache4_read(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """Enqueue the reading of the batch's rows into k and v (fp16 or bf16 [n_rows, H, D])."""
    _move("hqmq_cache4_read", params, cache, batch, k, v, stream)


def hqmq_cache4_attend_workspace_bytes(params: Cache4Params, batch: Cache4Batch, n_rows: int, n_q_heads: int, window: int = 0) -> int:
    return int(_load().hqmq_cache4_attend_workspace_bytes(C.byref(params), C.byref(batch.struct), int(n_rows), int(n_q_heads), int(window)))


def hqmq_cache4_attend(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, q: torch.Tensor, scale: float, out: torch.Tensor,
                       workspace: torch.Tensor | None = None, window: int = 0, lse: torch.Tensor | None = None, stream=None) -> None:
    """Enqueue the causal attention of q (fp16 or bf16 [n_rows, n_q_heads, D]) over the pages of the batch's sequences, with a
    window of that many tokens if it is not 0.  lse: optional fp32 output [n_rows, n_q_heads]."""
    q_rows = _rows_struct("q", q, None, params.D)
    out_rows = _rows_struct("out", out, q.shape[1], params.D, q)
    if lse is not None:
        _rows_of("lse", lse, torch.float32, q.shape[:2])
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    buffers = _hold_cache(params, cache, batch, q, out, lse, workspace)
    rc = _load().hqmq_cache4_attend(C.byref(params), C.byref(buffers), C.byref(batch.struct), q.shape[0], q.shape[1], _TYPES[q.dtype],
                                    C.byref(q_rows), float(scale), int(window), C.byref(out_rows), None if lse is None else lse.data_ptr(),
                                    None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes,
                                    _stream_ptr(stream))
    _check(rc, "hqmq_cache4_attend")
