"""Python binding of include/hqmq_cache4.h: a paged KV cache held in 4 bits, written token by token, read back and attended
to.  Argument marshalling only, as in binding.py; the same conventions on buffers and streams."""
from __future__ import annotations

import ctypes as C
import functools
import struct

import torch

from . import binding
from .binding import _check, _raw_stream, _stream_ptr
from .serving import _rows_of

HQMQ_CACHE4_FLOAT = 0
HQMQ_CACHE4_INT = 1
_TYPES = {torch.float16: 0, torch.bfloat16: 1}


class Cache4Params(C.Structure):
    """n_pages, page_size (a power of two, 16 or more), H kv heads, D channels of a head, format (HQMQ_CACHE4_*)."""
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("H", C.c_int32), ("D", C.c_int32), ("format", C.c_int32)]

    def __setattr__(self, name, value):
        if not -2 ** 31 <= value < 2 ** 31:  # the field would keep the low bits
            raise ValueError(f"{name} must fit 32 bits")
        super().__setattr__(name, value)


class _Buffers(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p)]


class _Batch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("pages_per_seq", C.c_int32), ("max_rows", C.c_int32), ("max_length", C.c_int32),
                ("block_table", C.c_void_p), ("lengths", C.c_void_p), ("starts", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_row", C.c_int64), ("stride_head", C.c_int64)]


# The calls get their structs as bytes or addresses: objects of ctypes and the checks of their types are a fifth of a call's time here.
_pack_rows, _pack_buffers = struct.Struct("@Pqq").pack, struct.Struct("@4P").pack


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = binding._load()
        P, S = C.POINTER(Cache4Params), C.POINTER(_Batch)
        I, V, U = C.c_int32, C.c_void_p, C.c_uint64
        lib.hqmq_cache4_sizes.restype = I
        lib.hqmq_cache4_sizes.argtypes = [P, C.POINTER(U), C.POINTER(U)]
        for name in ("hqmq_cache4_write", "hqmq_cache4_read"):
            getattr(lib, name).restype = I
            getattr(lib, name).argtypes = [V, V, V, I, I, V, V, V]
        lib.hqmq_cache4_attend.restype = I
        lib.hqmq_cache4_attend.argtypes = [V, V, V, I, I, I, V, C.c_float, I, V, V, V, U, V]
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


class Cache4Buffers:
    """The pages: uint8 tensors of hqmq_cache4_sizes(params) bytes (any shape, contiguous), of one device.  They are looked at when
    they are set and with the first call of other params; they have to stay in place from then on."""

    def __init__(self, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor):
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_held", None)  # params, and the calls' argument and device for them

    def as_struct(self) -> _Buffers:
        return _Buffers(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(), self.v_scales.data_ptr())

    def _argument(self, params: Cache4Params) -> tuple:
        key, held = bytes(params), self._held
        if held is None or held[0] != key:
            codes, scales = hqmq_cache4_sizes(params)
            tensors = ((self.k_codes, codes), (self.v_codes, codes), (self.k_scales, scales), (self.v_scales, scales))
            if any(t.dtype is not torch.uint8 or t.nbytes < n or not t.is_contiguous() for t, n in tensors):
                raise ValueError(f"the cache's codes must be contiguous uint8 and hold {codes} bytes, its scales {scales}")
            device = self.k_codes.get_device()
            if any(t.get_device() != device for t, _ in tensors):
                raise ValueError("the cache's tensors must be on one device")
            held = (key, (key, _pack_buffers(*(t.data_ptr() for t in (self.k_codes, self.k_scales, self.v_codes, self.v_scales))), device))
            object.__setattr__(self, "_held", held)
        return held[1]


def alloc_cache4(params: Cache4Params, device) -> Cache4Buffers:
    codes, scales = hqmq_cache4_sizes(params)
    return Cache4Buffers(*(torch.empty(n, dtype=torch.uint8, device=device) for n in (codes, scales, codes, scales)))


def _count(n: int) -> int:  # an argument of 32 bits: what is larger means the same as 2^30
    return max(-1, min(n, 2 ** 30))


class Cache4Batch:
    """Which rows a call has and where their tokens lie: block_table (int32 [n_seqs, pages_per_seq]), lengths (int32 [n_seqs], the
    call's rows included), starts (int32 [n_seqs + 1], ascending; None: equal shares).  max_rows and max_length: the largest as
    far as the host knows them, by default all rows (of starts) and all that the table has room for; they shape the launch, and
    every row and token counts whatever they say.  A max_length near the lengths makes short steps fast.  A length past the table's room
    counts as that room, so that write replaces the last tokens kept: give the table its next page before the step that needs it.  The tensors are read when the calls run, so that one batch serves many steps; they have to stay in place."""

    def __init__(self, block_table: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor | None = None, max_rows: int | None = None,
                 max_length: int | None = None):
        if block_table.dim() != 2:
            raise ValueError("block_table must be [n_seqs, pages_per_seq]")
        n, pages = block_table.shape
        if (n | pages) >> 31:
            raise ValueError("block_table must have less than 2^31 rows and columns")
        _rows_of("block_table", block_table, torch.int32, (n, pages))
        _rows_of("lengths", lengths, torch.int32, (n,))
        if starts is not None:
            _rows_of("starts", starts, torch.int32, (n + 1,))
        self._tensors = (block_table, lengths, starts)
        self._device = block_table.get_device()
        if any(t is not None and t.get_device() != self._device for t in self._tensors):
            raise ValueError("block_table, lengths and starts must be on one device")
        self.struct = _Batch(n, pages, 2 ** 30 if max_rows is None else _count(int(max_rows)), 2 ** 30 if max_length is None else _count(int(max_length)),
                             block_table.data_ptr(), lengths.data_ptr(), None if starts is None else starts.data_ptr())
        self._argument = C.addressof(self.struct)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device  # without asking whether the runtime is up
_ELSEWHERE = "every tensor must be on torch's current device"


def _rows(name: str, x: torch.Tensor, D: int) -> tuple:
    """x [n_rows, heads, D] with contiguous channels: (argument of the calls, its shape, its type)."""
    shape, stride, code = x.shape, x.stride(), _TYPES.get(x.dtype)
    if code is None or len(shape) != 3 or shape[2] != D or (stride[2] != 1 and D > 1 and x.numel()):
        raise ValueError(f"{name} must be fp16 or bf16 [n_rows, heads, {D}] with contiguous channels")
    if (shape[0] | shape[1]) >> 31:  # a count that a 32-bit argument would lose bits of
        raise ValueError(f"{name} must have less than 2^31 rows and heads")
    return _pack_rows(x.data_ptr(), stride[0], stride[1]), shape, code


def _stream(stream, device: int) -> int:
    return _raw_stream(device) if stream is None and _raw_stream is not None else _stream_ptr(stream)


def _move(name, params, cache, batch, k, v, stream) -> None:
    k_rows, shape, code = _rows("k", k, params.D)
    v_rows, v_shape, v_code = _rows("v", v, params.D)
    if shape[1] != params.H or v_shape != shape or v_code != code:
        raise ValueError(f"k and v must be of one type, [n_rows, {params.H}, {params.D}] both")
    params, buffers, device = cache._argument(params)
    if not (device == batch._device == k.get_device() == v.get_device() == _current_device()):
        raise ValueError(_ELSEWHERE)
    rc = getattr(_lib or _load(), name)(params, buffers, batch._argument, shape[0], code, k_rows, v_rows, _stream(stream, device))
    if rc:
        _check(rc, name)


def hqmq_cache4_write(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """Enqueue the quantisation of k and v (fp16 or bf16 [n_rows, H, D]) into the pages of the batch's sequences."""
    _move("hqmq_cache4_write", params, cache, batch, k, v, stream)


def hqmq_cache4_read(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """Enqueue the reading of the batch's rows into k and v (fp16 or bf16 [n_rows, H, D])."""
    _move("hqmq_cache4_read", params, cache, batch, k, v, stream)


def hqmq_cache4_attend_workspace_bytes(params: Cache4Params, batch: Cache4Batch, n_rows: int, n_q_heads: int, window: int = 0) -> int:
    n_rows, n_q_heads = int(n_rows), int(n_q_heads)
    if (n_rows | n_q_heads) >> 31:  # as every number of rows or heads that the calls refuse
        return 0
    return int(_load().hqmq_cache4_attend_workspace_bytes(C.byref(params), C.byref(batch.struct), n_rows, n_q_heads, _count(window)))


def hqmq_cache4_attend(params: Cache4Params, cache: Cache4Buffers, batch: Cache4Batch, q: torch.Tensor, scale: float, out: torch.Tensor,
                       workspace: torch.Tensor | None = None, window: int = 0, lse: torch.Tensor | None = None, stream=None) -> None:
    """Enqueue the causal attention of q (fp16 or bf16 [n_rows, n_q_heads, D]) over the pages of the batch's sequences, with a
    window of that many tokens if it is not 0.  lse: optional fp32 output [n_rows, n_q_heads]."""
    q_rows, shape, code = _rows("q", q, params.D)
    out_rows, out_shape, out_code = _rows("out", out, params.D)
    if out_shape != shape or out_code != code:
        raise ValueError("out must have the shape and the type of q")
    if lse is not None:
        _rows_of("lse", lse, torch.float32, shape[:2])
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    params, buffers, device = cache._argument(params)
    if (not (device == batch._device == q.get_device() == out.get_device() == _current_device())
            or (lse is not None and lse.get_device() != device) or (workspace is not None and workspace.get_device() != device)):
        raise ValueError(_ELSEWHERE)
    rc = (_lib or _load()).hqmq_cache4_attend(params, buffers, batch._argument, shape[0], shape[1], code, q_rows, scale, _count(window), out_rows,
                                              None if lse is None else lse.data_ptr(), None if workspace is None else workspace.data_ptr(),
                                              0 if workspace is None else workspace.nbytes, _stream(stream, device))
    if rc:
        _check(rc, "hqmq_cache4_attend")
