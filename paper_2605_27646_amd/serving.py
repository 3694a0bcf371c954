"""Python binding of include/hqmq_serve.h: attention of a batch over shared packed prefixes, the attention weight that
cached tokens accumulate, the choice of the tokens to keep and the compaction of packed tensors.  Argument marshalling
only, as in binding.py; the same conventions on buffers and streams."""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding
from .binding import EncodedBuffers, HqmqParams, _check, _Encoded, _stream_ptr, hqmq_sizes

HQMQ_MAX_SHARE = 1024


class _Own(C.Structure):
    _fields_ = [("params", C.POINTER(HqmqParams)), ("enc_k", C.POINTER(_Encoded)), ("enc_v", C.POINTER(_Encoded)),
                ("cap_k", C.c_uint64), ("cap_v", C.c_uint64), ("visible", C.c_void_p)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = binding._load()
        P, I, F, V, U = C.POINTER(HqmqParams), C.c_int32, C.c_float, C.c_void_p, C.c_uint64
        E = C.POINTER(_Encoded)
        lib.hqmq_attend_shared.restype = I
        lib.hqmq_attend_shared.argtypes = [P, I, I, V, F, E, U, V, E, U, V, V, C.POINTER(_Own), V, V, V, U, V]
        lib.hqmq_attend_shared_workspace_bytes.restype = U
        lib.hqmq_attend_shared_workspace_bytes.argtypes = [P, I, I, P]
        lib.hqmq_attend_mass.restype = I
        lib.hqmq_attend_mass.argtypes = [P, I, I, V, F, E, U, V, V, V, V, F, V, V]
        lib.hqmq_evict_select.restype = I
        lib.hqmq_evict_select.argtypes = [I, I, I, V, V, I, I, I, V, V, V, V, U, V]
        lib.hqmq_evict_select_workspace_bytes.restype = U
        lib.hqmq_evict_select_workspace_bytes.argtypes = [I, I, I, I]
        lib.hqmq_evict_compact.restype = I
        lib.hqmq_evict_compact.argtypes = [P, I, I, E, C.POINTER(U), C.POINTER(V), E, C.POINTER(U), V, U, V]
        lib.hqmq_evict_compact_workspace_bytes.restype = U
        lib.hqmq_evict_compact_workspace_bytes.argtypes = [P, I, I]
        _lib = lib
    return _lib


def _on_this_device(*tensors) -> None:
    """The library enqueues on a stream of the current device: a tensor of another one would be read across devices."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:  # -1: of the host
            raise ValueError("every tensor must be on torch's current device")


@functools.lru_cache(maxsize=1024)
def _row_bytes(params: bytes) -> tuple:
    info = hqmq_sizes(HqmqParams.from_buffer_copy(params))
    return info.code_bytes, info.sigma_bytes, info.flag_bytes, info.row_off_bytes


def _hold_rows(params: HqmqParams, enc: EncodedBuffers) -> torch.Tensor:
    """What a call reads of a packed tensor is long enough for the rows that params describes, which the library cannot know, and on
    one device: that of the code words, which are returned."""
    c, s, f, r, o = enc.codes, enc.sigma, enc.flags, enc.row_off, enc.outliers
    n_c, n_s, n_f, n_r = _row_bytes(bytes(params))
    if (c.nbytes < n_c or s.nbytes < n_s or f.nbytes < n_f or r.nbytes < n_r or o.nbytes < 8 * o.shape[0]
            or not (c.is_contiguous() and s.is_contiguous() and f.is_contiguous() and r.is_contiguous() and o.is_contiguous())
            or not (c.get_device() == s.get_device() == f.get_device() == r.get_device() == o.get_device())):
        raise ValueError(f"codes, sigma, flags, row_off and outliers must be contiguous, on one device, and hold {n_c}, {n_s}, {n_f}, {n_r} "
                         "bytes and 8 per payload")
    return c


def _rows_of(name, t, dtype, shape) -> None:
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {str(dtype)[6:]} {list(shape)}")


def _share_of(params: HqmqParams, q: torch.Tensor) -> int:
    shape, B = q.shape, params.B
    if q.dtype is not torch.float16 or len(shape) != 3 or shape[2] != params.D or not q.is_contiguous():
        raise ValueError("q must be contiguous fp16 [n_seqs, n_q_heads, D]")
    if B <= 0 or shape[0] % B or shape[0] == 0:
        raise ValueError("q must have a multiple of the caches' batch entries")
    return shape[0] // B


def _hold(params: HqmqParams, encs) -> None:
    info = hqmq_sizes(params)
    need = {"codes": info.code_bytes, "sigma": info.sigma_bytes, "flags": info.flag_bytes, "row_off": info.row_off_bytes,
            "outliers": 0, "n_outliers": info.n_outliers_bytes, "status": info.status_bytes}
    for e in encs:
        _hold_rows(params, e)
        for name, nbytes in need.items():
            t = getattr(e, name)
            if not t.is_contiguous() or t.numel() * t.element_size() < nbytes:
                raise ValueError(f"{name} must be contiguous and hold {nbytes} bytes")


class OwnTokens:
    """The packed tokens of every sequence's own, for hqmq_attend_shared: params (B = number of sequences), K and V, and how
    many of them each query head sees (int32 [n_seqs, n_q_heads]; None: all).  Built once, reusable while the buffers stay
    in place."""

    def __init__(self, params: HqmqParams, enc_k: EncodedBuffers, enc_v: EncodedBuffers, visible: torch.Tensor | None = None):
        _hold(params, (enc_k, enc_v))
        params = HqmqParams.from_buffer_copy(params)  # as they were checked
        self.params = params
        self.visible = visible
        self.keep = (enc_k, enc_v, enc_k.as_struct(), enc_v.as_struct())
        self.struct = _Own(C.pointer(params), C.pointer(self.keep[2]), C.pointer(self.keep[3]), enc_k.outlier_capacity,
                           enc_v.outlier_capacity, None if visible is None else visible.data_ptr())


def hqmq_attend_shared_workspace_bytes(params: HqmqParams, n_share: int, n_q_heads: int, own_params: HqmqParams | None = None) -> int:
    return int(_load().hqmq_attend_shared_workspace_bytes(C.byref(params), int(n_share), int(n_q_heads),
                                                          None if own_params is None else C.byref(own_params)))


def hqmq_attend_shared(params: HqmqParams, q: torch.Tensor, scale: float, enc_k: EncodedBuffers, sec_k: torch.Tensor,
                       enc_v: EncodedBuffers, sec_v: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                       own: OwnTokens | None = None, visible: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                       stream=None) -> None:
    """Enqueue the attention of q (fp16 [B * n_share, n_q_heads, D]) over the packed prefixes that params describes, n_share
    sequences each, and over the sequences' own packed tokens.  visible: int32 [B * n_share, n_q_heads], the prefix tokens
    that each query head sees (None: all); lse: optional fp32 output of the same shape."""
    n_share = _share_of(params, q)
    shape = q.shape
    rows, sec_shape = shape[:2], (params.H, params.S, 4)
    _rows_of("out", out, torch.float16, shape)
    _rows_of("sec", sec_k, torch.float32, sec_shape)
    _rows_of("sec", sec_v, torch.float32, sec_shape)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if visible is not None:
        _rows_of("visible", visible, torch.int32, rows)
    if lse is not None:
        _rows_of("lse", lse, torch.float32, rows)
    _on_this_device(q, out, sec_k, sec_v, workspace, visible, lse, _hold_rows(params, enc_k), _hold_rows(params, enc_v))
    if own is not None:
        if own.visible is not None:
            _rows_of("the own tokens' visible", own.visible, torch.int32, rows)
        _on_this_device(own.visible, own.keep[0].codes, own.keep[1].codes)
    rc = _load().hqmq_attend_shared(C.byref(params), n_share, shape[1], q.data_ptr(), float(scale),
                                    C.byref(enc_k.as_struct()), enc_k.outlier_capacity, sec_k.data_ptr(),
                                    C.byref(enc_v.as_struct()), enc_v.outlier_capacity, sec_v.data_ptr(),
                                    None if visible is None else visible.data_ptr(),
                                    None if own is None else C.byref(own.struct), out.data_ptr(),
                                    None if lse is None else lse.data_ptr(), workspace.data_ptr(),
                                    workspace.nbytes, _stream_ptr(stream))
    _check(rc, "hqmq_attend_shared")


def hqmq_attend_mass(params: HqmqParams, q: torch.Tensor, scale: float, enc_k: EncodedBuffers, sec_k: torch.Tensor,
                     lse: torch.Tensor, mass: torch.Tensor | None, decay: float = 1.0, visible: torch.Tensor | None = None,
                     out: torch.Tensor | None = None, stream=None) -> None:
    """Enqueue out = decay * mass + the attention weights of every cached token, summed over the query heads that read its
    kv head (fp32 [B, H, T]; out None: in place; mass is not read, and may be None, if decay is 0).  lse: fp32
    [B * n_share, n_q_heads] as the attention returned it."""
    n_share = _share_of(params, q)
    rows = q.shape[:2]
    out = mass if out is None else out
    if out is None or (mass is None and decay != 0.0):
        raise ValueError("mass is needed unless decay is 0 and out is given")
    _rows_of("out", out, torch.float32, (params.B, params.H, params.T))
    if mass is not None and mass is not out:
        _rows_of("mass", mass, torch.float32, out.shape)
    _rows_of("lse", lse, torch.float32, rows)
    _rows_of("sec", sec_k, torch.float32, (params.H, params.S, 4))
    if visible is not None:
        _rows_of("visible", visible, torch.int32, rows)
    _on_this_device(q, sec_k, lse, mass, out, visible, _hold_rows(params, enc_k))
    rc = _load().hqmq_attend_mass(C.byref(params), n_share, rows[1], q.data_ptr(), float(scale),
                                  C.byref(enc_k.as_struct()), enc_k.outlier_capacity, sec_k.data_ptr(), lse.data_ptr(),
                                  None if visible is None else visible.data_ptr(), None if mass is None else mass.data_ptr(),
                                  float(decay), out.data_ptr(), _stream_ptr(stream))
    _check(rc, "hqmq_attend_mass")


def hqmq_evict_select_workspace_bytes(B: int, H: int, T: int, n_keep: int) -> int:
    return int(_load().hqmq_evict_select_workspace_bytes(int(B), int(H), int(T), int(n_keep)))


def hqmq_evict_select(mass: torch.Tensor, n_sink: int, n_recent: int, keep: torch.Tensor, n_kept: torch.Tensor,
                      workspace: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                      kept_mass: torch.Tensor | None = None, stream=None) -> None:
    """Enqueue the choice of the keep.shape[2] tokens that every (b, h) of mass (fp32 [B, H, T]) keeps: the first n_sink and
    last n_recent of lengths[b] (int32 [B]; None: T), and those of largest mass between them.  keep: int32 [B, H, n_keep],
    ascending, -1 behind the last; n_kept: int32 [B, H]; kept_mass: optional fp32 [B, H, n_keep]."""
    shape, kept = mass.shape, keep.shape
    if len(shape) != 3 or len(kept) != 3:
        raise ValueError("mass must be [B, H, T] and keep [B, H, n_keep]")
    B, H, T = shape
    _rows_of("mass", mass, torch.float32, shape)
    _rows_of("keep", keep, torch.int32, (B, H, kept[2]))
    _rows_of("n_kept", n_kept, torch.int32, (B, H))
    if kept_mass is not None:
        _rows_of("kept_mass", kept_mass, torch.float32, kept)
    if lengths is not None:
        _rows_of("lengths", lengths, torch.int32, (B,))
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _on_this_device(mass, keep, n_kept, kept_mass, lengths, workspace)
    rc = _load().hqmq_evict_select(B, H, T, mass.data_ptr(), None if lengths is None else lengths.data_ptr(), int(n_sink),
                                   int(n_recent), kept[2], keep.data_ptr(), n_kept.data_ptr(),
                                   None if kept_mass is None else kept_mass.data_ptr(),
                                   None if workspace is None else workspace.data_ptr(),
                                   0 if workspace is None else workspace.nbytes, _stream_ptr(stream))
    _check(rc, "hqmq_evict_select")


def hqmq_evict_compact_workspace_bytes(params: HqmqParams, n_keep: int, n_tensors: int) -> int:
    return int(_load().hqmq_evict_compact_workspace_bytes(C.byref(params), int(n_keep), int(n_tensors)))


def compacted_params(params: HqmqParams, n_keep: int) -> HqmqParams:
    """params of the tensors that hqmq_evict_compact makes, contiguous strides: [B, H, n_keep, D]."""
    n, D = int(n_keep), params.D
    return HqmqParams(params.B, params.H, n, D, params.H * n * D, n * D, D, params.S, params.b_r, params.C, params.flags)


class CompactBatch:
    """Marshalled argument arrays of hqmq_evict_compact, built once and reusable across calls (the buffers must stay alive and
    in place): packed tensors of one shape, one int32 [B, H, n_keep] of row indices for each (they may be the same tensor),
    and the packed tensors to write."""

    def __init__(self, params: HqmqParams, encs, keeps, outs, workspace: torch.Tensor):
        n = len(encs)
        if not (n == len(keeps) == len(outs)) or n == 0:
            raise ValueError("encs, keeps and outs must be non-empty lists of equal length")
        if keeps[0].dim() != 3:
            raise ValueError("keeps must be [B, H, n_keep]")
        n_keep = int(keeps[0].shape[2])
        for k in keeps:
            _rows_of("keep", k, torch.int32, (params.B, params.H, n_keep))
        for p, tensors in ((params, encs), (compacted_params(params, n_keep), outs)):
            _hold(p, tensors)
            for e in tensors:
                _on_this_device(e.codes, e.sigma, e.flags, e.row_off, e.outliers, e.n_outliers, e.status)
        _on_this_device(*keeps, workspace)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        self.params = HqmqParams.from_buffer_copy(params)  # as they were checked
        self.n = n
        self.n_keep = n_keep
        self.workspace = workspace
        self.keep = (list(encs), list(keeps), list(outs))
        self.enc = (_Encoded * n)(*[e.as_struct() for e in encs])
        self.out = (_Encoded * n)(*[e.as_struct() for e in outs])
        self.cap = (C.c_uint64 * n)(*[e.outlier_capacity for e in encs])
        self.out_cap = (C.c_uint64 * n)(*[e.outlier_capacity for e in outs])
        self.rows = (C.c_void_p * n)(*[k.data_ptr() for k in keeps])


def hqmq_evict_compact(batch: CompactBatch, stream=None) -> None:
    """Enqueue the move of the rows that each tensor of the batch keeps into its new packed tensor."""
    ws = batch.workspace
    _on_this_device(ws)
    rc = _load().hqmq_evict_compact(C.byref(batch.params), batch.n_keep, batch.n, batch.enc, batch.cap, batch.rows, batch.out,
                                    batch.out_cap, ws.data_ptr(), ws.nbytes, _stream_ptr(stream))
    _check(rc, "hqmq_evict_compact")
