"""ctypes binding of include/kvio_attn.h: the operators on the paged cache.

Like kvio.py it only packs arguments; tensors stand in for pointers.  The calls run on `stream`
(a torch.cuda.Stream or a raw hipStream_t), or with None on torch's current stream, and allocate
what they return or need there.  Tensors that a call reads or writes on another stream than their
own are the caller's to order, as with any kernel.  There is no backward pass: tensors that require
gradients are refused where autograd records.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .kvio import KVIO_EINVAL, KvioError, _check, _lib

KVIO_BF16 = 0
KVIO_FP16 = 1
KVIO_E4M3 = 2
KVIO_APPEND_INTERLEAVED = 0x1

_TYPES = {torch.bfloat16: KVIO_BF16, torch.float16: KVIO_FP16}
_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class kvio_batch(ctypes.Structure):
    _fields_ = [("num_seqs", _i32), ("num_tokens", _i32), ("max_pages", _i32), ("max_query", _i32),
                ("table_stride", _i64), ("page_table", _vp), ("ctx_len", _vp), ("q_start", _vp)]


class kvio_append_args(ctypes.Structure):
    _fields_ = [("batch", kvio_batch), ("dtype", _i32), ("cache_dtype", _i32), ("num_q_heads", _i32), ("rot_dim", _i32),
                ("flags", _i32), ("reserved", _i32), ("k", _vp), ("v", _vp), ("q", _vp), ("q_out", _vp),
                ("k_stride", _i64), ("v_stride", _i64), ("q_stride", _i64), ("q_out_stride", _i64),
                ("inv_freq", _vp), ("positions", _vp), ("k_scale", _vp), ("v_scale", _vp), ("scale_stride", _i64)]


class kvio_attend_args(ctypes.Structure):
    _fields_ = [("batch", kvio_batch), ("dtype", _i32), ("cache_dtype", _i32), ("num_q_heads", _i32), ("window", _i32),
                ("softmax_scale", ctypes.c_float), ("reserved", _i32), ("q", _vp), ("out", _vp), ("lse", _vp),
                ("q_stride", _i64), ("out_stride", _i64), ("k_scale", _vp), ("v_scale", _vp), ("scale_stride", _i64),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


for _name, _args in {"kvio_append": [_vp, _i32, ctypes.POINTER(kvio_append_args), _vp],
                     "kvio_attend": [_vp, _i32, ctypes.POINTER(kvio_attend_args), _vp],
                     "kvio_attend_workspace": [_vp, ctypes.POINTER(kvio_attend_args),
                                               ctypes.POINTER(ctypes.c_size_t)]}.items():
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = ctypes.c_int


def kvio_append(pool: int, layer: int, args: kvio_append_args, stream: Optional[int] = None) -> None:
    _check(_lib.kvio_append(pool, layer, ctypes.byref(args), stream))


def kvio_attend(pool: int, layer: int, args: kvio_attend_args, stream: Optional[int] = None) -> None:
    _check(_lib.kvio_attend(pool, layer, ctypes.byref(args), stream))


def kvio_attend_workspace(pool: int, args: kvio_attend_args) -> int:
    n = ctypes.c_size_t()
    _check(_lib.kvio_attend_workspace(pool, ctypes.byref(args), ctypes.byref(n)))
    return n.value


def _refused(text: str) -> KvioError:
    return KvioError(KVIO_EINVAL, text)


def _need(ok: bool, text: str) -> None:
    if not ok:
        raise _refused(text)


def _number(fn: str, name: str, v: int) -> int:
    """v, which the C struct holds in 32 bits and would cut to its lowest ones."""
    if not 0 <= v < 1 << 31:
        raise _refused(f"{fn}: {name} {v} outside [0, 2^31)")
    return v


class Batch:
    """Where the new tokens of several sequences belong (kvio_batch): page_table, int32 (B, max_pages), whose rows
    may lie apart; ctx_len, int32 (B,), the tokens of each context with the new ones; q_start, int32 (B + 1,), the
    first row of each sequence in q, k and v, or None for one new token each; max_query, the most new tokens of any
    sequence where it is known (0: as many as there are rows).  The tensors are read when a call runs and can be
    written between calls; the Batch keeps them alive."""

    def __init__(self, page_table: torch.Tensor, ctx_len: torch.Tensor, q_start: Optional[torch.Tensor] = None,
                 max_query: int = 0):
        for name, t in (("page_table", page_table), ("ctx_len", ctx_len), ("q_start", q_start)):
            _need(t is None or (t.dtype == torch.int32 and t.is_cuda), f"Batch: {name} must be int32 on the GPU")
        _need(page_table.dim() == 2 and (page_table.stride(1) == 1 or page_table.shape[1] <= 1),
              "Batch: page_table must be (sequences, pages) with the pages of a sequence side by side")
        B, pages = page_table.shape
        _need(ctx_len.shape == (B,) and ctx_len.is_contiguous(), f"Batch: ctx_len must be {B} numbers side by side")
        _need(q_start is None or (q_start.shape == (B + 1,) and q_start.is_contiguous()),
              f"Batch: q_start must be {B + 1} numbers side by side")
        stride = page_table.stride(0) if B > 1 else pages
        self.tensors = (page_table, ctx_len, q_start)
        self.device = page_table.device
        _need(all(t is None or t.device == self.device for t in self.tensors), "Batch: tensors on several GPUs")
        self.num_seqs, self._args = B, kvio_batch(
            B, 0, pages, _number("Batch", "max_query", max_query), stride, page_table.data_ptr(), ctx_len.data_ptr(),
            None if q_start is None else q_start.data_ptr())

    def args(self, num_tokens: int) -> kvio_batch:
        b = kvio_batch.from_buffer_copy(self._args)
        b.num_tokens = num_tokens
        return b


def _rows(fn: str, name: str, x: torch.Tensor, heads: Optional[int], pool, like: Optional[torch.Tensor]):
    """Check (N, heads, D) with heads and dims side by side; the elements from one token to the next."""
    D = pool.tensor.shape[4]
    shape, stride = x.shape, x.stride()
    if not (len(shape) == 3 and shape[2] == D and (heads is None or shape[1] == heads)):
        raise _refused(f"{fn}: {name} must be (tokens, {'heads' if heads is None else heads}, {D}), not {tuple(shape)}")
    if x.dtype not in _TYPES or (like is not None and x.dtype != like.dtype):
        raise _refused(f"{fn}: {name} has the type {x.dtype}")
    if like is not None and shape[0] != like.shape[0]:
        raise _refused(f"{fn}: {name} has {shape[0]} tokens, not {like.shape[0]}")
    if x.requires_grad and torch.is_grad_enabled():
        raise _refused(f"{fn}: {name} requires gradients and {fn} has no backward pass; call it under torch.no_grad()")
    if x.device != pool.tensor.device:
        raise _refused(f"{fn}: {name} is on {x.device}, the pool on {pool.tensor.device}")
    if stride[2] != 1 or (shape[1] != 1 and stride[1] != D):
        raise _refused(f"{fn}: {name}: heads must lie side by side")
    return stride[0] if shape[0] > 1 else shape[1] * D


def _on(pool, stream, call):
    """Run call(raw stream) with `stream` and the pool's GPU current."""
    dev = pool.tensor.device
    if stream is None and dev.index == torch.cuda.current_device():
        return call(torch._C._cuda_getCurrentRawStream(dev.index))   # current_stream() takes microseconds
    with torch.cuda.device(dev):
        s = torch.cuda.current_stream() if stream is None else stream
        if isinstance(s, int):
            s = torch.cuda.ExternalStream(s) if s else torch.cuda.default_stream()
        elif not isinstance(s, torch.cuda.Stream):
            s = torch.cuda.ExternalStream(s.cuda_stream)         # a kvio Stream
        with torch.cuda.stream(s):
            return call(s.cuda_stream)


def _cache(fn: str, pool, args, layer: int, like: torch.Tensor) -> None:
    args.dtype = _TYPES[like.dtype]
    if not 0 <= layer < pool.num_layers:
        raise _refused(f"{fn}: layer {layer} outside [0, {pool.num_layers})")
    if pool.scales is None:
        _need(pool.tensor.element_size() != 1, f"{fn}: an 8-bit pool needs scales")
        if pool.tensor.dtype != like.dtype:
            raise _refused(f"{fn}: new tokens in {like.dtype}, the pool in {pool.tensor.dtype}")
        args.cache_dtype = args.dtype
        return
    args.cache_dtype, args.scale_stride = KVIO_E4M3, pool.scales.stride(2)
    args.k_scale, args.v_scale = pool.scales[0, layer].data_ptr(), pool.scales[1, layer].data_ptr()


def append(pool, layer: int, batch: Batch, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
           q_out: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
           positions: Optional[torch.Tensor] = None, interleaved: bool = False, stream=None) -> Optional[torch.Tensor]:
    """kvio_append with tensors; see KVPool.append."""
    fn = "append"
    H = pool.tensor.shape[3]
    a = kvio_append_args(flags=KVIO_APPEND_INTERLEAVED if interleaved else 0)
    a.k_stride, a.v_stride = _rows(fn, "k", k, H, pool, None), _rows(fn, "v", v, H, pool, k)
    a.batch = batch.args(k.shape[0])
    _cache(fn, pool, a, layer, k)
    a.k, a.v = k.data_ptr(), v.data_ptr()
    if inv_freq is not None:
        _need(inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous() and
              inv_freq.device == pool.tensor.device, f"{fn}: inv_freq must be float32 numbers side by side on the pool's GPU")
        a.rot_dim, a.inv_freq = 2 * inv_freq.numel(), inv_freq.data_ptr()
    if positions is not None:
        _need(positions.dtype == torch.int32 and positions.shape == (k.shape[0],) and positions.is_contiguous(),
              f"{fn}: positions must be {k.shape[0]} int32 numbers side by side")
        a.positions = positions.data_ptr()
    _need(q is not None or q_out is None, f"{fn}: q_out without q")

    def call(s):
        out = q_out
        if q is not None:
            a.q_stride, a.q, a.num_q_heads = _rows(fn, "q", q, None, pool, k), q.data_ptr(), q.shape[1]
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            a.q_out_stride, a.q_out = _rows(fn, "q_out", out, q.shape[1], pool, k), out.data_ptr()
        kvio_append(pool.handle, layer, a, s)
        return out

    return _on(pool, stream, call)


def attend(pool, layer: int, batch: Batch, q: torch.Tensor, out: Optional[torch.Tensor] = None,
           lse: Optional[torch.Tensor] = None, scale: Optional[float] = None, window: int = 0,
           workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """kvio_attend with tensors; see KVPool.attend."""
    fn = "attend"
    a = kvio_attend_args(window=_number(fn, "window", window))
    a.q_stride, a.q = _rows(fn, "q", q, None, pool, None), q.data_ptr()
    a.batch, a.num_q_heads = batch.args(q.shape[0]), q.shape[1]
    _cache(fn, pool, a, layer, q)
    a.softmax_scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.shape == q.shape[:2] and lse.is_contiguous(),
              f"{fn}: lse must be float32 {tuple(q.shape[:2])}, side by side")
        a.lse = lse.data_ptr()

    def call(s):
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        a.out_stride, a.out = _rows(fn, "out", o, q.shape[1], pool, q), o.data_ptr()
        need = kvio_attend_workspace(pool.handle, a)
        if need:
            w = torch.empty(need, dtype=torch.uint8, device=q.device) if workspace is None else workspace
            _need(w.is_contiguous() and w.device == q.device, f"{fn}: workspace must lie on the pool's GPU in one piece")
            a.workspace, a.workspace_bytes = w.data_ptr(), w.numel() * w.element_size()
        kvio_attend(pool.handle, layer, a, s)
        return o

    return _on(pool, stream, call)


def attend_workspace(pool, batch: Batch, q: torch.Tensor, window: int = 0) -> int:
    """Bytes of workspace that attend takes for these; see KVPool.attend."""
    fn = "attend_workspace"
    a = kvio_attend_args(window=_number(fn, "window", window), softmax_scale=1.0)
    _rows(fn, "q", q, None, pool, None)
    a.batch, a.num_q_heads = batch.args(q.shape[0]), q.shape[1]
    _cache(fn, pool, a, 0, q)
    return kvio_attend_workspace(pool.handle, a)
