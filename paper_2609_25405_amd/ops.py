"""Operators beside the step, on torch tensors: the 8-bit paged KV cache (append, read-back,
attention) and scores of tokens under logits.

Marshalling around include/orthrus/kv8.h and include/orthrus/score.h; the arithmetic runs in
liborthrus.so, on torch's current stream unless ``stream`` names another.  Tensors live on the current device.
"""
from __future__ import annotations

import ctypes
from ctypes import POINTER, byref, c_double, c_int32, c_void_p
from typing import Optional

import numpy as np
import torch

from . import _abi as A
from . import _abi_ops as O
from . import runtime as R
from .runtime import current_stream

PAGE = 16
_DTYPES = {"bf16": (A.ORTHRUS_BF16, torch.bfloat16), "f32": (A.ORTHRUS_F32, torch.float32)}


def _check(rc: int, where: str) -> None:
    if rc != A.ORTHRUS_OK:
        raise A.OrthrusError(rc, where)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise A.OrthrusError(A.ORTHRUS_EINVAL, what)


# A call costs the host about as much as a small launch costs the device, so the checks below are few
# and cheap: plain integers for pointers, one device query, one stream query, cached structs.
def _here(*tensors) -> int:
    """The current device, to which the device tensors of a call belong (its stream is the default one)."""
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else -2     # (-1: a host tensor)
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "tensor on another device than the current one")
    return dev


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream, dev=None):
    if stream is not None:
        return stream
    return current_stream() if dev is None else torch._C._cuda_getCurrentRawStream(dev)


class HeadShape:
    """Heads of a layer and how they turn (orthrus_head_shape).  ``rot_dims`` None: the whole head;
    ``rope_freq``: angle per position of each pair (rot_dims / 2 float64), None: from ``rope_base``."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: str = "bf16", rot_dims: Optional[int] = None,
                 interleaved: bool = False, rope_base: float = 10000.0, rope_freq=None, rope_magnitude: float = 1.0,
                 norm_eps: float = 1e-6):
        _need(dtype in _DTYPES, "dtype")
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype = n_q_heads, n_kv_heads, head_dim, dtype
        self.torch_dtype = _DTYPES[dtype][1]
        rot = head_dim if rot_dims is None else rot_dims
        self._freq = None
        fp = None
        if rope_freq is not None:
            self._freq = np.ascontiguousarray(rope_freq, np.float64)
            _need(self._freq.shape == (rot // 2,), "rope_freq length")
            fp = self._freq.ctypes.data_as(POINTER(c_double))
        self.c = O.orthrus_head_shape(n_q_heads, n_kv_heads, head_dim, PAGE, _DTYPES[dtype][0], rot, int(interleaved), rope_base,
                                      rope_magnitude, norm_eps, fp)


class DeviceKV8:
    """An 8-bit paged cache on the GPU: e4m3 pools k [L][n_pages][n_kv][16][hd] and
    v [L][n_pages][n_kv][4][16][hd / 16][4], fp32 scales [L][n_pages][n_kv], the int32 block table."""

    def __init__(self, shape: HeadShape, n_layers: int, n_pages: int, n_seq: int, max_blocks: int, device="cuda"):
        nkv, hd = shape.n_kv_heads, shape.head_dim
        code = lambda *s: torch.zeros((n_layers, n_pages, nkv) + s, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
        scale = lambda: torch.zeros((n_layers, n_pages, nkv), dtype=torch.float32, device=device)
        self._set(shape, code(PAGE, hd), code(4, 16, hd // 16, 4), scale(), scale(),
                  torch.full((n_seq, max_blocks), -1, dtype=torch.int32, device=device))

    @classmethod
    def from_pools(cls, shape: HeadShape, k, v, k_scale, v_scale, block_table) -> "DeviceKV8":
        """A cache over tensors that the caller holds (not copied).  Scales are powers of two: of another only the
        exponent would count."""
        kv = cls.__new__(cls)
        kv._set(shape, k, v, k_scale, v_scale, block_table)
        return kv

    def _set(self, shape, k, v, k_scale, v_scale, block_table):
        nkv, hd = shape.n_kv_heads, shape.head_dim
        L, P = k.shape[:2]
        _need(k.dtype == v.dtype == torch.float8_e4m3fn and k.shape == (L, P, nkv, PAGE, hd) and
              v.shape == (L, P, nkv, 4, 16, hd // 16, 4), "8-bit pools")
        _need(k_scale.dtype == v_scale.dtype == torch.float32 and k_scale.shape == v_scale.shape == (L, P, nkv), "scales")
        _need(block_table.dtype == torch.int32 and block_table.dim() == 2, "block table")
        _need(all(t.is_contiguous() for t in (k, v, k_scale, v_scale, block_table)), "contiguous cache tensors")
        self.shape, self._tensors = shape, (k, v, k_scale, v_scale, block_table)
        self.n_layers, self.n_pages = L, P
        self.n_seq, self.max_blocks = block_table.shape
        self._device = k.get_device()
        _need(all(t.get_device() == self._device for t in self._tensors), "cache tensors on one device")
        self._struct = O.orthrus_kv8(*[t.data_ptr() for t in self._tensors], L, P, self.n_seq, self.max_blocks)
        self._ref = byref(self._struct)

    # the tensors stay the ones the cache was made of
    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_scale = property(lambda self: self._tensors[2])
    v_scale = property(lambda self: self._tensors[3])
    block_table = property(lambda self: self._tensors[4])

    def set_block_table(self, bt: np.ndarray) -> None:
        self.block_table.copy_(torch.from_numpy(np.ascontiguousarray(bt, np.int32)))

    def struct(self) -> O.orthrus_kv8:
        return O.orthrus_kv8.from_buffer_copy(self._struct)

    def _fits(self, shape: HeadShape) -> None:
        if shape is not self.shape:
            _need((shape.n_kv_heads, shape.head_dim) == (self.shape.n_kv_heads, self.shape.head_dim), "cache of other heads")

    def _on(self, dev: int) -> None:
        _need(self._device == dev, "cache on another device than the current one")


def _segments(segments):
    a = np.asarray(segments)
    _need(a.size == 0 or a.dtype.kind in "iu" and bool((a >= -2 ** 31).all() and (a < 2 ** 31).all()), "segment values")
    return np.ascontiguousarray(a.astype(np.int32).reshape(-1, 3))


class RaggedRows:
    """The rows of the calls below (orthrus_rows): a host handle, and the workspace that holds its plan
    and partial results.  One call in flight at a time."""

    def __init__(self, shape: HeadShape, max_rows: int, max_segments: int, max_keys: int, device="cuda"):
        self.shape = shape
        self.handle = c_void_p()
        _check(O.load().orthrus_rows_create(byref(shape.c), byref(self.handle)), "orthrus_rows_create")
        self.nbytes = int(O.load().orthrus_rows_workspace_bytes(self.handle, max_rows, max_segments, max_keys))
        if self.nbytes == 0:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "orthrus_rows_workspace_bytes")
        self.n_rows = 0
        self.buf = None
        if torch.device(device).type == "cuda":
            self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
            _here(self.buf)
            _check(A.orthrus_workspace_init(c_void_p(self.buf.data_ptr()), c_void_p(_stream(None))), "orthrus_workspace_init")

    def plan(self, kv: DeviceKV8, segments, stream: Optional[int] = None) -> None:
        """Plan the rows: (sequence, offset, length) of each segment, in the order of their rows."""
        kv._fits(self.shape)
        dev = _here(self.buf)
        kv._on(dev)
        seg = _segments(segments)
        _check(O.load().orthrus_rows_plan(self.handle, kv._ref, seg.ctypes.data, len(seg), _ptr(self.buf), self.nbytes,
                                          _stream(stream, dev)), "orthrus_rows_plan")
        self.n_rows = int(seg[:, 2].sum())

    def items(self, kv: DeviceKV8, segments):
        """(counts, items[n, 8]) of a plan, on the host alone (orthrus_rows_items)."""
        seg = _segments(segments)
        counts = (c_int32 * 4)()
        args = (self.handle, kv._ref, seg.ctypes.data, len(seg))
        _check(O.load().orthrus_rows_items(*args, counts, None, 0), "orthrus_rows_items")
        items = np.zeros((counts[0] + counts[1], 8), np.int32)
        _check(O.load().orthrus_rows_items(*args, counts, items.ctypes.data, len(items)), "orthrus_rows_items")
        return list(counts), items

    def device_error(self) -> int:
        bits = c_int32(0)
        rc = A.orthrus_device_error(c_void_p(self.buf.data_ptr()), c_void_p(_stream(None)), byref(bits))
        if rc not in (A.ORTHRUS_OK, A.ORTHRUS_EDEVICE):
            raise A.OrthrusError(rc, "orthrus_device_error")
        return bits.value

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            O.load().orthrus_rows_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows_of(self, t: torch.Tensor, width: int, dtype, what: str) -> int:
        """Row stride of a call's tensor: [rows or more][width], elements of a row side by side."""
        n, w = t.shape if t.dim() == 2 else (0, 0)
        if t.dtype != dtype or w != width or n < self.n_rows:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, what + " shape")
        stride, inner = t.stride()
        if inner != 1:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, what + " strides")
        return stride if n > 1 else width          # (one row's stride is nobody's)


def _gain(t, hd):
    if t is None:
        return None
    _need(t.dtype == torch.float32 and t.shape == (hd,) and t.is_contiguous(), "gain shape")
    return t.data_ptr()


def kv8_append(rows: RaggedRows, kv: DeviceKV8, layer: int, qkv: torch.Tensor, q_out: torch.Tensor,
               q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> None:
    """Head norms, rotation and append of the planned rows of qkv [rows][(n_q + 2 n_kv) hd] (the
    shape's dtype, or fp32); the rotated queries go to q_out [rows][n_q hd], which may be the query columns of qkv
    in the same dtype."""
    s = rows.shape
    kv._fits(s)
    dev = _here(qkv, q_out, q_gain, k_gain)
    kv._on(dev)
    f32 = qkv.dtype == torch.float32
    width = (s.n_q_heads + 2 * s.n_kv_heads) * s.head_dim
    stride = rows._rows_of(qkv, width, torch.float32 if f32 else s.torch_dtype, "qkv")
    q_stride = rows._rows_of(q_out, s.n_q_heads * s.head_dim, s.torch_dtype, "q_out")
    rc = O.load().orthrus_kv8_append(rows.handle, kv._ref, layer, qkv.data_ptr(), A.ORTHRUS_F32 if f32 else A.ORTHRUS_BF16, stride,
                                     _gain(q_gain, s.head_dim), _gain(k_gain, s.head_dim), q_out.data_ptr(), q_stride,
                                     _stream(stream, dev))
    _check(rc, "orthrus_kv8_append")


def kv8_read(rows: RaggedRows, kv: DeviceKV8, layer: int, k_out: torch.Tensor, v_out: torch.Tensor,
             stream: Optional[int] = None) -> None:
    """What the cache holds at the planned rows' positions, as bf16 [rows][n_kv hd] (exact)."""
    kv._fits(rows.shape)
    dev = _here(k_out, v_out)
    kv._on(dev)
    width = rows.shape.n_kv_heads * rows.shape.head_dim
    for t in (k_out, v_out):
        if rows._rows_of(t, width, torch.bfloat16, "read-back") != width:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "contiguous read-back")
    _check(O.load().orthrus_kv8_read(rows.handle, kv._ref, layer, k_out.data_ptr(), v_out.data_ptr(), _stream(stream, dev)),
           "orthrus_kv8_read")


def kv8_attend(rows: RaggedRows, kv: DeviceKV8, layer: int, q: torch.Tensor, out: torch.Tensor, scale: Optional[float] = None,
               stream: Optional[int] = None) -> None:
    """Causal attention of the planned rows: q, out [rows][n_q hd] of the shape's dtype (out may be
    q); ``scale`` None: 1 / sqrt(hd)."""
    s = rows.shape
    kv._fits(s)
    dev = _here(q, out)
    kv._on(dev)
    sc = 0.0 if scale is None else ctypes.c_float(scale).value       # (what rounds to zero is not the usual scale)
    _need(scale is None or sc > 0, "scale")
    width = s.n_q_heads * s.head_dim
    stride, out_stride = rows._rows_of(q, width, s.torch_dtype, "q"), rows._rows_of(out, width, s.torch_dtype, "out")
    _check(O.load().orthrus_kv8_attend(rows.handle, kv._ref, layer, q.data_ptr(), stride, sc, out.data_ptr(), out_stride,
                                       _stream(stream, dev)), "orthrus_kv8_attend")


class WorkspaceKV8(R.Workspace):
    """Workspace of `step_kv8` (sizes as those of runtime.Workspace; a chunk's end counts as a context)."""

    def __init__(self, emb: R.DeviceModel, gen: R.DeviceModel, max_tokens: int, max_chunks: int, max_decode: int, max_ctx: int,
                 device="cuda"):
        self.nbytes = int(O.load().orthrus_step_kv8_bytes(emb.handle, gen.handle, max_tokens, max_chunks, max_decode, max_ctx))
        if self.nbytes == 0:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "orthrus_step_kv8_bytes")
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        _here(self.buf)
        _check(A.orthrus_workspace_init(_ptr(self.buf), _stream(None)), "orthrus_workspace_init")


def step_kv8(emb: R.DeviceModel, gen: R.DeviceModel, batch, emb_kv: DeviceKV8, gen_kv: DeviceKV8, acc_sum: torch.Tensor,
             acc_w: torch.Tensor, out_logits: Optional[torch.Tensor], out_emb: Optional[torch.Tensor], ws: WorkspaceKV8,
             stream: Optional[int] = None, packed: Optional[R.PackedBatch] = None, hidden: Optional[torch.Tensor] = None) -> None:
    """One mixed step through 8-bit caches (orthrus_step_kv8): arguments as those of runtime.step."""
    dev = _here(ws.buf, acc_sum, acc_w, out_logits, out_emb, hidden)
    pb = packed if packed is not None else R.PackedBatch(batch)
    for kv, m in ((emb_kv, emb), (gen_kv, gen)):
        kv._on(dev)
        _need((kv.shape.n_kv_heads, kv.shape.head_dim) == (m.cfg.n_kv_heads, m.cfg.head_dim), "cache of other heads")
    if hidden is not None:
        _need(hidden.dtype == torch.float32 and hidden.is_contiguous() and hidden.dim() == 3 and
              hidden.shape[0] >= emb_kv.n_seq and hidden.shape[1:] == (pb.c.hidden_stride, emb.cfg.d_model), "hidden buffer shape")
        pb.c.hidden = hidden.data_ptr()
    rc = O.load().orthrus_step_kv8(emb.handle, gen.handle, byref(pb.c), emb_kv._ref, gen_kv._ref, _ptr(acc_sum), _ptr(acc_w),
                                   _ptr(out_logits), _ptr(out_emb), _ptr(ws.buf), ws.nbytes, _stream(stream, dev))
    _check(rc, "orthrus_step_kv8")


def logprobs_workspace(rows: int, vocab: int, n_top: int = 0, device="cuda") -> Optional[torch.Tensor]:
    """The workspace of `logprobs` for these sizes (None where it needs none)."""
    n = int(O.load().orthrus_logprobs_bytes(rows, vocab, n_top))
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
             entropy: Optional[torch.Tensor] = None, rank: Optional[torch.Tensor] = None, top_ids: Optional[torch.Tensor] = None,
             top_logprobs: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> None:
    """Scores of one token a row of fp32 logits [rows][vocab], and the row's largest entries: fills the
    given outputs (fp32 [rows], int32 [rows], and [rows][n] for the n largest)."""
    _need(logits.dtype == torch.float32 and logits.dim() == 2 and (logits.shape[1] == 1 or logits.stride(1) == 1), "logits")
    R, V = logits.shape
    tops = [t for t in (top_ids, top_logprobs) if t is not None]
    n = tops[0].shape[-1] if tops else 0
    _need(not tops or n > 0, "top outputs")
    for t, dt, shape in ((tokens, torch.int32, (R,)), (rank, torch.int32, (R,)), (logprob, torch.float32, (R,)),
                         (entropy, torch.float32, (R,)), (top_ids, torch.int32, (R, n)), (top_logprobs, torch.float32, (R, n))):
        if t is not None and not (t.dtype == dt and t.shape == shape and t.is_contiguous()):
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "score tensors")
    dev = _here(logits, tokens, logprob, entropy, rank, top_ids, top_logprobs, workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    stride = logits.stride(0) if R > 1 else max(V, logits.stride(0))
    _check(O.load().orthrus_logprobs(_ptr(logits), stride, R, V, _ptr(tokens), n, _ptr(logprob), _ptr(entropy), _ptr(rank),
                                     _ptr(top_ids), _ptr(top_logprobs), _ptr(workspace), ws_bytes, _stream(stream, dev)), "orthrus_logprobs")
