"""ctypes binding of the rotary positions and of the paged cache (include/xkv_paged.h): same names as the C ABI,
argument marshalling only.

Every step runs in the library's CUDA kernels, on torch's current stream of the tensors' device.  torch is
used for device memory and streams.  There is no CPU fallback.
No call takes part in autograd: results carry no gradient, whatever the inputs ask for (xkv_rotary with inverse=True takes
gradients of its outputs to gradients of its inputs).
"""
from __future__ import annotations

import ctypes as C
import struct
from dataclasses import dataclass, field, replace

from .xkv import XKV_E_INVALID, XkvError, _i32, _i64, _sz, _vp, lib

BF16, FP16 = 0, 1
MASK_CAUSAL, MASK_FULL = 0, 1
_DTYPE_NAMES = {"bf16": BF16, "fp16": FP16}

EXPORTED = [
    "xkv_rotary", "xkv_paged_workspace_bytes", "xkv_paged_create", "xkv_paged_destroy", "kv_paged_append",
    "attn_paged_causal", "kv_paged_weights", "kv_paged_evict", "xkv_paged_poll_status",
]


class xkv_rotary_params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rotary_dim", "n_axes", "interleaved", "original_tokens")] + \
               [(n, C.c_double) for n in ("base", "factor", "beta_fast", "beta_slow", "magnitude")]


class xkv_paged_params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "dtype", "page_tokens", "n_pages", "max_seqs",
                                         "reserved")] + \
               [(n, C.c_int64) for n in ("page_stride", "head_stride", "slot_stride")]


class xkv_paged_batch(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_tokens", "max_new", "table_width")] + \
               [(n, C.c_void_p) for n in ("q_start", "lens", "table")]


_f = C.c_float
_batch = C.POINTER(xkv_paged_batch)
_rotary = C.POINTER(xkv_rotary_params)
_rows_of = C.c_char_p            # an array of xkv_rows, packed
lib.xkv_rotary.restype = C.c_int
lib.xkv_rotary.argtypes = [_rotary, _i32, _i32, _vp, _i64, _i32, _rows_of, _i32, _i32, _i32, _vp]
lib.xkv_paged_workspace_bytes.restype = _sz
lib.xkv_paged_workspace_bytes.argtypes = [C.POINTER(xkv_paged_params), _i32]
lib.xkv_paged_create.restype = C.c_int
lib.xkv_paged_create.argtypes = [C.POINTER(xkv_paged_params), _vp, _vp, _vp, _vp, _sz, _vp, C.POINTER(_vp)]
lib.xkv_paged_destroy.restype = C.c_int
lib.xkv_paged_destroy.argtypes = [_vp]
lib.kv_paged_append.restype = C.c_int
lib.kv_paged_append.argtypes = [_vp, _batch, _rows_of, _rotary, _vp, _i64, _vp]
lib.attn_paged_causal.restype = C.c_int
lib.attn_paged_causal.argtypes = [_vp, _batch, _rows_of, _vp, _f, _i32, _i32, _vp]
lib.kv_paged_weights.restype = C.c_int
lib.kv_paged_weights.argtypes = [_vp, _batch, _rows_of, _vp, _f, _f, _i32, _vp]
lib.kv_paged_evict.restype = C.c_int
lib.kv_paged_evict.argtypes = [_vp, _batch, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp]
lib.xkv_paged_poll_status.restype = C.c_int
lib.xkv_paged_poll_status.argtypes = [_vp, _vp]


# xkv_rows: data, tok_stride, head_stride, of one, two or four token tensors
_pack1, _pack2, _pack4 = (struct.Struct(f"{3 * n}q").pack for n in (1, 2, 4))
_ABSENT = (0, 0, 0)


def _refuse(where: str, what: str) -> None:
    raise XkvError(XKV_E_INVALID, f"{where}: {what}")


def _require(ok: bool, where: str, what: str) -> None:
    if not ok:
        _refuse(where, what)


# torch, its 16-bit types, and its queries for the current device and its stream (the public ones build an object at each call,
# which takes as long as a launch)
_torch = _bf16 = _fp16 = _int32 = _fp32 = _device_now = _stream_of = None


def _t():
    global _torch, _bf16, _fp16, _int32, _fp32, _device_now, _stream_of
    if _torch is None:
        import torch
        _bf16, _fp16, _int32, _fp32 = torch.bfloat16, torch.float16, torch.int32, torch.float32
        _device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda device: torch.cuda.current_stream(device).cuda_stream)
        _torch = torch
    return _torch


def _rows(t, where: str, name: str, device: int, dtype, shape: tuple) -> tuple[int, int, int]:
    """(pointer, tok_stride, head_stride) of a token tensor, a [heads][n][d] view with contiguous channels.
    (The stride of a dimension with one entry is never used; torch may give it any value.)"""
    if t.shape != shape:
        _refuse(where, f"{name} is {list(shape)}, not {list(t.shape)}")
    if t.dtype != dtype or t.get_device() != device:
        _refuse(where, f"{name} has another type or device")
    hs, ts, cs = t.stride()
    if cs != 1:
        _refuse(where, f"the channels of {name} are not contiguous")
    heads, n, d = shape
    return t.data_ptr(), (ts if n > 1 else d), (hs if heads > 1 else d)


def _ints(t, where: str, name: str, device: int, shape: tuple) -> int:
    if t.dtype != _int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        _refuse(where, f"{name} is a contiguous int32 tensor of shape {list(shape)} on the same device")
    return t.data_ptr()


def _call(device: int, fn, where: str, *args) -> None:
    """fn(*args, the device's current stream), with that device current."""
    if _device_now() == device:
        status = fn(*args, _stream_of(device))
    else:
        with _torch.cuda.device(device):
            status = fn(*args, _stream_of(device))
    if status:
        raise XkvError(status, where)


@dataclass(frozen=True)
class RotaryParams:
    """How positions turn channels; see xkv_rotary_params."""
    rotary_dim: int
    n_axes: int = 1
    interleaved: bool = False
    base: float = 10000.0
    factor: float = 1.0
    original_tokens: int = 0
    beta_fast: float = 32.0
    beta_slow: float = 1.0
    magnitude: float = 1.0
    struct: xkv_rotary_params = field(init=False, repr=False, compare=False)
    ref: object = field(init=False, repr=False, compare=False)

    def __post_init__(self):
        object.__setattr__(self, "struct", xkv_rotary_params(
            self.rotary_dim, self.n_axes, int(self.interleaved), self.original_tokens, self.base, self.factor,
            self.beta_fast, self.beta_slow, self.magnitude))
        object.__setattr__(self, "ref", C.byref(self.struct))


def _positions(positions, where: str, device: int, n_axes: int, n: int) -> tuple[int, int]:
    if positions.dim() == 1:
        positions = positions[None]
    if positions.dtype != _int32 or positions.get_device() != device or positions.shape != (n_axes, n) or \
            (n > 1 and positions.stride(1) != 1):
        _refuse(where, f"positions is int32 [{n_axes}][{n}] on the same device")
    # (one row, or a stride that torch chose for a dimension with one entry)
    return positions.data_ptr(), (positions.stride(0) if n_axes > 1 else n)


def xkv_rotary(params: RotaryParams, positions, q, k=None, q_out=None, k_out=None, inverse: bool = False):
    """q and k ([heads][n][d] views) turned by their tokens' positions (int32 [n] or [n_axes][n]).
    Returns (q_out, k_out), new tensors unless given; an output may be its input."""
    torch = _torch or _t()
    where = "xkv_rotary"
    if q.dim() != 3 or not q.is_cuda:
        _refuse(where, "q is a [heads][n][d] CUDA tensor")
    device, shape, dtype = q.get_device(), q.shape, q.dtype
    if dtype != _bf16 and dtype != _fp16:
        _refuse(where, "tensors are bf16 or fp16")
    H, n, d = shape
    if q_out is None:
        q_out = torch.empty_like(q)
    rq, ro = _rows(q, where, "q", device, dtype, shape), _rows(q_out, where, "q_out", device, dtype, shape)
    rk = rko = _ABSENT
    K = 0
    if k is not None:
        K = k.shape[0]
        if k_out is None:
            k_out = torch.empty_like(k)
        shape = (K, n, d)
        rk, rko = _rows(k, where, "k", device, dtype, shape), _rows(k_out, where, "k_out", device, dtype, shape)
    pp, ps = _positions(positions, where, device, params.n_axes, n)
    _call(device, lib.xkv_rotary, where, params.ref, BF16 if dtype == _bf16 else FP16, d, pp, ps, n, _pack4(*rq, *ro, *rk, *rko),
          H, K, 1 if inverse else 0)
    return q_out, k_out


class _Fixed:
    """Attributes of `_fixed` are set once: the library has pointers and numbers of them, which another value would not reach."""
    _fixed = frozenset()

    def __setattr__(self, name, value):
        if name in self._fixed and name in self.__dict__:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: make another {type(self).__name__}")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed")
        object.__delattr__(self, name)


@dataclass
class PagedParams:
    n_heads: int
    n_kv_heads: int
    head_dim: int
    page_tokens: int
    n_pages: int
    max_seqs: int
    dtype: str = "bf16"


class PagedBatch(_Fixed):
    """The sequences of a call (xkv_paged_batch): q_start [n_seqs + 1], lens [n_seqs] and table [n_seqs][width] are
    int32 CUDA tensors, read when the kernels run (their contents may change, the tensors are these); n_tokens = rows of the
    token tensors, no sequence has more than max_new new tokens."""
    _fixed = frozenset(("device", "n_seqs", "n_tokens", "max_new", "q_start", "lens", "table", "struct", "ref"))

    def __init__(self, q_start, lens, table, n_tokens: int, max_new: int):
        where = "PagedBatch"
        _t()
        _require(lens.dim() == 1 and table.dim() == 2 and lens.is_cuda, where, "lens is [n_seqs], table [n_seqs][width], on a GPU")
        self.device, n = lens.get_device(), lens.shape[0]
        self.n_seqs, self.n_tokens, self.max_new = n, n_tokens, max_new
        self.q_start, self.lens, self.table = q_start, lens, table
        self.struct = xkv_paged_batch(n, n_tokens, max_new, table.shape[1],
                                      _ints(q_start, where, "q_start", self.device, (n + 1,)),
                                      _ints(lens, where, "lens", self.device, (n,)),
                                      _ints(table, where, "table", self.device, (n, table.shape[1])))
        self.ref = C.byref(self.struct)


class PagedCache(_Fixed):
    """A handle on two pools of pages, [n_pages][n_kv_heads][page_tokens][d] views of any order with contiguous
    channels, and on the weights of their slots (fp32 [n_pages][n_kv_heads][page_tokens], contiguous; optional).
    The caller owns the pools; the handle owns its workspace.  p is a copy: changing it changes nothing."""
    _fixed = frozenset(("p", "device", "dtype", "k_pages", "v_pages", "weights", "workspace", "_heads", "_kv_heads", "_head_dim"))

    def __init__(self, p: PagedParams, k_pages, v_pages, weights=None):
        torch = _t()
        where = "xkv_paged_create"
        self.p = p = replace(p)
        self._heads, self._kv_heads, self._head_dim = p.n_heads, p.n_kv_heads, p.head_dim
        self.handle = _vp()
        _require(p.dtype in _DTYPE_NAMES, where, "dtype is bf16 or fp16")
        self.dtype = torch.bfloat16 if p.dtype == "bf16" else torch.float16
        shape = (p.n_pages, p.n_kv_heads, p.page_tokens, p.head_dim)
        _require(k_pages.is_cuda, where, "the pages are CUDA tensors")
        self.device = k_pages.get_device()
        for t in (k_pages, v_pages):
            _require(t.shape == shape and t.dtype == self.dtype and t.get_device() == self.device and t.stride(3) == 1, where,
                     f"the pages are {list(shape)} views of type {p.dtype} with contiguous channels")
        _require(k_pages.stride() == v_pages.stride(), where, "both pools have the same strides")
        if weights is not None:
            _require(weights.shape == shape[:3] and weights.dtype == torch.float32 and weights.is_contiguous() and
                     weights.get_device() == self.device, where, "weights is contiguous fp32 [n_pages][n_kv_heads][page_tokens]")
        self.k_pages, self.v_pages, self.weights = k_pages, v_pages, weights
        ps, hs, ts, _ = k_pages.stride()
        c = xkv_paged_params(p.n_heads, p.n_kv_heads, p.head_dim, _DTYPE_NAMES[p.dtype], p.page_tokens, p.n_pages, p.max_seqs, 0,
                             ps if p.n_pages > 1 else shape[1] * shape[2] * shape[3], hs if p.n_kv_heads > 1 else shape[2] * shape[3], ts)
        sms = torch.cuda.get_device_properties(self.device).multi_processor_count
        nbytes = int(lib.xkv_paged_workspace_bytes(C.byref(c), sms))
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=k_pages.device)
        _call(self.device, lambda stream: lib.xkv_paged_create(
            C.byref(c), k_pages.data_ptr(), v_pages.data_ptr(), weights.data_ptr() if weights is not None else None,
            self.workspace.data_ptr(), nbytes, stream, C.byref(self.handle)), where)
        self.scale = p.head_dim ** -0.5

    def close(self) -> None:
        if self.handle:
            lib.xkv_paged_destroy(self.handle)
            self.handle = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _shape(self, where: str, batch: PagedBatch, heads: int) -> tuple:
        if batch.device != self.device:
            _refuse(where, "the batch is on another device")
        return heads, batch.n_tokens, self._head_dim

    # ---- the C calls, same names ------------------------------------------
    def kv_paged_append(self, batch: PagedBatch, k, v, q=None, q_out=None, rotary: RotaryParams | None = None, positions=None):
        """New tokens' k (turned by rotary and positions, if given) and v to their slots; q turned into q_out,
        a new tensor unless given.  Returns q_out."""
        where = "kv_paged_append"
        device, dtype = self.device, self.dtype
        shape = self._shape(where, batch, self._kv_heads)
        rk, rv = _rows(k, where, "k", device, dtype, shape), _rows(v, where, "v", device, dtype, shape)
        rq = ro = _ABSENT
        if q is not None:
            shape = (self._heads, batch.n_tokens, self._head_dim)
            if q_out is None:
                q_out = _torch.empty_like(q)
            rq, ro = _rows(q, where, "q", device, dtype, shape), _rows(q_out, where, "q_out", device, dtype, shape)
        ref, pp, ps = None, 0, 0
        if rotary is not None:
            if positions is None:
                _refuse(where, "rotary needs positions")
            pp, ps = _positions(positions, where, device, rotary.n_axes, batch.n_tokens)
            ref = rotary.ref
        _call(device, lib.kv_paged_append, where, self.handle, batch.ref, _pack4(*rk, *rv, *rq, *ro), ref, pp, ps)
        return q_out

    def attn_paged_causal(self, batch: PagedBatch, q, out=None, lse=None, scale: float | None = None, mask: int = MASK_CAUSAL,
                          impl: int = 0):
        """Attention of the new tokens over what their sequences hold; out is a new tensor unless given, lse (fp32
        [n_heads][n_tokens], contiguous) is filled if given.  Returns out."""
        where = "attn_paged_causal"
        shape = self._shape(where, batch, self._heads)
        if out is None:
            out = _torch.zeros_like(q)        # rows that belong to nobody are not written
        rq, ro = _rows(q, where, "q", self.device, self.dtype, shape), _rows(out, where, "out", self.device, self.dtype, shape)
        pl = 0 if lse is None else self._lse(lse, where, shape)
        _call(self.device, lib.attn_paged_causal, where, self.handle, batch.ref, _pack2(*rq, *ro), pl,
              self.scale if scale is None else scale, mask, impl)
        return out

    def _lse(self, lse, where: str, shape: tuple) -> int:
        if lse.dtype != _fp32 or lse.shape != shape[:2] or not lse.is_contiguous() or lse.get_device() != self.device:
            _refuse(where, "lse is contiguous fp32 [n_heads][n_tokens]")
        return lse.data_ptr()

    def kv_paged_weights(self, batch: PagedBatch, q, lse, scale: float | None = None, decay: float = 1.0, mask: int = MASK_CAUSAL) -> None:
        """weights = decay * weights + what the new tokens' softmax gave every cached token (q, lse, scale and mask as
        in attn_paged_causal).  Slots that sequences of the batch share get all updates with decay 1, else one of them."""
        where = "kv_paged_weights"
        shape = self._shape(where, batch, self._heads)
        rq = _rows(q, where, "q", self.device, self.dtype, shape)
        _call(self.device, lib.kv_paged_weights, where, self.handle, batch.ref, _pack1(*rq), self._lse(lse, where, shape),
              self.scale if scale is None else scale, decay, mask)

    def kv_paged_evict(self, batch: PagedBatch, dst_table, keep: int, n_first: int = 0, n_recent: int = 0, kept=None, lens_out=None):
        """Every sequence down to `keep` tokens, moved to the pages of dst_table.  Returns (kept int32
        [n_seqs][n_kv_heads][keep], lens_out int32 [n_seqs]), new tensors unless given."""
        where = "kv_paged_evict"
        device, n = self.device, batch.n_seqs
        if batch.device != device or dst_table.dim() != 2:
            _refuse(where, "dst_table is [n_seqs][width], the batch on the same device")
        if kept is None:
            kept = _torch.empty(n, self._kv_heads, max(keep, 0), dtype=_int32, device=dst_table.device)
        if lens_out is None:
            lens_out = _torch.empty(n, dtype=_int32, device=dst_table.device)
        width = dst_table.shape[1]
        _call(device, lib.kv_paged_evict, where, self.handle, batch.ref, _ints(dst_table, where, "dst_table", device, (n, width)), width,
              keep, n_first, n_recent, _ints(kept, where, "kept", device, (n, self._kv_heads, max(keep, 0))),
              _ints(lens_out, where, "lens_out", device, (n,)))
        return kept, lens_out

    def xkv_paged_poll_status(self) -> int:
        with _torch.cuda.device(self.device):
            return int(lib.xkv_paged_poll_status(self.handle, _stream_of(self.device)))
