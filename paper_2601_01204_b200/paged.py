"""ctypes binding of the rotary positions and of the paged cache (include/xkv_paged.h): same names as the C ABI,
argument marshalling only.

Every step runs in the library's CUDA kernels, on torch's current stream of the tensors' device.  torch is
used for device memory and streams.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass, field

from .xkv import XKV_E_INVALID, XkvError, _check, _i32, _i64, _sz, _vp, lib

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
lib.xkv_rotary.restype = C.c_int
lib.xkv_rotary.argtypes = [_rotary, _i32, _i32, _vp, _i64, _i32, _vp, _vp, _i32, _i64, _i64, _i64, _i64,
                           _vp, _vp, _i32, _i64, _i64, _i64, _i64, _i32, _vp]
lib.xkv_paged_workspace_bytes.restype = _sz
lib.xkv_paged_workspace_bytes.argtypes = [C.POINTER(xkv_paged_params), _i32]
lib.xkv_paged_create.restype = C.c_int
lib.xkv_paged_create.argtypes = [C.POINTER(xkv_paged_params), _vp, _vp, _vp, _vp, _sz, _vp, C.POINTER(_vp)]
lib.xkv_paged_destroy.restype = C.c_int
lib.xkv_paged_destroy.argtypes = [_vp]
lib.kv_paged_append.restype = C.c_int
lib.kv_paged_append.argtypes = [_vp, _batch, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64,
                                _rotary, _vp, _i64, _vp]
lib.attn_paged_causal.restype = C.c_int
lib.attn_paged_causal.argtypes = [_vp, _batch, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _f, _i32, _i32, _vp]
lib.kv_paged_weights.restype = C.c_int
lib.kv_paged_weights.argtypes = [_vp, _batch, _vp, _i64, _i64, _vp, _f, _f, _i32, _vp]
lib.kv_paged_evict.restype = C.c_int
lib.kv_paged_evict.argtypes = [_vp, _batch, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp]
lib.xkv_paged_poll_status.restype = C.c_int
lib.xkv_paged_poll_status.argtypes = [_vp, _vp]


def _require(ok: bool, where: str, what: str) -> None:
    if not ok:
        raise XkvError(XKV_E_INVALID, f"{where}: {what}")


_torch = None


def _t():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _dtype_code(t, where: str) -> int:
    torch = _t()
    _require(t.dtype in (torch.bfloat16, torch.float16), where, "tensors are bf16 or fp16")
    return BF16 if t.dtype == torch.bfloat16 else FP16


def _rows(t, where: str, name: str, device: int, dtype, heads: int, n: int, d: int) -> tuple[int, int, int]:
    """(pointer, tok_stride, head_stride) of a token tensor, a [heads][n][d] view with contiguous channels.
    (The stride of a dimension with one entry is never used; torch may give it any value.)"""
    _require(t.shape == (heads, n, d), where, f"{name} is [{heads}][{n}][{d}], not {list(t.shape)}")
    _require(t.dtype == dtype and t.get_device() == device, where, f"{name} has another type or device")
    hs, ts, cs = t.stride()
    _require(cs == 1, where, f"the channels of {name} are not contiguous")
    return t.data_ptr(), (ts if n > 1 else d), (hs if heads > 1 else d)


def _ints(t, where: str, name: str, device: int, shape: tuple) -> int:
    _require(t.dtype == _t().int32 and t.shape == shape and t.is_contiguous() and t.get_device() == device, where,
             f"{name} is a contiguous int32 tensor of shape {list(shape)} on the same device")
    return t.data_ptr()


class _On:
    """The device's current stream, with that device current for the call."""

    def __init__(self, device: int):
        torch = _t()
        self.stream = torch.cuda.current_stream(device).cuda_stream
        self.guard = None if torch.cuda.current_device() == device else torch.cuda.device(device)

    def __enter__(self) -> int:
        if self.guard is not None:
            self.guard.__enter__()
        return self.stream

    def __exit__(self, *e) -> None:
        if self.guard is not None:
            self.guard.__exit__(*e)


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

    def __post_init__(self):
        object.__setattr__(self, "struct", xkv_rotary_params(
            self.rotary_dim, self.n_axes, int(self.interleaved), self.original_tokens, self.base, self.factor,
            self.beta_fast, self.beta_slow, self.magnitude))


def _positions(positions, where: str, device: int, n_axes: int, n: int) -> tuple[int, int]:
    if positions.dim() == 1:
        positions = positions[None]
    _require(positions.dtype == _t().int32 and positions.get_device() == device and positions.shape == (n_axes, n) and
             (n <= 1 or positions.stride(1) == 1), where, f"positions is int32 [{n_axes}][{n}] on the same device")
    # (one row, or a stride that torch chose for a dimension with one entry)
    return positions.data_ptr(), (positions.stride(0) if n_axes > 1 else n)


def xkv_rotary(params: RotaryParams, positions, q, k=None, q_out=None, k_out=None, inverse: bool = False):
    """q and k ([heads][n][d] views) turned by their tokens' positions (int32 [n] or [n_axes][n]).
    Returns (q_out, k_out), new tensors unless given; an output may be its input."""
    torch = _t()
    where = "xkv_rotary"
    _require(q.dim() == 3 and q.is_cuda, where, "q is a [heads][n][d] CUDA tensor")
    device, (H, n, d) = q.get_device(), q.shape
    code = _dtype_code(q, where)
    if q_out is None:
        q_out = torch.empty_like(q)
    pq, qt, qh = _rows(q, where, "q", device, q.dtype, H, n, d)
    po, ot, oh = _rows(q_out, where, "q_out", device, q.dtype, H, n, d)
    pk = pko = kt = kh = kot = koh = K = 0
    if k is not None:
        _require(k.dim() == 3, where, "k is a [heads][n][d] tensor")
        K = k.shape[0]
        if k_out is None:
            k_out = torch.empty_like(k)
        pk, kt, kh = _rows(k, where, "k", device, q.dtype, K, n, d)
        pko, kot, koh = _rows(k_out, where, "k_out", device, q.dtype, K, n, d)
    pp, ps = _positions(positions, where, device, params.n_axes, n)
    with _On(device) as stream:
        _check(lib.xkv_rotary(C.byref(params.struct), code, d, pp, ps, n, pq, po, H, qt, qh, ot, oh,
                              pk, pko, K, kt, kh, kot, koh, 1 if inverse else 0, stream), where)
    return q_out, k_out


@dataclass
class PagedParams:
    n_heads: int
    n_kv_heads: int
    head_dim: int
    page_tokens: int
    n_pages: int
    max_seqs: int
    dtype: str = "bf16"


class PagedBatch:
    """The sequences of a call (xkv_paged_batch): q_start [n_seqs + 1], lens [n_seqs] and table [n_seqs][width] are
    int32 CUDA tensors, read when the kernels run; n_tokens = rows of the token tensors, no sequence has more
    than max_new new tokens."""

    def __init__(self, q_start, lens, table, n_tokens: int, max_new: int):
        where = "PagedBatch"
        _require(lens.dim() == 1 and table.dim() == 2 and lens.is_cuda, where, "lens is [n_seqs], table [n_seqs][width], on a GPU")
        self.device, n = lens.get_device(), lens.shape[0]
        self.n_seqs, self.n_tokens = n, n_tokens
        self.q_start, self.lens, self.table = q_start, lens, table
        self.struct = xkv_paged_batch(n, n_tokens, max_new, table.shape[1],
                                      _ints(q_start, where, "q_start", self.device, (n + 1,)),
                                      _ints(lens, where, "lens", self.device, (n,)),
                                      _ints(table, where, "table", self.device, (n, table.shape[1])))
        self.ref = C.byref(self.struct)


class PagedCache:
    """A handle on two pools of pages, [n_pages][n_kv_heads][page_tokens][d] views of any order with contiguous
    channels, and on the weights of their slots (fp32 [n_pages][n_kv_heads][page_tokens], contiguous; optional).
    The caller owns the pools; the handle owns its workspace."""

    def __init__(self, p: PagedParams, k_pages, v_pages, weights=None):
        torch = _t()
        where = "xkv_paged_create"
        self.p = p
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
        with _On(self.device) as stream:
            _check(lib.xkv_paged_create(C.byref(c), k_pages.data_ptr(), v_pages.data_ptr(),
                                        weights.data_ptr() if weights is not None else None, self.workspace.data_ptr(),
                                        nbytes, stream, C.byref(self.handle)), where)
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

    def _tokens(self, t, where: str, name: str, batch: PagedBatch, heads: int) -> tuple[int, int, int]:
        return _rows(t, where, name, self.device, self.dtype, heads, batch.n_tokens, self.p.head_dim)

    # ---- the C calls, same names ------------------------------------------
    def kv_paged_append(self, batch: PagedBatch, k, v, q=None, q_out=None, rotary: RotaryParams | None = None, positions=None):
        """New tokens' k (turned by rotary and positions, if given) and v to their slots; q turned into q_out,
        a new tensor unless given.  Returns q_out."""
        where = "kv_paged_append"
        p = self.p
        _require(batch.device == self.device, where, "the batch is on another device")
        pk, kt, kh = self._tokens(k, where, "k", batch, p.n_kv_heads)
        pv, vt, vh = self._tokens(v, where, "v", batch, p.n_kv_heads)
        pq = po = qt = qh = ot = oh = pp = ps = 0
        if q is not None:
            pq, qt, qh = self._tokens(q, where, "q", batch, p.n_heads)
            if q_out is None:
                q_out = _t().empty_like(q)
            po, ot, oh = self._tokens(q_out, where, "q_out", batch, p.n_heads)
        if rotary is not None:
            _require(positions is not None, where, "rotary needs positions")
            pp, ps = _positions(positions, where, self.device, rotary.n_axes, batch.n_tokens)
        with _On(self.device) as stream:
            _check(lib.kv_paged_append(self.handle, batch.ref, pk, kt, kh, pv, vt, vh, pq, qt, qh, po, ot, oh,
                                       C.byref(rotary.struct) if rotary is not None else None, pp, ps, stream), where)
        return q_out

    def attn_paged_causal(self, batch: PagedBatch, q, out=None, lse=None, scale: float | None = None, mask: int = MASK_CAUSAL,
                          impl: int = 0):
        """Attention of the new tokens over what their sequences hold; out is a new tensor unless given, lse (fp32
        [n_heads][n_tokens], contiguous) is filled if given.  Returns out."""
        where = "attn_paged_causal"
        H = self.p.n_heads
        _require(batch.device == self.device, where, "the batch is on another device")
        pq, qt, qh = self._tokens(q, where, "q", batch, H)
        if out is None:
            out = _t().zeros_like(q)        # rows that belong to nobody are not written
        po, ot, oh = self._tokens(out, where, "out", batch, H)
        pl = 0 if lse is None else self._lse(lse, where, batch)
        with _On(self.device) as stream:
            _check(lib.attn_paged_causal(self.handle, batch.ref, pq, qt, qh, po, ot, oh, pl,
                                         self.scale if scale is None else scale, mask, impl, stream), where)
        return out

    def _lse(self, lse, where: str, batch: PagedBatch) -> int:
        _require(lse.dtype == _t().float32 and lse.shape == (self.p.n_heads, batch.n_tokens) and lse.is_contiguous() and
                 lse.get_device() == self.device, where, "lse is contiguous fp32 [n_heads][n_tokens]")
        return lse.data_ptr()

    def kv_paged_weights(self, batch: PagedBatch, q, lse, scale: float | None = None, decay: float = 1.0, mask: int = MASK_CAUSAL) -> None:
        """weights = decay * weights + what the new tokens' softmax gave every cached token (q, lse, scale and mask as
        in attn_paged_causal)."""
        where = "kv_paged_weights"
        _require(batch.device == self.device, where, "the batch is on another device")
        pq, qt, qh = self._tokens(q, where, "q", batch, self.p.n_heads)
        with _On(self.device) as stream:
            _check(lib.kv_paged_weights(self.handle, batch.ref, pq, qt, qh, self._lse(lse, where, batch),
                                        self.scale if scale is None else scale, decay, mask, stream), where)

    def kv_paged_evict(self, batch: PagedBatch, dst_table, keep: int, n_first: int = 0, n_recent: int = 0, kept=None, lens_out=None):
        """Every sequence down to `keep` tokens, moved to the pages of dst_table.  Returns (kept int32
        [n_seqs][n_kv_heads][keep], lens_out int32 [n_seqs]), new tensors unless given."""
        torch = _t()
        where = "kv_paged_evict"
        _require(batch.device == self.device and dst_table.dim() == 2, where, "dst_table is [n_seqs][width], the batch on the same device")
        n = batch.n_seqs
        if kept is None:
            kept = torch.empty(n, self.p.n_kv_heads, max(keep, 0), dtype=torch.int32, device=dst_table.device)
        if lens_out is None:
            lens_out = torch.empty(n, dtype=torch.int32, device=dst_table.device)
        pd = _ints(dst_table, where, "dst_table", self.device, (n, dst_table.shape[1]))
        pk = _ints(kept, where, "kept", self.device, (n, self.p.n_kv_heads, max(keep, 0)))
        pl = _ints(lens_out, where, "lens_out", self.device, (n,))
        with _On(self.device) as stream:
            _check(lib.kv_paged_evict(self.handle, batch.ref, pd, dst_table.shape[1], keep, n_first, n_recent, pk, pl, stream), where)
        return kept, lens_out

    def xkv_paged_poll_status(self) -> int:
        with _On(self.device) as stream:
            return int(lib.xkv_paged_poll_status(self.handle, stream))
