"""Thin ctypes binding over libsale.so (the C ABI declared in include/sale.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  torch supplies device memory and the current stream.  Importing this
module fails loudly when the built library is missing; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, fields
from functools import cached_property
from operator import index

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsale.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it with `python -m paper_2505_24179_amd.build` "
        "(there is no CPU or PyTorch fallback for the SALE kernels)")
_lib = ctypes.CDLL(_LIB_PATH)

OK = 0
FLAG_STATS_CAUSAL = 1
FLAG_SELECT_16BIT = 2
FLAG_SEGMENT_LOCAL = 4
FLAG_ATTN_INT8_QK = 8
FLAG_ATTN_FP8_PV = 16
WS_SELECT = 1
WS_SPARSE_ATTN = 2
WS_DENSE_ATTN = 3
WS_CALIBRATE = 4
WS_INT8_OPERANDS = 5
WS_FP8_OPERANDS = 6
WS_SPARSE_ATTN_MIN = 7
WS_PROMPT_ATTN = 8
PARKED_ROW_BYTES = 33792      # one parking slot of sparse_attn's workspace (see include/sale.h)


class _Params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "seq_len", "head_dim",
        "block_q", "block_k", "sink_blocks", "local_blocks")] + [("flags", ctypes.c_uint32)] + \
        [(n, ctypes.c_int64 * 3) for n in ("q_stride", "k_stride", "v_stride", "o_stride")] + \
        [("n_seqs", ctypes.c_int32), ("cu_seqlens", ctypes.POINTER(ctypes.c_int32))]


@dataclass(frozen=True)
class Params:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    seq_len: int
    head_dim: int = 128
    block_q: int = 64
    block_k: int = 64
    sink_blocks: int = 1
    local_blocks: int = 4
    flags: int = 0
    cu_seqlens: tuple = ()      # variable-length batch: token offsets (0, ..., seq_len) of the packed sequences

    def c(self, q=None, k=None, v=None, o=None) -> _Params:
        """The C struct.  Strides of Q, K, V, O are taken from the tensors given: zero (= contiguous) for a
        contiguous tensor, otherwise its (batch, head, token) element strides, e.g. for a [B, N, H, d]
        projection output viewed as [B, H, N, d] with .transpose(1, 2)."""
        cp = _Params(self.batch, self.n_q_heads, self.n_kv_heads, self.seq_len, self.head_dim,
                     self.block_q, self.block_k, self.sink_blocks, self.local_blocks, self.flags)
        for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o)):
            if t is not None and not t.is_contiguous():
                getattr(cp, name)[:] = [int(x) for x in t.stride()[:3]]
        if self.cu_seqlens:
            offsets = (ctypes.c_int32 * len(self.cu_seqlens))(*self.cu_seqlens)
            cp.n_seqs = len(self.cu_seqlens) - 1
            cp.cu_seqlens = ctypes.cast(offsets, ctypes.POINTER(ctypes.c_int32))
            cp._offsets = offsets      # (the host array lives as long as the struct)
        return cp

    # What follows from the fields alone is made once: a call of a small layer is as long as its host side.  (Offsets that
    # are not a tuple may be changed between calls: they are read by every call.)
    @cached_property
    def _kept(self):
        return ctypes.byref(self.c())

    @property
    def _contiguous(self):
        """The C struct of contiguous tensors, as an argument.  (The library reads it during the call and never writes it, so
        calls and threads may share it.)"""
        return self._kept if isinstance(self.cu_seqlens, tuple) else ctypes.byref(self.c())

    @cached_property
    def _ws_bytes(self) -> dict:
        return {}

    @cached_property
    def _numels(self):
        """Elements of Q (and O), of K (and V)."""
        n = self.batch * self.seq_len * self.head_dim
        return self.n_q_heads * n, self.n_kv_heads * n

    def __reduce__(self):      # (copies and pickles carry the fields, not what was made from them)
        return type(self), tuple(getattr(self, f.name) for f in fields(self))

    @property
    def n_q(self) -> int:
        return self.seq_len // self.block_q

    @property
    def n_k(self) -> int:
        return self.seq_len // self.block_k

    @property
    def words(self) -> int:
        """Mask words per row: those of the longest sequence."""
        longest = self.seq_len
        if self.cu_seqlens:
            longest = max(b - a for a, b in zip(self.cu_seqlens[:-1], self.cu_seqlens[1:]))
        return (longest // self.block_k + 63) // 64


class _Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + \
        [(n, ctypes.c_int64 * 3) for n in ("k_stride", "v_stride")] + \
        [(n, ctypes.c_int32) for n in ("n_pages", "page_tokens", "dtype", "table_width")] + \
        [(n, ctypes.c_void_p) for n in ("table", "lens")]


PAGE_BF16 = 0
PAGE_FP8 = 1


@dataclass(frozen=True, eq=False)
class Cache:
    """Keys and values of many sequences in pages (see include/sale.h): tensors that the program owns and fills as it likes.

    k, v             [pages, KV heads, tokens of a page, head_dim], torch.bfloat16 or torch.float8_e4m3fn, of any strides whose
                     last dimension is contiguous
    table            int32 [sequences, width]: the pages of each sequence in order, -1 (or anything that is no page) where
                     there is none (decode_attn's launches and workspace go by the width: no wider than needed is faster)
    lens             int32 [sequences]: tokens that each sequence holds
    k_scale, v_scale fp32 [KV heads], 8-bit pages only: a key is value * k_scale

    Forking a sequence is copying its row of `table` and `lens` and, if its last page is partly filled, that page
    (`cache_copy`) to a fresh one; freeing is handing its pages to others; compacting is `cache_copy` and new numbers in `table`.
    Contents may change between calls, shapes and strides may not (a new Cache takes others)."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    lens: torch.Tensor
    k_scale: torch.Tensor = None
    v_scale: torch.Tensor = None

    def __post_init__(self):
        for name, t in (("k", self.k), ("v", self.v)):
            if not t.is_cuda:
                raise ValueError(f"{name}: expected a device tensor, got {t.device}")
            if t.dtype not in (torch.bfloat16, torch.float8_e4m3fn) or t.dtype != self.k.dtype:
                raise ValueError(f"{name}: expected pages of torch.bfloat16 or torch.float8_e4m3fn, K and V alike, got {t.dtype}")
            if t.dim() != 4 or t.shape != self.k.shape or t.numel() == 0:
                raise ValueError(f"{name}: expected [pages, KV heads, tokens, head_dim], K and V alike, got {tuple(t.shape)}")
            if t.stride(3) != 1 or t.stride(2) < t.shape[3]:
                raise ValueError(f"{name}: the last dimension has to be contiguous and tokens at least head_dim apart, got strides "
                                 f"{t.stride()}")
        if self.table.dim() != 2:
            raise ValueError(f"table: expected [sequences, pages], got {tuple(self.table.shape)}")
        _expect("table", self.table, torch.int32, self.table.numel())
        _expect("lens", self.lens, torch.int32, self.table.shape[0])
        if self.k.dtype == torch.float8_e4m3fn:
            _expect("k_scale", self.k_scale, torch.float32, self.k.shape[1])
            _expect("v_scale", self.v_scale, torch.float32, self.k.shape[1])
        for name in ("v", "table", "lens", "k_scale", "v_scale"):
            t = getattr(self, name)
            if t is not None and t.device != self.k.device:
                raise ValueError(f"{name}: on {t.device}, the pages of K on {self.k.device}")

    # What follows from shapes and strides is made once; the addresses are read by every call.
    @cached_property
    def _struct(self):
        c = _Cache(n_pages=self.k.shape[0], page_tokens=self.k.shape[2], table_width=self.table.shape[1],
                   dtype=PAGE_FP8 if self.k.dtype == torch.float8_e4m3fn else PAGE_BF16)
        for name, t in (("k_stride", self.k), ("v_stride", self.v)):
            if not t.is_contiguous():
                getattr(c, name)[:] = t.stride()[:3]
        return c, self.k.shape[1], self.k.shape[3], self.table.shape[0], self.k.get_device(), (self.k.dtype, self.k.shape[2], self.table.shape[1])

    def __reduce__(self):      # (as that of Params)
        return type(self), tuple(getattr(self, f.name) for f in fields(self))

    def _arg(self, p: "Params", sequences=None):
        """The C struct for a call with parameters p (over so many sequences)."""
        c, heads, head_dim, rows, device, _ = self._struct
        if heads != p.n_kv_heads or head_dim != p.head_dim:
            raise ValueError(f"cache: pages of {heads} KV heads x {head_dim} channels, the call has {p.n_kv_heads} x {p.head_dim}")
        if sequences is not None and rows != sequences:
            raise ValueError(f"cache: a table of {rows} sequences, the call has {sequences}")
        if device != torch._C._cuda_getDevice():
            raise ValueError(f"cache: expected pages on the current device, got {self.k.device}")
        c.k, c.v, c.table, c.lens = self.k.data_ptr(), self.v.data_ptr(), self.table.data_ptr(), self.lens.data_ptr()
        if c.dtype == PAGE_FP8:
            c.k_scale, c.v_scale = self.k_scale.data_ptr(), self.v_scale.data_ptr()
        return c


_vp, _sz, _i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
_pp, _pc = ctypes.POINTER(_Params), ctypes.POINTER(_Cache)
_SIGS = {
    "sale_workspace_bytes": (_sz, [_pp, ctypes.c_int]),
    "sale_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "sale_quantize_qk": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sale_select": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_select_static": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp]),
    "sale_sparse_attn": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_dense_attn": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_qk_int4_products": (ctypes.c_int, [_pp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp]),
    "sale_attn_int8_operands": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_attn_fp8_operands": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_calibrate_tau": (ctypes.c_int, [_pp, _vp, _vp, _vp, ctypes.c_float, ctypes.c_float, _i32, _vp, _vp, _vp,
                                          _vp, _sz, _vp]),
    "sale_prompt_attn": (ctypes.c_int, [_pp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sale_cache_append": (ctypes.c_int, [_pp, _pc, _vp, _vp, _vp]),
    "sale_cache_copy": (ctypes.c_int, [_pp, _pc, _vp, _vp, _i32, _vp]),
    "sale_decode_attn": (ctypes.c_int, [_pp, _pc, _vp, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "sale_decode_workspace_bytes": (_sz, [_pp, _pc, _i32]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTED = tuple(_SIGS)


class SaleError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"libsale status {status}: {_lib.sale_status_string(status).decode()}")


def _check(status: int) -> None:
    if status != OK:
        raise SaleError(status)


def _ptr(t):
    return None if t is None else t.data_ptr()      # (the argument types make it a void pointer)


def _expect(name: str, t, dtype, numel: int, optional: bool = False):
    """Host-side check of one tensor argument before anything is launched: the C ABI takes raw device pointers
    of contiguous buffers, so a wrong dtype, a strided view or a short buffer would be read or written out of
    bounds on the GPU."""
    if t is not None and t.dtype in (dtype if isinstance(dtype, tuple) else (dtype,)) and t.numel() == numel and t.is_cuda and \
            t.is_contiguous():
        return
    if t is None:
        if optional:
            return
        raise ValueError(f"{name}: required tensor is None")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor, got {t.device}")
    dtypes = dtype if isinstance(dtype, tuple) else (dtype,)
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: expected dtype {dtypes}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor (the library takes no strides), got strides {t.stride()}")
    if t.numel() != numel:
        raise ValueError(f"{name}: expected {numel} elements for these parameters, got {t.numel()} (shape {tuple(t.shape)})")


def _expect_bhnd(name: str, t, p: "Params", heads: int):
    """Q, K, V or O: a bf16 device tensor, either contiguous with batch * heads * seq_len * head_dim elements or
    a strided view of shape [batch, heads, seq_len, head_dim] whose last dimension is contiguous (its other
    three strides then go into the C struct: non-negative multiples of 8 elements)."""
    if t is not None and t.is_cuda and not t.is_contiguous():
        want = (p.batch, heads, p.seq_len, p.head_dim)
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{name}: expected dtype torch.bfloat16, got {t.dtype}")
        if tuple(t.shape) != want:
            raise ValueError(f"{name}: a strided tensor must have shape {want}, got {tuple(t.shape)}")
        st = t.stride()
        if st[3] != 1 or any(x < 0 or x % 8 for x in st[:3]) or st[2] < p.head_dim:
            raise ValueError(f"{name}: strides {st} are not supported (last dimension contiguous, the others "
                             "non-negative multiples of 8 elements, rows at least head_dim apart)")
        return
    _expect(name, t, torch.bfloat16, p.batch * heads * p.seq_len * p.head_dim)


_NO = object()


def _args(p: "Params", q=_NO, k=_NO, v=_NO, o=_NO):
    """Checks Q, K, V, O as _expect_bhnd does -> the C struct for them, as an argument."""
    nq, nk = p._numels
    plain = True
    for name, t, numel, heads in (("q", q, nq, p.n_q_heads), ("k", k, nk, p.n_kv_heads), ("v", v, nk, p.n_kv_heads),
                                  ("o", o, nq, p.n_q_heads)):
        if t is _NO:
            continue
        if t is None or t.dtype is not torch.bfloat16 or t.numel() != numel or not t.is_cuda or not t.is_contiguous():
            _expect_bhnd(name, t, p, heads)
            plain = False
    if plain:
        return p._contiguous
    return ctypes.byref(p.c(*(None if t is _NO else t for t in (q, k, v, o))))


def _expect_ws(ws):
    """-> the workspace's size in BYTES (whatever its dtype).  Size and alignment are the library's to judge
    (SALE_ERR_WORKSPACE)."""
    if ws is None or not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("workspace: expected a contiguous device tensor")
    return ws.numel() * ws.element_size()


def _qkv_numel(p: "Params"):
    return (p.batch * p.n_q_heads * p.seq_len * p.head_dim, p.batch * p.n_kv_heads * p.seq_len * p.head_dim)


def _stream():
    # (the handle alone: torch.cuda.current_stream() builds a Stream object around it on every call)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def raw():
    """The ctypes library handle (tests of error paths call entry points directly)."""
    return _lib


def workspace_bytes(p: Params, which: int) -> int:
    n = p._ws_bytes.get(which)
    if n is None:
        n = int(_lib.sale_workspace_bytes(p._contiguous, which))
        if isinstance(p.cu_seqlens, tuple):
            p._ws_bytes[which] = n
    return n


def status_string(status: int) -> str:
    return _lib.sale_status_string(status).decode()


def quantize_qk(p: Params, q: torch.Tensor, k: torch.Tensor, out=None):
    """-> (q4 u8 [B,Hq,N,64], k4 u8 [B,Hkv,N,64], q_scale f32 [B,Hq,N/bq], k_scale f32 [B,Hkv,N/bk])"""
    dev = q.device
    if out is None:
        q4 = torch.empty(p.batch, p.n_q_heads, p.seq_len, p.head_dim // 2, dtype=torch.uint8, device=dev)
        k4 = torch.empty(p.batch, p.n_kv_heads, p.seq_len, p.head_dim // 2, dtype=torch.uint8, device=dev)
        qs = torch.empty(p.batch, p.n_q_heads, p.seq_len // p.block_q, dtype=torch.float32, device=dev)
        ks = torch.empty(p.batch, p.n_kv_heads, p.seq_len // p.block_k, dtype=torch.float32, device=dev)
    else:
        q4, k4, qs, ks = out
    args = _args(p, q, k)
    if out is not None:      # (what was allocated above fits)
        nq, nk = p._numels
        _expect("q4", q4, torch.uint8, nq // 2); _expect("k4", k4, torch.uint8, nk // 2)
        _expect("q_scale", qs, torch.float32, p.batch * p.n_q_heads * (p.seq_len // p.block_q))
        _expect("k_scale", ks, torch.float32, p.batch * p.n_kv_heads * (p.seq_len // p.block_k))
    _check(_lib.sale_quantize_qk(args, _ptr(q), _ptr(k), _ptr(q4), _ptr(k4), _ptr(qs), _ptr(ks), _stream()))
    return q4, k4, qs, ks


def select(p: Params, q, k, q4, k4, q_scale, k_scale, tau: torch.Tensor, want_stats: bool = False, out=None, ws=None):
    """-> (block_mask int64-viewed-u64 [B,Hq,Nq,W], row_counts i32 [B,Hq,Nq], m~, l~ or None)"""
    dev = q.device
    if out is None:
        mask = torch.empty(p.batch, p.n_q_heads, p.n_q, p.words, dtype=torch.int64, device=dev)
        counts = torch.empty(p.batch, p.n_q_heads, p.n_q, dtype=torch.int32, device=dev)
    else:
        mask, counts = out
    m = l = None
    if want_stats:
        m = torch.empty(p.batch, p.n_q_heads, p.seq_len, dtype=torch.float32, device=dev)
        l = torch.empty_like(m)
    if ws is None:
        ws = torch.empty(max(1, workspace_bytes(p, WS_SELECT)), dtype=torch.uint8, device=dev)
    nq, nk = p._numels
    est16 = bool(p.flags & FLAG_SELECT_16BIT)          # the 16-bit estimate does not read the codes
    args = _args(p, q, k)
    _expect("q4", q4, torch.uint8, nq // 2, optional=est16); _expect("k4", k4, torch.uint8, nk // 2, optional=est16)
    _expect("q_scale", q_scale, torch.float32, p.batch * p.n_q_heads * p.n_q, optional=est16)
    _expect("k_scale", k_scale, torch.float32, p.batch * p.n_kv_heads * p.n_k, optional=est16)
    if tau.numel() not in (1, p.n_q_heads):
        raise ValueError(f"tau: expected 1 or {p.n_q_heads} thresholds, got {tau.numel()}")
    _expect("tau", tau, torch.float32, tau.numel())
    if out is not None:
        _expect("block_mask", mask, (torch.int64, torch.uint64), p.batch * p.n_q_heads * p.n_q * p.words)
        _expect("row_counts", counts, torch.int32, p.batch * p.n_q_heads * p.n_q)
    _check(_lib.sale_select(args, _ptr(q), _ptr(k), _ptr(q4), _ptr(k4), _ptr(q_scale), _ptr(k_scale),
                            _ptr(tau), tau.numel(), _ptr(mask), _ptr(counts), _ptr(m), _ptr(l),
                            _ptr(ws), _expect_ws(ws), _stream()))
    return mask, counts, m, l


SELECT_STATIC_MAX_BYTES = 64 << 20


def select_static(p: Params, q, k, q4, k4, q_scale, k_scale, tau: torch.Tensor, out):
    """sale_select on the library's static scratch: allocates nothing, so `out` = (block_mask, row_counts) is
    required.  -> (block_mask, row_counts)"""
    mask, counts = out
    nq, nk = _qkv_numel(p)
    est16 = bool(p.flags & FLAG_SELECT_16BIT)
    _expect_bhnd("q", q, p, p.n_q_heads); _expect_bhnd("k", k, p, p.n_kv_heads)
    _expect("q4", q4, torch.uint8, nq // 2, optional=est16); _expect("k4", k4, torch.uint8, nk // 2, optional=est16)
    _expect("q_scale", q_scale, torch.float32, p.batch * p.n_q_heads * p.n_q, optional=est16)
    _expect("k_scale", k_scale, torch.float32, p.batch * p.n_kv_heads * p.n_k, optional=est16)
    _expect("tau", tau, torch.float32, tau.numel())
    _expect("block_mask", mask, (torch.int64, torch.uint64), p.batch * p.n_q_heads * p.n_q * p.words)
    _expect("row_counts", counts, torch.int32, p.batch * p.n_q_heads * p.n_q)
    _check(_lib.sale_select_static(ctypes.byref(p.c(q, k)), _ptr(q), _ptr(k), _ptr(q4), _ptr(k4), _ptr(q_scale), _ptr(k_scale),
                                   _ptr(tau), tau.numel(), _ptr(mask), _ptr(counts), None, None, _stream()))
    return mask, counts


def sparse_attn(p: Params, q, k, v, block_mask, row_counts=None, want_lse: bool = False, out=None, ws=None):
    """-> (o bf16 [B,Hq,N,d], lse f32 [B,Hq,N] or None)"""
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty(p.batch, p.n_q_heads, p.seq_len, dtype=torch.float32, device=q.device) if want_lse else None
    if ws is None:
        ws = torch.empty(max(1, workspace_bytes(p, WS_SPARSE_ATTN)), dtype=torch.uint8, device=q.device)
    args = _args(p, q, k, v, o)
    _expect("block_mask", block_mask, (torch.int64, torch.uint64), p.batch * p.n_q_heads * p.n_q * p.words)
    _expect("row_counts", row_counts, torch.int32, p.batch * p.n_q_heads * p.n_q, optional=True)
    _check(_lib.sale_sparse_attn(args, _ptr(q), _ptr(k), _ptr(v), _ptr(block_mask), _ptr(row_counts),
                                 _ptr(o), _ptr(lse), _ptr(ws), _expect_ws(ws), _stream()))
    return o, lse


def dense_attn(p: Params, q, k, v, want_lse: bool = False, out=None, ws=None):
    """-> (o bf16 [B,Hq,N,d], lse f32 [B,Hq,N] or None)"""
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty(p.batch, p.n_q_heads, p.seq_len, dtype=torch.float32, device=q.device) if want_lse else None
    if ws is None:
        ws = torch.empty(max(1, workspace_bytes(p, WS_DENSE_ATTN)), dtype=torch.uint8, device=q.device)
    args = _args(p, q, k, v, o)
    _check(_lib.sale_dense_attn(args, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                _ptr(ws), _expect_ws(ws), _stream()))
    return o, lse


def qk_int4_products(p: Params, q4, k4, q_head: int, q_block: int, k_block_begin: int, k_block_end: int):
    """-> int32 [block_q, (k_block_end - k_block_begin) * block_k]"""
    nq, nk = _qkv_numel(p)
    _expect("q4", q4, torch.uint8, nq // 2); _expect("k4", k4, torch.uint8, nk // 2)
    out = torch.empty(p.block_q, max(0, k_block_end - k_block_begin) * p.block_k, dtype=torch.int32, device=q4.device)
    _check(_lib.sale_qk_int4_products(ctypes.byref(p.c()), _ptr(q4), _ptr(k4), q_head, q_block,
                                      k_block_begin, k_block_end, _ptr(out), _stream()))
    return out


def attn_int8_operands(p: Params, q, k):
    """-> (q8 int8 [B,Hq,N,d], k8 int8 [B,Hkv,N,d], q_scale8 f32 [B,Hq,N/64], k_scale8 f32 [B,Hkv,N/64],
    k_mean f32 [B,Hkv,d]): the 8-bit operands of the quantized Computation-Pass (parity hook)."""
    dev = q.device
    nq, nk = _qkv_numel(p)
    _expect_bhnd("q", q, p, p.n_q_heads); _expect_bhnd("k", k, p, p.n_kv_heads)
    q8 = torch.empty(p.batch, p.n_q_heads, p.seq_len, p.head_dim, dtype=torch.int8, device=dev)
    k8 = torch.empty(p.batch, p.n_kv_heads, p.seq_len, p.head_dim, dtype=torch.int8, device=dev)
    qs = torch.empty(p.batch, p.n_q_heads, p.seq_len // 64, dtype=torch.float32, device=dev)
    ks = torch.empty(p.batch, p.n_kv_heads, p.seq_len // 64, dtype=torch.float32, device=dev)
    mean = torch.empty(p.batch, p.n_kv_heads, p.head_dim, dtype=torch.float32, device=dev)
    ws = torch.empty(max(1, workspace_bytes(p, WS_INT8_OPERANDS)), dtype=torch.uint8, device=dev)
    _check(_lib.sale_attn_int8_operands(ctypes.byref(p.c(q, k)), _ptr(q), _ptr(k), _ptr(q8), _ptr(k8), _ptr(qs), _ptr(ks),
                                        _ptr(mean), _ptr(ws), ws.numel(), _stream()))
    return q8, k8, qs, ks, mean


def attn_fp8_operands(p: Params, v):
    """-> (v8 uint8 [B,Hkv,N,d] FP8 E4M3 bit patterns, v_scale f32 [B,Hkv,d]): the FP8 operand of the low-precision
    second product (parity hook)."""
    dev = v.device
    _expect_bhnd("v", v, p, p.n_kv_heads)
    v8 = torch.empty(p.batch, p.n_kv_heads, p.seq_len, p.head_dim, dtype=torch.uint8, device=dev)
    vs = torch.empty(p.batch, p.n_kv_heads, p.head_dim, dtype=torch.float32, device=dev)
    ws = torch.empty(max(1, workspace_bytes(p, WS_FP8_OPERANDS)), dtype=torch.uint8, device=dev)
    _check(_lib.sale_attn_fp8_operands(ctypes.byref(p.c(v=v)), _ptr(v), _ptr(v8), _ptr(vs), _ptr(ws), _expect_ws(ws),
                                       _stream()))
    return v8, vs


def calibrate_tau(p: Params, q, k, v, tau0: float = 0.008, theta: float = 0.4, max_halvings: int = 8, ws=None):
    """-> (tau f32 [Hq], err f32 [Hq], halvings i32 [Hq]); synchronises the current stream."""
    dev = q.device
    nq, nk = _qkv_numel(p)
    _expect_bhnd("q", q, p, p.n_q_heads); _expect_bhnd("k", k, p, p.n_kv_heads); _expect_bhnd("v", v, p, p.n_kv_heads)
    tau = torch.empty(p.n_q_heads, dtype=torch.float32, device=dev)
    err = torch.empty(p.n_q_heads, dtype=torch.float32, device=dev)
    halv = torch.empty(p.n_q_heads, dtype=torch.int32, device=dev)
    if ws is None:
        ws = torch.empty(max(1, workspace_bytes(p, WS_CALIBRATE)), dtype=torch.uint8, device=dev)
    _check(_lib.sale_calibrate_tau(ctypes.byref(p.c(q, k, v)), _ptr(q), _ptr(k), _ptr(v), tau0, theta, max_halvings,
                                   _ptr(tau), _ptr(err), _ptr(halv), _ptr(ws), _expect_ws(ws),
                                   _stream()))
    return tau, err, halv


def _on_current_device(names: str, *tensors):
    """The calls are launched on the current device's stream."""
    at = torch._C._cuda_getDevice()
    for i, t in enumerate(tensors):
        if t is not None and t.get_device() != at:
            raise ValueError(f"{names.split()[i]}: expected a tensor on the current device, cuda:{at}, got {t.device}")


def _n_sequences(p: Params) -> int:
    return len(p.cu_seqlens) - 1 if p.cu_seqlens else p.batch


def prompt_attn(p: Params, q, k, v, want_lse: bool = False, out=None, ws=None):
    """Causal attention over whole prompts of any lengths (p.seq_len, or packed ones by p.cu_seqlens; p's blocks are not read).
    -> (o bf16 [B,Hq,N,d], lse f32 [B,Hq,N] or None)"""
    o = torch.empty_like(q) if out is None else out
    args = _args(p, q, k, v, o)
    lse = torch.empty(p.batch, p.n_q_heads, p.seq_len, dtype=torch.float32, device=q.device) if want_lse else None
    if ws is None:
        ws = torch.empty(max(1, workspace_bytes(p, WS_PROMPT_ATTN)), dtype=torch.uint8, device=q.device)
    _on_current_device("q k v out workspace", q, k, v, o, ws)
    _check(_lib.sale_prompt_attn(args, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(ws), _expect_ws(ws), _stream()))
    return o, lse


def cache_append(p: Params, cache: Cache, k, v) -> None:
    """Writes K, V bf16 [B,Hkv,n,d] of the n = p.seq_len new tokens of every sequence (packed ones: p.cu_seqlens) into its pages,
    as the last n of the cache.lens[s] tokens that it holds with them."""
    c = cache._arg(p, _n_sequences(p))
    args = _args(p, k=k, v=v)
    _on_current_device("k v", k, v)
    _check(_lib.sale_cache_append(args, c, _ptr(k), _ptr(v), _stream()))


def _host_pages(name: str, pages):
    if not isinstance(pages, torch.Tensor):
        try:
            pages = torch.tensor([index(x) for x in pages], dtype=torch.int32)      # (a float would be rounded without a word)
        except (TypeError, RuntimeError) as e:
            raise ValueError(f"{name}: expected a list of pages, whole numbers of 32 bits") from e
    if pages.is_cuda or pages.dtype != torch.int32 or pages.dim() != 1 or not pages.is_contiguous():
        raise ValueError(f"{name}: expected a list of pages, or a contiguous one-dimensional int32 tensor on the host")
    return pages


def cache_copy(p: Params, cache: Cache, src, dst) -> None:
    """Copies pages of K and V: dst[i] becomes src[i].  src, dst: lists or int32 tensors on the HOST; the dst all different, none
    of them among the src."""
    src, dst = _host_pages("src", src), _host_pages("dst", dst)
    if src.numel() != dst.numel():
        raise ValueError(f"cache_copy: {src.numel()} sources, {dst.numel()} destinations")
    c = cache._arg(p)
    _check(_lib.sale_cache_copy(p._contiguous, c, _ptr(src), _ptr(dst), src.numel(), _stream()))


_MOST_KEPT_SIZES = 256


def _decode_size(p: Params, cache: Cache, prefix_len: int):
    """-> bytes of workspace, and what to keep them by if they are not kept yet.  (The library says 0 of a cache that it refuses,
    too, while another of these sizes may be a good one: 0 is kept once a call without a workspace has gone through.)"""
    key = (*cache._struct[5], prefix_len)
    n = p._ws_bytes.get(key)
    if n is not None:
        return n, None
    return int(_lib.sale_decode_workspace_bytes(p._contiguous, cache._arg(p, _n_sequences(p)), prefix_len)), key


def _keep_size(p: Params, key, n: int) -> None:
    if len(p._ws_bytes) >= _MOST_KEPT_SIZES:      # (a program may go through any number of prefix lengths)
        p._ws_bytes.clear()
    p._ws_bytes[key] = n


def decode_workspace_bytes(p: Params, cache: Cache, prefix_len: int = 0) -> int:
    n, key = _decode_size(p, cache, prefix_len)
    if n and key is not None:
        _keep_size(p, key, n)
    return n


def decode_attn(p: Params, cache: Cache, q, prefix=None, prefix_len: int = 0, want_lse: bool = False, out=None, ws=None):
    """Attention of the last p.seq_len tokens of every sequence, q bf16 [B,Hq,n,d], to the prefix that all share (the pages
    `prefix`, int32 on the device, of which prefix_len tokens count) and to its own keys, the new tokens' among them.
    -> (o bf16 [B,Hq,n,d], lse f32 [B,Hq,n] or None)"""
    o = torch.empty_like(q) if out is None else out
    c = cache._arg(p, _n_sequences(p))
    args = _args(p, q, o=o)
    if prefix_len > 0:
        if prefix is None or prefix.dtype != torch.int32 or not prefix.is_contiguous() or \
                prefix.numel() * cache.k.shape[2] < prefix_len:
            raise ValueError(f"prefix: expected the pages of {prefix_len} tokens, a contiguous int32 tensor on the device")
    else:
        prefix = None
    lse = torch.empty(p.batch, p.n_q_heads, p.seq_len, dtype=torch.float32, device=q.device) if want_lse else None
    key = None
    if ws is None:
        n_ws, key = _decode_size(p, cache, prefix_len)
        if n_ws:
            ws = torch.empty(n_ws, dtype=torch.uint8, device=q.device)
    else:
        n_ws = _expect_ws(ws)
    _on_current_device("q prefix out workspace", q, prefix, o, ws)
    _check(_lib.sale_decode_attn(args, c, _ptr(q), _ptr(prefix), prefix_len, _ptr(o), _ptr(lse), _ptr(ws), n_ws, _stream()))
    if key is not None:
        _keep_size(p, key, n_ws)
    return o, lse
