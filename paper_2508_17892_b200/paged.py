"""Python binding of the paged cache in ``include/ilre_recall.h`` (argument marshalling only): what a compressed
prompt is answered from.

``PagedCache`` appends new rows (with their rotary positions), attends over the cached ones, gathers the attention
weight that each row receives and evicts by it; ``rope`` turns a tensor of heads alone.  Tensors are the caller's.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, fields
from typing import Optional, Tuple

import torch

from .recall import IlreError, load_library

_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_SCALINGS = {"none": 0, "linear": 1, "banded": 2, "yarn": 3}


class IlreRopeSpec(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_double), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("factor", ctypes.c_double), ("orig_len", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("attn_factor", ctypes.c_double)]


class IlrePagedConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_kv_heads", "n_q_heads", "head_dim", "page_size", "dtype", "max_seqs",
                                              "device")]


class IlrePagedBatch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_q_len", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p)]


class IlrePagedPool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("w", ctypes.c_void_p),
                ("k_page_stride", ctypes.c_int64), ("v_page_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32)]


def declare(lib: ctypes.CDLL) -> None:
    """Prototypes of the calls in this module."""
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    spec, batch, pool = (ctypes.POINTER(t) for t in (IlreRopeSpec, IlrePagedBatch, IlrePagedPool))
    lib.ilre_rope.argtypes = [spec, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, vp]
    lib.ilre_paged_create.argtypes = [ctypes.POINTER(IlrePagedConfig), ctypes.POINTER(vp)]
    lib.ilre_paged_append.argtypes = [vp, batch, spec, vp, vp, i64, vp, i64, vp, i64, vp, i64, pool, vp]
    lib.ilre_paged_attention.argtypes = [vp, batch, vp, i64, pool, vp, vp, vp]
    lib.ilre_paged_accumulate.argtypes = [vp, batch, vp, i64, vp, pool, vp]
    lib.ilre_paged_evict.argtypes = [vp, batch, i32, i32, i32, i32, pool, vp, i32, vp, vp, vp]
    for name in ("status", "last_launch_count", "check_guards", "destroy"):
        getattr(lib, "ilre_paged_" + name).argtypes = [vp]


def _int32(*values: int) -> None:
    """What goes into 32 bits of a C structure; ctypes would cut off the rest."""
    for v in values:
        if not -(1 << 31) <= v < 1 << 31:
            raise AssertionError("a number of more than 32 bits")


@dataclass(frozen=True)
class RopeSpec:
    """Rotary positions: layout, rotated part of the head and scaling (see ``ilre_rope_spec_t``).

    scaling: "none", "linear", "banded" (low, high: frequency factors) or "yarn" (low, high: the turns
    beta_slow, beta_fast).  attn_factor 0: 0.1 ln(factor) + 1 with "yarn", else 1."""
    theta: float = 500000.0
    rotary_dim: int = 128
    interleaved: bool = False
    scaling: str = "none"
    factor: float = 1.0
    orig_len: float = 8192
    low: float = 1.0
    high: float = 4.0
    attn_factor: float = 0.0

    def __post_init__(self):
        _int32(self.rotary_dim)
        object.__setattr__(self, "_c", IlreRopeSpec(
            self.theta, self.rotary_dim, int(self.interleaved), _SCALINGS[self.scaling], self.factor, self.orig_len,
            self.low, self.high, self.attn_factor))
        object.__setattr__(self, "ref", ctypes.byref(self._c))

    def __reduce__(self):                                  # copies and pickles hold the fields, not the C struct
        return type(self), tuple(getattr(self, f.name) for f in fields(self))


@dataclass(frozen=True)
class PagedBatch:
    """Sequences of one call (``ilre_paged_batch_t``); keeps its tensors alive.

    q_start int32 [n_seqs + 1] (None for ``evict``), kv_len int32 [n_seqs], block_table int32 [n_seqs, max_blocks],
    contiguous and on one device."""
    q_start: Optional[torch.Tensor]
    kv_len: torch.Tensor
    block_table: torch.Tensor
    n_tokens: int
    max_q_len: int

    def __post_init__(self):
        for t in (self.q_start, self.kv_len, self.block_table):
            if t is not None and not (t.dtype == torch.int32 and t.is_contiguous() and t.device == self.kv_len.device):
                raise AssertionError("the batch's arrays are contiguous int32 tensors of one device")
        n = self.kv_len.numel()
        if self.kv_len.dim() != 1 or self.block_table.dim() != 2 or self.block_table.shape[0] != n:
            raise AssertionError("kv_len [n_seqs] and block_table [n_seqs, max_blocks]")
        if self.q_start is not None and self.q_start.shape != (n + 1,):
            raise AssertionError("q_start [n_seqs + 1]")
        _int32(self.n_tokens, self.max_q_len)
        object.__setattr__(self, "_c", IlrePagedBatch(
            self.kv_len.numel(), self.n_tokens, self.max_q_len, self.block_table.shape[1], _ptr(self.q_start),
            self.kv_len.data_ptr(), self.block_table.data_ptr()))
        object.__setattr__(self, "ref", ctypes.byref(self._c))
        object.__setattr__(self, "index", self.kv_len.get_device())


def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _rows(t: torch.Tensor, index: int, dtype, heads: int, dim: int) -> int:
    """Stride in elements from token to token of a tensor [n, heads, dim] whose tokens are contiguous."""
    n, h, d = t.shape
    st, sh, sd = t.stride()
    if not (h == heads and d == dim and t.dtype == dtype and t.get_device() == index):
        raise AssertionError("rows of another shape, type or device")
    if n > 0 and (sd != 1 or (heads > 1 and sh != dim)):
        raise AssertionError("the heads of a token are not contiguous")
    return st if n > 1 else heads * dim


def _ints(t: torch.Tensor, index: int, n: int) -> None:
    if not (t.get_device() == index and t.dtype == torch.int32 and t.shape == (n,) and t.is_contiguous()):
        raise AssertionError("not a contiguous int32 array of this device and length")


def _on_stream(stream: torch.cuda.Stream, index: int, tensors):
    """The named stream of a call on device `index`: current inside, so tensors made inside are its own; the caller's
    tensors are marked as in use by it."""
    if stream.device.index != index:
        raise AssertionError("the stream is another device's")
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return torch.cuda.stream(stream)


_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)     # (a Stream object takes microseconds)


class _Rope(torch.autograd.Function):
    """``rope`` where a gradient is asked for: linear, so its gradient is the transposed map of what comes back."""

    @staticmethod
    def forward(ctx, x, positions, spec, transposed):
        ctx.save_for_backward(positions)
        ctx.spec, ctx.transposed = spec, transposed
        return rope(x, positions, spec, transposed)

    @staticmethod
    def backward(ctx, grad):
        grad = grad.contiguous()
        if grad.data_ptr() % 16:                           # a slice of a wider buffer
            grad = grad.clone()
        return rope(grad, ctx.saved_tensors[0], ctx.spec, not ctx.transposed), None, None, None


def rope(x: torch.Tensor, positions: torch.Tensor, spec: RopeSpec, transposed: bool = False,
         out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """x [n_tokens, n_heads, head_dim] (bf16 or fp16; tokens may be strided) turned by int32 ``positions``.

    ``out`` may be ``x``.  ``transposed`` applies the transposed map: the gradient of ``rope`` with
    respect to x is ``rope(grad, positions, spec, transposed=True)``.  Differentiable with respect to x
    where no ``out`` is given; with it a tensor that requires its gradient is refused."""
    if stream is not None:
        with _on_stream(stream, x.get_device(), (x, positions, out)):
            return rope(x, positions, spec, transposed, out)
    if (x.requires_grad or (out is not None and out.requires_grad)) and torch.is_grad_enabled():
        if out is not None:
            raise AssertionError("out has no gradient: without it, or under torch.no_grad()")
        return _Rope.apply(x, positions, spec, transposed)
    dtype, index = x.dtype, x.get_device()
    if index < 0 or dtype not in _DTYPES:
        raise AssertionError("x is not a bf16 or fp16 tensor of a CUDA device")
    n, heads, dim = x.shape
    _ints(positions, index, n)
    x_stride = _rows(x, index, dtype, heads, dim)
    if out is None:
        out = torch.empty(n, heads, dim, dtype=dtype, device=x.device)
    out_stride = _rows(out, index, dtype, heads, dim)
    if out.shape[0] != n:
        raise AssertionError("out has another number of tokens")
    args = (spec.ref, x.data_ptr(), x_stride, out.data_ptr(), out_stride, positions.data_ptr(), n, heads, dim,
            _DTYPES[dtype], int(transposed), _raw_stream(index))
    if torch.cuda.current_device() == index:
        rc = load_library().ilre_rope(*args)
    else:
        with torch.cuda.device(index):
            rc = load_library().ilre_rope(*args)
    if rc != 0:
        raise IlreError(rc, "ilre_rope")
    return out


class PagedCache:
    """Owns one ``ilre_paged_t`` handle; the pools, tables and lengths are the caller's tensors.

    k_pool, v_pool: [n_pages, page_size, n_kv_heads, 128], pages contiguous (the stride from page to page is
    free, so the two may be halves of one tensor); w_pool: fp32 [n_pages, n_kv_heads, page_size].
    For serving: results carry no graph, whatever the tensors require (``rope`` alone is differentiable).
    One stream at a time; graphs that hold calls of one handle must not run at the same time."""

    def __init__(self, n_kv_heads: int = 8, n_q_heads: int = 32, page_size: int = 64,
                 dtype: torch.dtype = torch.bfloat16, max_seqs: int = 256, head_dim: int = 128, device: int = 0):
        _int32(n_kv_heads, n_q_heads, page_size, max_seqs, head_dim, device)
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.cfg = IlrePagedConfig(n_kv_heads, n_q_heads, head_dim, page_size, _DTYPES[dtype], max_seqs, device)
        rc = self._lib.ilre_paged_create(ctypes.byref(self.cfg), ctypes.byref(self._h))
        if rc != 0:
            self._h = ctypes.c_void_p()
            raise IlreError(rc, "ilre_paged_create")
        self.dtype, self._n_q, self._dim = dtype, n_q_heads, head_dim
        self.device = torch.device("cuda", device)
        self._index = device
        self._page_shape = (page_size, n_kv_heads, head_dim)
        self._weight_shape = (n_kv_heads, page_size)
        self._page_stride = (n_kv_heads * head_dim, head_dim, 1)

    def batch(self, q_start: Optional[torch.Tensor], kv_len: torch.Tensor, block_table: torch.Tensor, n_tokens: int,
              max_q_len: int) -> PagedBatch:
        """q_start int32 [n_seqs + 1] (None for ``evict``), kv_len int32 [n_seqs] (the new tokens' rows among
        them), block_table int32 [n_seqs, max_blocks]; at most max_q_len new tokens per sequence."""
        if kv_len.device != self.device:
            raise AssertionError("the batch's arrays are on another device")
        return PagedBatch(q_start, kv_len, block_table, n_tokens, max_q_len)

    def _page_step(self, t: Optional[torch.Tensor], shape) -> int:
        """Stride in elements from page to page (0: back to back)."""
        if t is None:
            return 0
        if not (t.shape == shape and t.dtype == self.dtype and t.get_device() == self._index):
            raise AssertionError("a pool of another shape, type or device")
        step = t.stride()
        if not (step[1:] == self._page_stride or shape[0] == 0 or t[0].is_contiguous()):
            raise AssertionError("a page is not contiguous")
        if shape[0] <= 1:
            return 0
        if step[0] == 0:                                   # to the library that would say back to back
            raise AssertionError("the pool is one page shown many times")
        return step[0]

    def _pool(self, batch: PagedBatch, k: torch.Tensor, v: Optional[torch.Tensor], w: Optional[torch.Tensor]) -> IlrePagedPool:
        if batch.index != self._index:
            raise AssertionError("the batch's arrays are on another device")
        n_pages = k.shape[0]
        shape = (n_pages,) + self._page_shape
        if not (w is None or (w.shape == (n_pages,) + self._weight_shape and w.dtype == torch.float32 and
                             w.is_contiguous() and w.get_device() == self._index)):
            raise AssertionError("w_pool of another shape, type or device")
        return IlrePagedPool(k.data_ptr(), _ptr(v), _ptr(w), self._page_step(k, shape), self._page_step(v, shape), n_pages)

    def _q(self, batch: PagedBatch, q: torch.Tensor) -> int:
        n = batch.n_tokens
        if not (q.shape[0] == n and (n == 0 or batch.q_start is not None)):
            raise AssertionError("q has another number of tokens, or the batch no q_start")
        return _rows(q, self._index, self.dtype, self._n_q, self._dim)

    def append(self, batch: PagedBatch, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
               positions: Optional[torch.Tensor], spec: Optional[RopeSpec], k_pool: torch.Tensor, v_pool: torch.Tensor,
               w_pool: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
        """k turned and v copied to the new tokens' rows, their weights cleared; returns q turned (``q_out``, which
        may be q; made here if not given).  spec None: nothing is turned."""
        if stream is not None:
            with _on_stream(stream, self._index, (q, k, v, positions, k_pool, v_pool, w_pool, q_out, batch.q_start,
                                                  batch.kv_len, batch.block_table)):
                return self.append(batch, q, k, v, positions, spec, k_pool, v_pool, w_pool, q_out)
        n, n_kv, dim = batch.n_tokens, self._page_shape[1], self._dim
        if k.shape[0] != n or v.shape[0] != n:
            raise AssertionError("k or v has another number of tokens")
        k_stride = _rows(k, self._index, self.dtype, n_kv, dim)
        v_stride = _rows(v, self._index, self.dtype, n_kv, dim)
        if spec is not None and positions is None:
            raise AssertionError("a rotation without positions")
        if positions is not None:
            _ints(positions, self._index, n)
        pool = self._pool(batch, k_pool, v_pool, w_pool)
        q_stride = q_out_stride = 0
        if q is not None:
            q_stride = self._q(batch, q)
            if q_out is None:
                q_out = torch.empty(n, self._n_q, dim, dtype=q.dtype, device=q.device)
            q_out_stride = self._q(batch, q_out)
        else:
            if q_out is not None:
                raise AssertionError("q_out without q")
        rc = self._lib.ilre_paged_append(
            self._h, batch.ref, spec.ref if spec is not None else None, _ptr(positions), _ptr(q), q_stride, _ptr(q_out),
            q_out_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, ctypes.byref(pool), _raw_stream(self._index))
        if rc != 0:
            raise IlreError(rc, "ilre_paged_append")
        return q_out

    def attention(self, batch: PagedBatch, q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                  stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """Every new token over its sequence's cached rows up to itself: (out like q, lse fp32 [n_tokens, n_q_heads]
        or None).  Rows of tokens that belong to no sequence are left as they are."""
        if stream is not None:
            with _on_stream(stream, self._index, (q, k_pool, v_pool, out, lse, batch.q_start, batch.kv_len, batch.block_table)):
                return self.attention(batch, q, k_pool, v_pool, out, lse, want_lse)
        q_stride = self._q(batch, q)
        pool = self._pool(batch, k_pool, v_pool, None)
        shape = (batch.n_tokens, self._n_q, self._dim)
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        if not (out.shape == shape and out.dtype == self.dtype and out.is_contiguous() and out.get_device() == self._index):
            raise AssertionError("out is not a contiguous tensor like q")
        self._lse(batch, lse)
        rc = self._lib.ilre_paged_attention(self._h, batch.ref, q.data_ptr(), q_stride, ctypes.byref(pool), out.data_ptr(),
                                            _ptr(lse), _raw_stream(self._index))
        if rc != 0:
            raise IlreError(rc, "ilre_paged_attention")
        return out, lse

    def _lse(self, batch: PagedBatch, lse: Optional[torch.Tensor]) -> None:
        if not (lse is None or (lse.shape == (batch.n_tokens, self._n_q) and lse.dtype == torch.float32 and
                               lse.is_contiguous() and lse.get_device() == self._index)):
            raise AssertionError("lse is not a contiguous fp32 tensor [n_tokens, n_q_heads]")

    def accumulate(self, batch: PagedBatch, q: torch.Tensor, lse: torch.Tensor, k_pool: torch.Tensor,
                   w_pool: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Adds to w_pool the attention weight that every cached row received from the batch's new tokens (q and lse
        as ``attention`` had and returned them).  Returns w_pool."""
        if stream is not None:
            with _on_stream(stream, self._index, (q, lse, k_pool, w_pool, batch.q_start, batch.kv_len, batch.block_table)):
                return self.accumulate(batch, q, lse, k_pool, w_pool)
        q_stride = self._q(batch, q)
        if lse is None or w_pool is None:
            raise AssertionError("lse and w_pool are needed")
        self._lse(batch, lse)
        pool = self._pool(batch, k_pool, None, w_pool)
        rc = self._lib.ilre_paged_accumulate(self._h, batch.ref, q.data_ptr(), q_stride, lse.data_ptr(), ctypes.byref(pool),
                                             _raw_stream(self._index))
        if rc != 0:
            raise IlreError(rc, "ilre_paged_accumulate")
        return w_pool

    def evict(self, batch: PagedBatch, budget: int, n_sink: int, n_recent: int, k_pool: torch.Tensor,
              v_pool: torch.Tensor, w_pool: torch.Tensor, per_head: bool = False,
              dst_table: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None,
              new_len: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """Cuts every sequence to ``budget`` rows: its first n_sink, its last n_recent and the heaviest between them,
        moved to rows 0, 1, ... of its own pages or of dst_table's (int32 [n_seqs, dst_blocks]).  Returns (kept
        int32 [n_seqs, n_kv_heads or 1, budget], ascending, -1 behind a shorter sequence; new_len int32 [n_seqs],
        0 where a sequence's length was out of range; it may be batch.kv_len, which keeps such an entry)."""
        if stream is not None:
            with _on_stream(stream, self._index, (k_pool, v_pool, w_pool, dst_table, kept, new_len, batch.kv_len, batch.block_table)):
                return self.evict(batch, budget, n_sink, n_recent, k_pool, v_pool, w_pool, per_head, dst_table, kept, new_len)
        _int32(budget, n_sink, n_recent)
        n, index = batch.kv_len.numel(), self._index
        shape = (n, self._page_shape[1] if per_head else 1, budget)
        if budget < 1 or w_pool is None:
            raise AssertionError("a budget of at least 1 and w_pool are needed")
        pool = self._pool(batch, k_pool, v_pool, w_pool)
        dst_blocks = 0
        if dst_table is not None:
            if not (dst_table.get_device() == index and dst_table.dtype == torch.int32 and dst_table.is_contiguous()):
                raise AssertionError("dst_table is not a contiguous int32 tensor of the cache's device")
            if dst_table.dim() != 2 or dst_table.shape[0] != n:
                raise AssertionError("dst_table [n_seqs, dst_blocks]")
            dst_blocks = dst_table.shape[1]
        if kept is None:
            kept = torch.empty(shape, dtype=torch.int32, device=self.device)
        else:
            if not (kept.shape == shape and kept.dtype == torch.int32 and kept.is_contiguous() and kept.get_device() == index):
                raise AssertionError("kept of another shape, type or device")
        if new_len is None:
            new_len = torch.empty(n, dtype=torch.int32, device=self.device)
        else:
            _ints(new_len, index, n)
        rc = self._lib.ilre_paged_evict(self._h, batch.ref, budget, n_sink, n_recent, int(per_head), ctypes.byref(pool),
                                        _ptr(dst_table), dst_blocks, kept.data_ptr(), new_len.data_ptr(), _raw_stream(index))
        if rc != 0:
            raise IlreError(rc, "ilre_paged_evict")
        return kept, new_len

    # -- diagnostics -------------------------------------------------------------------
    def status(self) -> int:
        return self._lib.ilre_paged_status(self._h)

    def check_status(self) -> None:
        rc = self.status()
        if rc != 0:
            raise IlreError(rc, "ilre_paged_status")

    def check_guards(self) -> int:
        """Number of workspace buffers whose guard zone was written to (0 = none); synchronises."""
        rc = self._lib.ilre_paged_check_guards(self._h)
        if rc < 0:
            raise IlreError(rc, "ilre_paged_check_guards")
        return rc

    def last_launch_count(self) -> int:
        return self._lib.ilre_paged_last_launch_count(self._h)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.ilre_paged_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
