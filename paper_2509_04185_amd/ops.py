"""Operators without a context: page tables, the paged e4m3 cache, the block-scaled e4m3 product.

Argument marshalling over the C ABI (``include/sbd.h`` has each call's semantics), as binding.py
does for ``Sbd``: tensors are checked for device, type and layout here, everything else by the
library.  A call enqueues on torch's current stream of its tensors' device and returns at once;
outputs and workspaces are allocated by torch on that stream, and the caller orders the use of
its own tensors on other streams, as for any torch operation.

An attention layer of a serving step, with ``pages`` shared by all layers:

    step = pages.plan(n_new, rows)                       # tables, slots and lengths of this step
    xq, xs = scaled_quantize(x)                          # activations, a scale per row and 128
    q, k, v = ...scaled_matmul(xq, xs, w_qkv, w_scale)... rotated by the caller
    kv.append(step, k, v)
    o = kv.attend(step, q, n_causal=n_causal)
    pages.cached += n_commit                             # after the last layer
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .binding import PagedKVArgs, PageTableArgs, _check, load_library

TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}  # SBD_TYPE_*
_HALVES = (torch.bfloat16, torch.float16)
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream  # no objects made on the way


def _run(fn, device: torch.device, where: str, *args):
    """fn(stream, *args) with the tensors' device as the current one, on torch's current stream of it."""
    index = device.index
    if index == _device():
        st = fn(_raw_stream(index), *args)
    else:
        with torch.cuda.device(index):
            st = fn(_raw_stream(index), *args)
    if st != 0:
        _check(load_library(), st, where)


def _tensor(t, what: str, dtype, shape, device=None):
    """t's address; a ValueError unless it is a contiguous CUDA tensor of that type and shape."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{what}: expected a CUDA tensor" + (f" on {device}" if device is not None else ""))
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)}, got "
                         f"{t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, what: str, heads: int, dim: int, device):
    """Address and row stride of [rows][heads][dim] on `device` (a CUDA one) whose rows may lie apart."""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise ValueError(f"{what}: expected a CUDA tensor on {device}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or t.dtype not in _HALVES:
        raise ValueError(f"{what}: expected bfloat16 or float16 [rows][{heads}][{dim}], got {t.dtype} {tuple(shape)}")
    n = shape[0]
    if n and (stride[2] != 1 or (heads > 1 and stride[1] != dim)):
        raise ValueError(f"{what}: the heads of a row must be contiguous (strides {stride})")
    return t.data_ptr(), (stride[0] if n > 1 else heads * dim)


class PagedStep:
    """The rows of one step: which sequence, page and offset each belongs to (from PageTable.plan,
    or made by hand from tensors of the same meaning)."""

    def __init__(self, table: torch.Tensor, row_start: torch.Tensor, kv_len: torch.Tensor, slots: torch.Tensor,
                 page_size: int):
        batch, width = table.shape
        dev = table.device
        _tensor(table, "table", torch.int32, (batch, width))
        _tensor(row_start, "row_start", torch.int32, (batch + 1,), dev)
        _tensor(kv_len, "kv_len", torch.int32, (batch,), dev)
        _tensor(slots, "slots", torch.int32, (slots.numel(),), dev)
        self.row_start, self.kv_len, self.slots = row_start, kv_len, slots
        self._set(table, page_size, slots.numel(), row_start.data_ptr(), kv_len.data_ptr(), slots.data_ptr())

    def _set(self, table, page_size, rows, p_row_start, p_kv_len, p_slots):
        self.table, self.page_size, self.rows = table, page_size, rows
        self.batch, self.max_pages = table.shape
        self.p_table, self.p_row_start, self.p_kv_len, self.p_slots = table.data_ptr(), p_row_start, p_kv_len, p_slots

    @classmethod
    def _of_buffer(cls, table, page_size, rows, buf):
        """From one int32 buffer that holds slots [rows], row_start [batch + 1], kv_len [batch], ..."""
        self = cls.__new__(cls)
        p, batch = buf.data_ptr(), table.shape[0]
        self.buf = buf
        self._set(table, page_size, rows, p + 4 * rows, p + 4 * (rows + batch + 1), p)
        return self

    def __getattr__(self, name):  # the views of a planned step are made when one is asked for
        buf = self.__dict__.get("buf")
        if buf is None or name not in ("row_start", "kv_len", "slots"):
            raise AttributeError(name)
        r, b = self.rows, self.batch
        self.slots, self.row_start, self.kv_len, _ = buf.split_with_sizes((r, b + 1, b, buf.numel() - r - 2 * b - 1))
        return self.__dict__[name]


class PageTable:
    """Page tables of `batch` sequences over a pool of pages, kept on the GPU (sbd_page_table).

    The tensors are the caller's to read; it changes only `cached`, by adding the committed
    rows of a step before the next plan."""

    def __init__(self, table: torch.Tensor, held: torch.Tensor, cached: torch.Tensor, free_list: torch.Tensor,
                 free_count: torch.Tensor, page_size: int):
        self.lib = load_library()
        self.batch, self.max_pages = table.shape
        self.n_pages, self.page_size, self.device = free_list.numel(), int(page_size), table.device
        self.table, self.held, self.cached, self.free_list, self.free_count = table, held, cached, free_list, free_count
        i, d = torch.int32, self.device
        self.args = PageTableArgs(self.batch, self.max_pages, self.n_pages, self.page_size,
                                  _tensor(table, "table", i, table.shape),
                                  _tensor(held, "held", i, (self.batch,), d),
                                  _tensor(cached, "cached", i, (self.batch,), d),
                                  _tensor(free_list, "free_list", i, (self.n_pages,), d),
                                  _tensor(free_count, "free_count", i, (1,), d))
        self._p = ctypes.addressof(self.args)

    @classmethod
    def empty(cls, batch: int, max_seq_len: int, n_pages: int, page_size: int, device="cuda"):
        """Tables of `batch` sequences of up to max_seq_len tokens that hold nothing yet."""
        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)
        width = max(1, -(-int(max_seq_len) // int(page_size)))
        return cls(ints(batch, width) - 1, ints(batch), ints(batch),
                   torch.arange(n_pages, dtype=torch.int32, device=device), ints(1) + n_pages, page_size)

    def plan(self, n_new: torch.Tensor, rows: int, release: Optional[torch.Tensor] = None) -> PagedStep:
        """sbd_paged_plan: n_new int32 [batch], rows the rows of the step's tensors, release uint8
        [batch] or None.  The step's kv_len is 0 for a sequence that could not be served."""
        B, rows, dev = self.batch, int(rows), self.device
        p_new = _tensor(n_new, "n_new", torch.int32, (B,), dev)
        p_rel = None if release is None else _tensor(release, "release", torch.uint8, (B,), dev)
        if rows < 0:
            raise ValueError(f"rows {rows} is negative")
        buf = torch.empty(rows + 5 * B + 3, dtype=torch.int32, device=dev)
        step = PagedStep._of_buffer(self.table, self.page_size, rows, buf)
        _run(self.lib.sbd_paged_plan, dev, "sbd_paged_plan", self._p, p_new, p_rel, rows, step.p_row_start,
             step.p_kv_len, step.p_slots, step.p_kv_len + 4 * B)
        return step


class PagedKV:
    """One layer's keys and values in pages of e4m3 codes with a power of two for each page and
    KV head (sbd_paged_kv).  The tensors are the caller's."""

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
        self.lib = load_library()
        if k_codes.dim() != 4:
            raise ValueError("k_codes: expected [n_pages][n_kv_heads][page_size][head_dim]")
        n, H, P, dh = k_codes.shape
        d = self.device = k_codes.device
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = n, H, P, dh
        self.k_codes, self.v_codes, self.k_exp, self.v_exp = k_codes, v_codes, k_exp, v_exp
        self.args = PagedKVArgs(n, P, H, dh, _tensor(k_codes, "k_codes", torch.uint8, (n, H, P, dh)),
                                _tensor(v_codes, "v_codes", torch.uint8, (n, H, dh, P), d),
                                _tensor(k_exp, "k_exp", torch.int8, (n, H), d),
                                _tensor(v_exp, "v_exp", torch.int8, (n, H), d))
        self._p = ctypes.addressof(self.args)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, device="cuda"):
        def codes(*shape):
            return torch.empty(shape, dtype=torch.uint8, device=device)
        def exps():
            return torch.zeros((n_pages, n_kv_heads), dtype=torch.int8, device=device)
        return cls(codes(n_pages, n_kv_heads, page_size, head_dim), codes(n_pages, n_kv_heads, head_dim, page_size),
                   exps(), exps())

    def _step(self, step: PagedStep, t: torch.Tensor, what: str):
        if step.table.device != self.device or step.page_size != self.page_size:
            raise ValueError(f"the step has pages of {step.page_size} on {step.table.device}, the cache of "
                             f"{self.page_size} on {self.device}")
        if t.shape[0] != step.rows:
            raise ValueError(f"{what}: {t.shape[0]} rows, the step has {step.rows}")

    def append(self, step: PagedStep, k: torch.Tensor, v: torch.Tensor):
        """sbd_paged_append: the step's keys (after RoPE) and values [rows][n_kv_heads][head_dim],
        bfloat16 or float16; rows may be strided (slices of one projection's output)."""
        pk, sk = _rows(k, "k", self.n_kv_heads, self.head_dim, self.device)
        pv, sv = _rows(v, "v", self.n_kv_heads, self.head_dim, self.device)
        self._step(step, k, "k")
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError(f"k and v differ: {k.dtype} {tuple(k.shape)} and {v.dtype} {tuple(v.shape)}")
        _run(self.lib.sbd_paged_append, self.device, "sbd_paged_append", self._p, TYPES[k.dtype], step.batch, step.rows,
             step.p_row_start, step.p_slots, pk, sk, pv, sv)

    def attend(self, step: PagedStep, q: torch.Tensor, n_causal: Optional[torch.Tensor] = None,
               scale: Optional[float] = None, max_kv: Optional[int] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """sbd_paged_attention: q [rows][n_q_heads][head_dim] -> out of the same shape and type.

        n_causal int32 [batch] or None (every row causal); scale defaults to 1 / sqrt(head_dim);
        max_kv: about the longest kv_len where the caller knows it (default: the table's width),
        for speed only.  Padding rows of a given `out` are left as they were, those of a new one
        hold anything."""
        if q.dim() != 3:
            raise ValueError("q: expected [rows][n_q_heads][head_dim]")
        n_q = q.shape[1]
        pq, sq = _rows(q, "q", n_q, self.head_dim, self.device)
        self._step(step, q, "q")
        p_nc = None if n_causal is None else _tensor(n_causal, "n_causal", torch.int32, (step.batch,), self.device)
        width = step.max_pages * self.page_size
        kv = width if max_kv is None else int(max_kv)
        need = ctypes.c_size_t(0)
        if out is None:
            out = torch.empty((step.rows, n_q, self.head_dim), dtype=q.dtype, device=self.device)
            po, so = out.data_ptr(), n_q * self.head_dim
        else:
            po, so = _rows(out, "out", n_q, self.head_dim, self.device)
            self._step(step, out, "out")
            if out.dtype != q.dtype:
                raise ValueError("out has another type than q")
        _check(self.lib, self.lib.sbd_paged_attention_workspace(self._p, step.batch, step.rows, n_q, kv,
                                                                ctypes.byref(need)), "sbd_paged_attention_workspace")
        ws = torch.empty(need.value, dtype=torch.uint8, device=self.device) if need.value else None
        _run(self.lib.sbd_paged_attention, self.device, "sbd_paged_attention", self._p, TYPES[q.dtype], step.batch,
             step.rows, n_q, step.p_row_start, step.p_kv_len, step.p_table, step.max_pages, p_nc,
             1.0 / math.sqrt(self.head_dim) if scale is None else float(scale), kv, pq, sq, po, so,
             None if ws is None else ws.data_ptr(), need.value)
        return out


def scaled_quantize(x: torch.Tensor, block_rows: int = 1):
    """sbd_scaled_quantize: (e4m3 codes uint8 [rows][cols], scales float32) of x [rows][cols]
    (bfloat16, float16 or float32; rows may be strided).  block_rows 1: activations, scales
    [ceil(cols / 128)][rows]; 128: weights, scales [ceil(rows / 128)][ceil(cols / 128)]."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 2 or x.dtype not in TYPES:
        raise ValueError("x: expected a CUDA matrix of bfloat16, float16 or float32")
    rows, cols = x.shape
    if rows and cols > 1 and x.stride(1) != 1:
        raise ValueError("x: the elements of a row must be contiguous")
    lib = load_library()
    kb = -(-cols // 128)
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    shape = (kb, rows) if block_rows == 1 else (-(-rows // 128), kb)
    scales = torch.empty(shape, dtype=torch.float32, device=x.device)
    _run(lib.sbd_scaled_quantize, x.device, "sbd_scaled_quantize", TYPES[x.dtype], rows, cols, x.data_ptr(),
         x.stride(0) if rows > 1 else cols, int(block_rows), codes.data_ptr(), scales.data_ptr())
    return codes, scales


def scaled_matmul(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                  out_dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sbd_scaled_matmul: [m][n] of e4m3 codes a uint8 [m][k] (rows may be strided), a_scale float32
    [ceil(k / 128)][m], b uint8 [n][k], b_scale float32 [ceil(n / 128)][ceil(k / 128)]."""
    if not isinstance(a, torch.Tensor) or not a.is_cuda or a.dim() != 2 or a.dtype != torch.uint8:
        raise ValueError("a: expected a CUDA matrix of e4m3 codes (uint8)")
    if not isinstance(b, torch.Tensor) or b.dim() != 2:
        raise ValueError("b: expected a CUDA matrix of e4m3 codes (uint8)")
    (m, k), n, dev = a.shape, b.shape[0], a.device
    if m and k > 1 and a.stride(1) != 1:
        raise ValueError("a: the elements of a row must be contiguous")
    kb = -(-k // 128)
    p_b = _tensor(b, "b", torch.uint8, (n, k), dev)
    p_bs = _tensor(b_scale, "b_scale", torch.float32, (-(-n // 128), kb), dev)
    p_as = _tensor(a_scale, "a_scale", torch.float32, (kb, m), dev)
    lib = load_library()
    need = ctypes.c_size_t(0)
    if out is None:
        if out_dtype not in TYPES:
            raise ValueError(f"out_dtype {out_dtype}: expected bfloat16, float16 or float32")
        out = torch.empty((m, n), dtype=out_dtype, device=dev)
    elif not out.is_cuda or out.device != dev or out.dtype not in TYPES or tuple(out.shape) != (m, n) or (
            m and n > 1 and out.stride(1) != 1):
        raise ValueError(f"out: expected a CUDA matrix of shape {(m, n)} with contiguous rows on {dev}")
    _check(lib, lib.sbd_scaled_matmul_workspace(m, n, k, ctypes.byref(need)), "sbd_scaled_matmul_workspace")
    ws = torch.empty(need.value, dtype=torch.uint8, device=dev) if need.value else None
    _run(lib.sbd_scaled_matmul, dev, "sbd_scaled_matmul", m, n, k, a.data_ptr(), a.stride(0) if m > 1 else k, p_as, p_b,
         p_bs, TYPES[out.dtype], out.data_ptr(), out.stride(0) if m > 1 else n, None if ws is None else ws.data_ptr(),
         need.value)
    return out
