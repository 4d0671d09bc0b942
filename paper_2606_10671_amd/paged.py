"""Paged window memory: sinks and a sliding window for many sequences at once.

A thin torch-facing owner of the library's paged store (include/fademem.h,
fademem_paged_*), beside ``fademem.Cache``: argument marshalling only.

    cache = PagedCache(seqs=4, pages=4096, page_tokens=64, heads=12, head_dim=128, max_tokens=1 << 20,
                       max_rows=4 * 4680, block_tokens=4680, window=4, sinks=1, grid=(30, 52))
    cache.plan(kept, added, rows=q.shape[0], max_new=4680)      # once a step
    for layer ...:                                              # q, k, v of the step's new tokens
        q = rotary.apply(q, cache.pos[:rows])
        cache.insert(k, v, layer, rotary=rotary)
        out = cache.attend(q, layer)
"""
from __future__ import annotations

from typing import Optional, Tuple

from . import fademem as fm
from .rotary import Rotary, empty_rows, rows_of


class PagedCache:
    """Owns a device pool and a handle of the paged store.

    Rows of a step are the new tokens of sequence 0, then of sequence 1, ...;
    tensors are [rows][heads][head_dim] in the store's dtype on its device,
    heads and elements contiguous.  All calls enqueue on torch's current
    stream of that device unless one is given.  After a plan, ``q_start``
    (int32 [seqs+1]), ``slots`` (int64 [max_rows]), ``pos`` (int32
    [max_rows][3]), ``status`` and ``held`` (int32 [seqs]), ``table`` (int32
    [seqs][pages of max_tokens]) and ``free`` (int32 [1]) are views of the
    step's plan on the device.  The store is for inference: no gradient passes
    through insert and attend.
    """

    def __init__(self, seqs: int, pages: int, page_tokens: int, heads: int, head_dim: int,
                 kv_heads: Optional[int] = None, dtype=None, layers: int = 1, max_tokens: Optional[int] = None,
                 max_rows: Optional[int] = None, block_tokens: int = 1, window: int = 0, sinks: int = 0,
                 grid: Tuple[int, int] = (1, 1), device=None):
        import torch
        self.handle = None
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("dtype must be torch.float32 or torch.bfloat16")
        kv_heads = heads if kv_heads is None else kv_heads
        # Left open: all that the pages hold, and a step of as much, up to what the library takes.
        max_tokens = min(pages * page_tokens, 1 << 30) if max_tokens is None else max_tokens
        max_rows = min(max_tokens, 1 << 23, (1 << 30) // max(1, heads // max(1, kv_heads))) if max_rows is None else max_rows
        self.torch_dtype = dtype
        self.cfg = fm.fademem_paged_config(
            seqs=seqs, layers=layers, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
            dtype=fm.FADEMEM_BF16 if dtype == torch.bfloat16 else fm.FADEMEM_F32, page_tokens=page_tokens, sinks=sinks,
            pages=pages, max_tokens=max_tokens, max_rows=max_rows, block_tokens=block_tokens, window=window,
            grid_h=grid[0], grid_w=grid[1])
        self.pool_bytes = fm.fademem_paged_bytes(self.cfg)
        device = torch.device("cuda" if device is None else device)
        if device.index is None:
            device = torch.device(device.type, torch.cuda.current_device())
        self.device = device
        self.rows = 0
        self._seqs, self._heads, self._kv_heads, self._dim = int(seqs), int(heads), int(kv_heads), int(head_dim)
        with torch.cuda.device(device):
            self.pool = torch.empty(self.pool_bytes, dtype=torch.uint8, device=device)
            self.handle = fm.fademem_paged_create(self.cfg, self.pool.data_ptr(), self.pool_bytes, fm.current_stream())
        self.q_start = self._array(fm.FADEMEM_PAGED_Q_START, torch.int32)
        self.slots = self._array(fm.FADEMEM_PAGED_SLOTS, torch.int64)
        self.pos = self._array(fm.FADEMEM_PAGED_POSITIONS, torch.int32).view(-1, 3)
        self.status = self._array(fm.FADEMEM_PAGED_STATUS, torch.int32)
        self.held = self._array(fm.FADEMEM_PAGED_HELD, torch.int32)
        self.table = self._array(fm.FADEMEM_PAGED_TABLE, torch.int32).view(seqs, -1)
        self.free = self._array(fm.FADEMEM_PAGED_FREE, torch.int32)

    def _array(self, which: int, dtype, layer: int = 0):
        import torch
        ptr, n = fm.fademem_paged_array(self.handle, which, layer)
        at = ptr - self.pool.data_ptr()
        return self.pool[at: at + n * torch.empty(0, dtype=dtype).element_size()].view(dtype)

    def _stream(self, stream) -> int:
        return fm.current_stream() if stream is None else int(stream.cuda_stream)

    def plan(self, kept, added, rows: int, max_new: int, stream=None):
        """A step: sequence s keeps its first kept[s] tokens and appends
        added[s] (int32 [seqs] tensors on the device); rows: rows of the step's
        tensors (at least the sum of added), max_new: the most that any
        added[s] is."""
        import torch
        for name, t in (("kept", kept), ("added", added)):
            if t.dtype != torch.int32 or t.shape != (self._seqs,) or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"{name}: expected a contiguous int32 [{self._seqs}] tensor on {self.device}")
        with fm.on_device(self.device.index):
            fm.fademem_paged_plan(self.handle, kept.data_ptr(), added.data_ptr(), rows, max_new, self._stream(stream))
        self.rows = rows

    def insert(self, k, v, layer: int = 0, rotary: Optional[Rotary] = None, stream=None):
        """The planned step's keys (turned by `rotary` to their positions) and
        values, [rows][kv_heads][head_dim], into the layer's pages."""
        k_stride = rows_of(k, "k", self.torch_dtype, self.device, self._kv_heads, self._dim, self.rows)
        v_stride = rows_of(v, "v", self.torch_dtype, self.device, self._kv_heads, self._dim, self.rows)
        with fm.on_device(self.device.index):
            fm.fademem_paged_insert(self.handle, layer, k.data_ptr(), k_stride, v.data_ptr(), v_stride,
                                    None if rotary is None else rotary.rope, self._stream(stream))

    def attend(self, q, layer: int = 0, scale: float = 0.0, out=None, lse=None, stream=None):
        """Attention of the planned step's queries, [rows][heads][head_dim],
        over the layer's pages.  Rows behind the last sequence's are left as
        they are in `out` and `lse` (float32 [heads][rows])."""
        import torch
        rows, heads, dim = self.rows, self._heads, self._dim
        q_stride = rows_of(q, "q", self.torch_dtype, self.device, heads, dim, rows)
        if out is None:
            out, out_stride = empty_rows((rows, heads, dim), self.torch_dtype, self.device, stream), heads * dim
        else:
            out_stride = rows_of(out, "out", self.torch_dtype, self.device, heads, dim, rows)
        if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != self.device
                                or lse.shape != (heads, rows)):
            raise ValueError("lse: expected a contiguous float32 [heads][rows] tensor")
        with fm.on_device(self.device.index):
            fm.fademem_paged_attend(self.handle, layer, q.data_ptr(), q_stride, scale, out.data_ptr(), out_stride,
                                    0 if lse is None else lse.data_ptr(), self._stream(stream))
        return out

    def pages(self, layer: int = 0):
        """The layer's pages, a [pages][2][kv_heads][page_tokens][head_dim] view (K, then V)."""
        c = self.cfg
        return self._array(fm.FADEMEM_PAGED_PAGES, self.torch_dtype, layer).view(c.pages, 2, c.kv_heads, c.page_tokens,
                                                                               c.head_dim)

    def close(self):
        if getattr(self, "handle", None):
            fm.fademem_paged_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
