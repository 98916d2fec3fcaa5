"""Torch-side buffers for one batch of stacked prompts over a paged cache.

PyTorch only provides device memory and the stream here.  A PagedBatch owns
the block tables, the stack of free pages and, per layer, the pages; it fills
``ippd_paged_batch_t`` and forwards every operation to libippd.

A decode step of a model, with one row per question:

    db.reserve(new, rows, Nt, slots, positions, served)     # once a step
    db.plan()
    for layer in range(layers):                              # q, k, v: views of the layer's projection
        db.append(layer, slots, positions, k, v, q, q_rot)
        db.decode(layer, q_rot, out, lse)

Calls on one PagedBatch follow each other on one stream: they share its tables,
plan and workspace.  Its decode calls on two streams at once need the C entry
points, with a workspace each.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import _lib as L
from .session import torch_dtype

# the current stream's handle without a Stream object around it (0.1 against 1.1 us)
_raw_stream = torch._C._cuda_getCurrentRawStream


class PagedBatch:
    """Prompts with ``q_count`` questions each on one GPU; sequences 0..B-1 are their
    contexts, B..B+Nt-1 the questions' segments, all empty at first.  ``q_count`` is
    fixed: a prompt that takes the place of one that ended has at most as many
    questions, the rest of the place staying inactive and empty.

    Tables and pages are made here (every page free, page 0 taken first) unless
    tensors that the caller keeps are given: seq_len int32 [B+Nt], block_table
    int32 [B+Nt, table_pages], free_pages int32 [num_pages], free_count int32
    [1], active uint8 [Nt], and per layer k_pages [num_pages, Hkv, page_tokens,
    D] and v_pages [num_pages, Hkv, page_tokens / 8, D, 8].
    """

    def __init__(self, q_count: Sequence[int], hq: int, hkv: int, head_dim: int, dtype: str, page_tokens: int,
                 num_pages: int, table_pages: int, rope_base: float = 10000.0, scale: float = 0.0,
                 max_questions: Optional[int] = None, layers: int = 1, device: str = "cuda",
                 seq_len: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                 free_pages: Optional[torch.Tensor] = None, free_count: Optional[torch.Tensor] = None,
                 active: Optional[torch.Tensor] = None, k_pages: Optional[Sequence[torch.Tensor]] = None,
                 v_pages: Optional[Sequence[torch.Tensor]] = None):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index if self.device.type == "cuda" else None
        self.dtype = dtype
        self.tdtype = torch_dtype(dtype)
        self.q_count = np.asarray(q_count, dtype=np.int64)
        self.B, self.Nt = len(self.q_count), int(self.q_count.sum())
        self.hq, self.hkv, self.D = hq, hkv, head_dim
        self.page_tokens, self.num_pages, self.table_pages = page_tokens, num_pages, table_pages
        self.max_questions = int(max_questions if max_questions is not None else max(1, int(self.q_count.max())))
        n, nt, dev = self.B + self.Nt, max(self.Nt, 1), self.device
        i32 = torch.int32
        q_start = np.concatenate([[0], np.cumsum(self.q_count)]).astype(np.int32)
        self.q_start = torch.from_numpy(q_start).to(dev)

        def own(t, name, shape, dt, make):
            if t is None:
                return make()
            self._expect(t, name, shape, dt)
            return t

        self.seq_len = own(seq_len, "seq_len", (n,), i32, lambda: torch.zeros(n, dtype=i32, device=dev))
        self.block_table = own(block_table, "block_table", (n, table_pages), i32,
                               lambda: torch.zeros(n, table_pages, dtype=i32, device=dev))
        self.free_pages = own(free_pages, "free_pages", (num_pages,), i32,
                              lambda: torch.arange(num_pages - 1, -1, -1, dtype=i32, device=dev))
        self.free_count = own(free_count, "free_count", (1,), i32,
                              lambda: torch.full((1,), num_pages, dtype=i32, device=dev))
        self.active = own(active, "active", (self.Nt,), torch.uint8,
                          lambda: torch.ones(nt, dtype=torch.uint8, device=dev))
        self.err = torch.zeros(1, dtype=i32, device=dev)
        if (k_pages is None) != (v_pages is None):
            raise ValueError("give the pages of keys and of values, or neither")
        kshape = (num_pages, hkv, page_tokens, head_dim)
        vshape = (num_pages, hkv, page_tokens // 8, head_dim, 8)
        if k_pages is None:
            self.k_pages = [torch.empty(kshape, dtype=self.tdtype, device=dev) for _ in range(layers)]
            self.v_pages = [torch.empty(vshape, dtype=self.tdtype, device=dev) for _ in range(layers)]
        else:
            self.k_pages, self.v_pages = list(k_pages), list(v_pages)
            if len(self.k_pages) != len(self.v_pages):
                raise ValueError("as many layers of value pages as of key pages")
            for k, v in zip(self.k_pages, self.v_pages):
                self._expect(k, "k_pages", kshape, self.tdtype)
                self._expect(v, "v_pages", vshape, self.tdtype)
        self.layers = len(self.k_pages)
        bt = L.IppdPagedBatch()
        bt.num_prompts, bt.num_questions = self.B, self.Nt
        bt.num_q_heads, bt.num_kv_heads, bt.head_dim = hq, hkv, head_dim
        bt.dtype = L.IPPD_DTYPE_F32 if dtype == "f32" else L.IPPD_DTYPE_BF16
        bt.page_tokens, bt.num_pages, bt.table_pages = page_tokens, num_pages, table_pages
        bt.max_questions = self.max_questions
        bt.rope_base, bt.scale = rope_base, scale
        bt.q_start, bt.seq_len, bt.block_table = self.q_start.data_ptr(), self.seq_len.data_ptr(), self.block_table.data_ptr()
        bt.free_pages, bt.free_count = self.free_pages.data_ptr(), self.free_count.data_ptr()
        # (an empty tensor has no address; a batch without questions reads none)
        bt.active = self.active.data_ptr() or self.err.data_ptr()
        bt.err_flag = self.err.data_ptr()
        self.batch = bt
        self.pages = []
        for k, v in zip(self.k_pages, self.v_pages):
            pg = L.IppdPages()
            pg.k, pg.v = k.data_ptr(), v.data_ptr()
            self.pages.append(pg)
        self.plan_bytes = L.ippd_paged_plan_bytes(bt)
        self.ws_bytes = L.ippd_paged_workspace_bytes(bt)
        if self.plan_bytes == 0 or self.ws_bytes == 0:
            raise ValueError("sizes outside the library's limits (see ippd_paged_batch_t)")
        self.plan_buf = torch.zeros(self.plan_bytes, dtype=torch.uint8, device=dev)
        self.ws = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=dev)

    # ------------------------------------------------------------------ helpers
    # A decode step makes a few calls a layer of some microseconds each, so the
    # checks below are a handful of attribute reads per tensor.
    def _expect(self, t: torch.Tensor, name: str, shape, dtype) -> int:
        """The address of a contiguous tensor of this shape and type on the batch's device."""
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name}: {dtype} {tuple(shape)} on {self.device}, contiguous")
        return t.data_ptr()

    def _row_stride(self, t: torch.Tensor, name: str, rows: int, heads: int) -> int:
        """Elements between the rows of [rows, heads * D] or [rows, heads, D], whose heads lie together."""
        shape, stride = t.shape, t.stride()
        flat = shape == (rows, heads * self.D) and stride[1] == 1
        if t.dtype is not self.tdtype or t.device != self.device or not (
                flat or (shape == (rows, heads, self.D) and stride[2] == 1 and (heads == 1 or stride[1] == self.D))):
            raise ValueError(f"{name}: {self.tdtype} [{rows}, {heads}, {self.D}] on {self.device}, a row's elements together")
        return stride[0] if rows > 1 else heads * self.D

    def _call(self, fn, *args) -> None:
        """fn(batch, *args, current stream of the batch's device), with that device the current one."""
        if self._index is None:
            raise ValueError("the batch's buffers are not on a GPU")
        if torch.cuda.current_device() == self._index:
            fn(self.batch, *args, _raw_stream(self._index))
        else:
            with torch.cuda.device(self._index):
                fn(self.batch, *args, _raw_stream(self._index))

    def err_flag(self) -> int:
        return int(self.err.item())

    def set_active(self, mask) -> None:
        m = torch.as_tensor(np.asarray(mask, dtype=np.uint8))
        self.active[: self.Nt].copy_(m.to(self.device))

    # ------------------------------------------------------------------ operators
    def reserve(self, new_tokens: torch.Tensor, token_start: torch.Tensor, num_rows: int, slot_map: torch.Tensor,
                positions: torch.Tensor, served: torch.Tensor) -> None:
        """Lengths, tables and slots of a change of the sequences: see ippd_paged_reserve."""
        n, i32 = self.B + self.Nt, torch.int32
        self._call(L.ippd_paged_reserve, self._expect(new_tokens, "new_tokens", (n,), i32),
                   self._expect(token_start, "token_start", (n + 1,), i32), num_rows,
                   self._expect(slot_map, "slot_map", (num_rows,), i32),
                   self._expect(positions, "positions", (num_rows,), i32), self._expect(served, "served", (n,), i32))

    def append(self, layer: int, slot_map: torch.Tensor, positions: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               q: Optional[torch.Tensor] = None, q_rot: Optional[torch.Tensor] = None) -> None:
        """Rotate the rows' tokens and write them into a layer's pages; with q, its rotation into q_rot."""
        rows = slot_map.shape[0]
        sm = self._expect(slot_map, "slot_map", (rows,), torch.int32)
        ps = self._expect(positions, "positions", (rows,), torch.int32)
        ks, vs = self._row_stride(k, "k", rows, self.hkv), self._row_stride(v, "v", rows, self.hkv)
        qs, qp, qr = 0, None, None
        if q is not None:
            if q_rot is None:
                raise ValueError("q needs q_rot")
            qs, qp = self._row_stride(q, "q", rows, self.hq), q.data_ptr()
            qr = self._expect(q_rot, "q_rot", (rows, self.hq, self.D), self.tdtype)
        if rows:
            self._call(L.ippd_paged_append, self.pages[layer], rows, sm, ps, qp, qs, k.data_ptr(), ks, v.data_ptr(), vs, qr)

    def plan(self) -> None:
        """Plan this step's attention from the lengths and active flags (once for all layers)."""
        self._call(L.ippd_paged_plan, self.plan_buf.data_ptr(), self.plan_bytes)

    def decode(self, layer: int, q_rot: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None) -> None:
        """The planned step's attention over a layer's pages: q_rot, out [Nt, Hq, D], lse float32 [Nt, Hq]."""
        if self.Nt == 0:
            return
        shape = (self.Nt, self.hq, self.D)
        qp, op = self._expect(q_rot, "q_rot", shape, self.tdtype), self._expect(out, "out", shape, self.tdtype)
        lp = None if lse is None else self._expect(lse, "lse", shape[:2], torch.float32)
        self._call(L.ippd_paged_decode_attention, self.pages[layer], self.plan_buf.data_ptr(), self.plan_bytes, qp, op,
                   lp, self.ws.data_ptr(), self.ws_bytes)
