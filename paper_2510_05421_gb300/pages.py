"""The pages of a paged cache handed out on the GPU (include/dvi.h, dvi_paged_plan)."""
from __future__ import annotations

import ctypes
import operator
from typing import NamedTuple, Optional, Union

import torch

from .dvi import DEV_BITS
from .paged import _raw_stream, elsewhere
from .sampling import _current, _module


class PagePoolC(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int), ("page_tokens", ctypes.c_int), ("n_seqs", ctypes.c_int),
                ("max_pages", ctypes.c_int), ("stack", ctypes.c_void_p), ("n_free", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("held", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class RowPlan(NamedTuple):
    """Where a pass's rows go: row_start int32 [B + 1]; slots int64 [n_rows] (page * P + position % P, -1 where the
    page is not held and behind the last row) and positions int32 [n_rows] (-1 behind the last row), or None."""
    row_start: torch.Tensor
    slots: Optional[torch.Tensor]
    positions: Optional[torch.Tensor]


_new_plan = tuple.__new__     # (a named tuple's own constructor takes 0.3 us)


class PagePool:
    """Pages of PagedCaches for B slots, planned on the GPU from the sequences' lengths.

    stack: int32 [n_pages], its first n_free (int32 [1]) entries the free pages, the last of them taken first; table:
    int32 [B, max_pages], a slot's pages in order and -1 behind them (what PagedCache's calls take); held: int32 [B]
    pages of each slot.  All contiguous on one GPU; `create` makes them for an unused cache.  One pool serves all
    caches that share a page table (one for each layer).

    A call runs on the current stream.  With `stream` it runs there, behind what the current one has in flight; wait
    for that stream before its results are used elsewhere."""

    def __init__(self, stack: torch.Tensor, n_free: torch.Tensor, table: torch.Tensor, held: torch.Tensor,
                 page_tokens: int = 64):
        page_tokens = operator.index(page_tokens)
        if page_tokens not in (16, 32, 64, 128):
            raise ValueError("PagePool: pages of 16, 32, 64 or 128 tokens")
        for t, dims in ((stack, 1), (n_free, 1), (table, 2), (held, 1)):
            if t.dtype != torch.int32 or t.dim() != dims:
                raise ValueError("PagePool: stack [n_pages], n_free [1], table [B, max_pages] and held [B] must be int32")
            if not t.is_cuda or t.device != stack.device or not t.is_contiguous():
                raise ValueError("PagePool: the tensors must be contiguous and on one CUDA device")
        B, width = table.shape
        if n_free.numel() != 1 or held.numel() != B:
            raise ValueError("PagePool: n_free must have one entry, held one for each row of the table")
        if not 1 <= B <= 1024 or not 1 <= width <= (1 << 30) // page_tokens or stack.numel() < 1:
            raise ValueError("PagePool: 1 to 1024 slots, tables of at most 2^30 positions, at least one page")
        self.stack, self.n_free, self.table, self.held, self.page_tokens = stack, n_free, table, held, page_tokens
        self.n_pages, self.n_seqs, self.max_pages = stack.numel(), B, width
        self.device, self._index = stack.device, stack.device.index
        self.status_word = torch.zeros(1, dtype=torch.int32, device=stack.device)
        self._c = PagePoolC(self.n_pages, page_tokens, B, width, stack.data_ptr(), n_free.data_ptr(), table.data_ptr(),
                            held.data_ptr(), self.status_word.data_ptr())
        self._calls, self._at = _module(), ctypes.addressof(self._c)
        self._tensors = (stack, n_free, table, held, self.status_word)

    @classmethod
    def create(cls, n_pages: int, n_seqs: int, max_pages: int, page_tokens: int = 64, device="cuda") -> "PagePool":
        """A pool of n_pages free pages (page 0 is taken first) and n_seqs slots that hold none."""
        return cls(torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.full((1,), n_pages, dtype=torch.int32, device=device),
                   torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_seqs, dtype=torch.int32, device=device), page_tokens)

    def plan(self, lens: torch.Tensor, rows: Union[int, torch.Tensor] = 0, n_rows: Optional[int] = None,
             stream=None) -> RowPlan:
        """Give every slot the pages that `rows` (int32 [B], or a number for all) more positions behind lens (int32
        [B]) need: pages past that go back to the stack, missing ones come off it, in order of the slots.  A slot whose
        missing pages are not all there, or not all in its table, gets none of them (KV_FULL) and is passed over.
        Returns the row starts, and with n_rows (how many rows the pass's buffers have) also slots and positions."""
        if stream is not None or _current() != self._index:
            got = elsewhere(self._index, stream, self._tensors, self._plan, (lens, rows, n_rows), "the pool's device")
        else:
            got = self._plan(lens, rows, n_rows)
        return _new_plan(RowPlan, got)

    def _plan(self, lens, rows, n_rows):
        return self._calls.plan(self._at, self._index, lens, rows, n_rows, True, _raw_stream(self._index))

    def trim(self, lens: torch.Tensor, stream=None) -> None:
        """Give back the pages past lens: of rejected rows, and (lens 0) of sequences that ended."""
        if stream is not None or _current() != self._index:
            elsewhere(self._index, stream, self._tensors, self.trim, (lens,), "the pool's device")
            return
        self._calls.plan(self._at, self._index, lens, 0, None, False, _raw_stream(self._index))

    def status(self) -> list:
        """Names of the DVI_DEV_* flags set since the last look (waits for the device), then cleared."""
        torch.cuda.synchronize(self._index)
        word = int(self.status_word.item())
        if word:
            self.status_word.bitwise_and_(~word)
            torch.cuda.synchronize(self._index)
        return [name for bit, name in DEV_BITS.items() if word & bit]
