"""Binding of the 8-bit paged KV cache (include/dvi.h): argument checks and
marshalling only.  The tensors are the caller's, and every call enqueues on
the caller's current stream (or the one it names).

The checks of append, attend and read and the library calls are made in the
CPython module _paged (csrc/paged_py.c): a decode step's calls take less time
on the GPU than ctypes and Python checks would take to enqueue them."""
from __future__ import annotations

import ctypes
import weakref
from typing import Optional, Tuple

import torch

from .dvi import DEV_BITS, DVIError, STATUS, lib

KV_FORMATS = {"int8": 0, "e4m3": 1}
_CODES = {"int8": (torch.int8,), "e4m3": (torch.uint8, torch.float8_e4m3fn)}
_TYPES = (torch.bfloat16, torch.float32)


# The current stream's handle, without the object around it (1.1 us on a Grace core)
# where torch has a way to it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
# Likewise a tensor on the current device (1.0 us, torch.empty 1.5; and a call 2 us less, as what
# runs between two launches pushes the launch's own code out of the caches).
_empty_strided = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)


class PagedCacheC(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int), ("n_kv_heads", ctypes.c_int), ("page_tokens", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("format", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class PagedBatchC(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int), ("max_pages", ctypes.c_int), ("n_rows", ctypes.c_int),
                ("max_rows", ctypes.c_int), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("row_start", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class PagedOptionsC(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int), ("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("window", ctypes.c_int), ("slopes", ctypes.c_void_p)]


_calls = None


def _module():
    """The CPython module with the library's entry points; raises if it was not built (there is no fallback)."""
    global _calls
    if _calls is None:
        L = lib()
        try:
            from . import _paged
        except ImportError as e:
            raise RuntimeError("_paged.so is missing: build it with `python -m paper_2510_05421_gb300.build`") from e
        append, attend, read, capture = (ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.dvi_paged_append, L.dvi_paged_attend, L.dvi_paged_read, L.dvi_paged_capture))
        _paged.init(append, attend, read, torch.int32, torch.float32, torch.bfloat16, capture)
        _calls = _paged
    return _calls


class _Workspaces:
    """attend's workspaces on one device and for one head_dim, shared by its caches (a stream's calls run one after
    another, whatever their cache): one for each stream, and one for the calls of the last capture on it.  A graph
    keeps its own, as it may be replayed beside other calls of the stream it was captured on.  Entries are (the
    tensor, its address, its size, the capture's id)."""

    def __init__(self):
        self.eager, self.captured = {}, {}


_workspaces = weakref.WeakValueDictionary()     # (device, head_dim): they go with their last cache


def rotary_table(n_pos: int, rot_dim: int, theta: float = 10000.0, device="cuda") -> torch.Tensor:
    """[n_pos, rot_dim / 2, 2] f32 (cos, sin) of p * theta^(-2 i / rot_dim), from 64-bit angles."""
    inv = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * inv
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous().to(device)


class PagedCache:
    """Keys and values of many sequences in pages of 8-bit codes.

    k, v: codes [n_pages, H_kv, P, head_dim] (torch.int8 for "int8"; uint8 or
    float8_e4m3fn for "e4m3"), k_scale, v_scale: f32 [n_pages, H_kv]; all
    contiguous on one GPU.  `create` allocates them.  Page tables (int32
    [B, max_pages]), lengths (int32 [B]) and the choice of pages are the
    caller's; a call's rows of sequence b take the positions lens[b],
    lens[b] + 1, ..., and lens itself is never written.

    Rows of a call lie sequence after sequence: with row_start None every
    sequence has the same number, else sequence b has rows row_start[b] ..
    row_start[b + 1] - 1 (int32 [B + 1]) and max_rows bounds the longest (the
    kernels are chosen by it: without it, by the rows of all sequences
    together, and single tokens pay for prompts that might be there).  Rows
    of no sequence (a buffer's unused end) are not written: in a tensor that
    the call made they hold anything.

    A call runs on the current stream.  With `stream` it runs there, behind
    what the current one has in flight; wait for that stream before its
    results are used elsewhere.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                 fmt: str = "int8"):
        if fmt not in KV_FORMATS:
            raise ValueError(f"PagedCache: fmt must be one of {sorted(KV_FORMATS)}")
        for t in (k, v):
            if t.dtype not in _CODES[fmt] or t.dim() != 4 or t.shape != k.shape:
                raise ValueError(f"PagedCache: k and v must be {fmt} codes [n_pages, H_kv, P, head_dim]")
        n_pages, H, P, D = k.shape
        if P not in (16, 32, 64, 128) or D not in (64, 128) or n_pages < 1 or not 1 <= H <= 1024:
            raise ValueError("PagedCache: pages of 16, 32, 64 or 128 tokens and head_dim 64 or 128")
        for t in (k_scale, v_scale):
            if t.dtype != torch.float32 or tuple(t.shape) != (n_pages, H):
                raise ValueError("PagedCache: k_scale and v_scale must be float32 [n_pages, H_kv]")
        for t in (k, v, k_scale, v_scale):
            if not t.is_contiguous() or not t.is_cuda or t.device != k.device:
                raise ValueError("PagedCache: the tensors must be contiguous and on one CUDA device")
            if t.data_ptr() % 16:
                raise ValueError("PagedCache: the tensors must be 16-byte aligned")
        self.k, self.v, self.k_scale, self.v_scale, self.fmt = k, v, k_scale, v_scale, fmt
        self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = n_pages, H, P, D
        self.device = k.device
        self._scale = D ** -0.5
        self._index = k.device.index
        self._one_device = torch.cuda.device_count() == 1
        self.status_word = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = PagedCacheC(n_pages, H, P, D, KV_FORMATS[fmt], k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                              v_scale.data_ptr())
        self._lib, self._calls = lib(), _module()
        self._at = (ctypes.addressof(self._c), self._index, self.status_word.data_ptr())
        self._spaces = _workspaces.setdefault((self._index, D), _Workspaces())

    @classmethod
    def create(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_tokens: int = 64, fmt: str = "int8",
               device="cuda") -> "PagedCache":
        """A cache of n_pages unused pages."""
        if fmt not in KV_FORMATS:
            raise ValueError(f"PagedCache: fmt must be one of {sorted(KV_FORMATS)}")
        td = torch.int8 if fmt == "int8" else torch.uint8
        shape = (n_pages, n_kv_heads, page_tokens, head_dim)
        return cls(torch.zeros(shape, dtype=td, device=device), torch.zeros(shape, dtype=td, device=device),
                   torch.ones(shape[:2], device=device), torch.ones(shape[:2], device=device), fmt)

    def _check(self, what, rc):
        if rc != 0:
            raise DVIError(f"{what}: {STATUS.get(rc, rc)}")

    def _on_device(self):
        """Whether the cache's device is current (the library launches on the current one)."""
        return self._one_device or self._index == torch.cuda.current_device()

    def _elsewhere(self, call, stream, *args):
        """`call` where the cache's device is not current, or on a stream of the caller's choice: there it waits for
        what the current stream has in flight (the inputs may be among it), and no tensor's memory is used again
        before both streams are done with it."""
        with torch.cuda.device(self._index):
            if stream is None:
                return call(*args)
            if stream.device != self.device:
                raise ValueError("stream: not on the cache's device")
            here = torch.cuda.current_stream(self._index)
            if here.cuda_stream == stream.cuda_stream:
                return call(*args)
            alone = not torch.cuda.is_current_stream_capturing()
            with torch.cuda.stream(stream):
                # (a capture cannot wait for work outside it)
                if not (alone and torch.cuda.is_current_stream_capturing()):
                    stream.wait_stream(here)
                got = call(*args)
            for t in (self.k, self.v, self.k_scale, self.v_scale, self.status_word, *args):
                if isinstance(t, torch.Tensor):
                    t.record_stream(stream)
            for t in got if isinstance(got, tuple) else (got,):
                if t is not None:
                    t.record_stream(here)
            return got

    def _new(self, shape, dtype):
        """An output (the cache's device is current)."""
        if _empty_strided is None or len(shape) != 3:
            return torch.empty(shape, dtype=dtype, device=self.device)
        n, heads, dim = shape
        return _empty_strided((n, heads, dim), (heads * dim, dim, 1), dtype)

    # -- calls ------------------------------------------------------------
    def append(self, table: torch.Tensor, lens: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               q: Optional[torch.Tensor] = None, rotary: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """Write rows k, v [n, H_kv, head_dim] (bf16 or f32) behind lens, the keys rotated by `rotary`
        ([n_pos, rot_dim / 2, 2], see rotary_table) at their positions.  Returns q [n, H_q, head_dim]
        rotated alike (into q_out, which may be q), or None without q."""
        if stream is not None or not self._on_device():
            return self._elsewhere(self.append, stream, table, lens, k, v, q, rotary, row_start, max_rows, q_out)
        if q is not None and q_out is None:
            q_out = self._new(q.shape, q.dtype)
        rc = self._calls.append(*self._at, table, lens, k, v, q, rotary, row_start, max_rows, q_out,
                                _raw_stream(self._index))
        if rc:
            self._check("append", rc)
        return q_out

    def attend(self, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None,
               softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of rows q [n, H_q, head_dim] (bf16 or f32), appended before at the same lens: the row at
        position p sees the held positions up to p (the last `window` of them).  scale: head_dim^-0.5 unless
        given; softcap c > 0: scores become c tanh(score / c); slopes f32 [H_q]: + slope (p_key - p)."""
        if stream is not None or not self._on_device():
            return self._elsewhere(self.attend, stream, table, lens, q, scale, softcap, window, slopes, row_start,
                                   max_rows, out)
        if out is None:
            out = self._new(q.shape, q.dtype)
        s = _raw_stream(self._index)
        capture = self._calls.capture(s)
        ws = (self._spaces.captured if capture else self._spaces.eager).get(s)
        if ws is None or ws[3] != capture:
            ws = self._workspace(s, capture)
        rc = self._calls.attend(*self._at, table, lens, q, out, self._scale if scale is None else scale, softcap, window,
                                slopes, row_start, max_rows, ws[1], ws[2], s)
        if rc:
            self._check("attend", rc)
        return out

    def read(self, table: torch.Tensor, lens: torch.Tensor, n_rows: int, row_start: Optional[torch.Tensor] = None,
             max_rows: Optional[int] = None, dtype: torch.dtype = torch.bfloat16,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Values of n_rows cached rows, positions lens[b], lens[b] + 1, ... of each sequence:
        (k, v) [n_rows, H_kv, head_dim] in dtype; zeros where no page is held."""
        if stream is not None or not self._on_device():
            return self._elsewhere(self.read, stream, table, lens, n_rows, row_start, max_rows, dtype)
        if dtype not in _TYPES or n_rows < 0:
            raise ValueError("read: dtype must be bfloat16 or float32, and n_rows at least 0")
        shape = (n_rows, self.n_kv_heads, self.head_dim)
        k = self._new(shape, dtype)
        v = self._new(shape, dtype)
        rc = self._calls.read(*self._at, table, lens, k, v, row_start, max_rows, _raw_stream(self._index))
        if rc:
            self._check("read", rc)
        return k, v

    def status(self) -> list:
        """Names of the DVI_DEV_* flags set since the last look (waits for the device: calls on any of its streams),
        then cleared."""
        torch.cuda.synchronize(self._index)
        word = int(self.status_word.item())
        if word:
            # only what is reported, and before any later call's flags
            self.status_word.bitwise_and_(~word)
            torch.cuda.synchronize(self._index)
        return [name for bit, name in DEV_BITS.items() if word & bit]

    def _workspace(self, stream: int, capture: int):
        """A workspace for the current stream's calls, or those of the capture that it is in: the memory is that
        stream's (the graph's), and its counters are cleared there, before the calls."""
        n = self._lib.dvi_paged_workspace_bytes(self.head_dim)
        ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        ws[:self._lib.dvi_paged_counter_bytes()].zero_()
        got = (ws, ws.data_ptr(), n, capture)
        (self._spaces.captured if capture else self._spaces.eager)[stream] = got
        return got
