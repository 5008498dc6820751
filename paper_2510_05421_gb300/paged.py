"""ctypes binding of the 8-bit paged KV cache (include/dvi.h): argument checks
and marshalling only.  The tensors are the caller's, and every call enqueues
on the caller's current stream (or the one it names)."""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from .dvi import DEV_BITS, DVI_BF16, DVI_F32, DVIError, STATUS, lib

KV_FORMATS = {"int8": 0, "e4m3": 1}
_CODES = {"int8": (torch.int8,), "e4m3": (torch.uint8, torch.float8_e4m3fn)}
_TYPES = {torch.bfloat16: (DVI_BF16, 2), torch.float32: (DVI_F32, 4)}


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


# PagedBatchC and PagedOptionsC as bytes: a pack is a fraction of a ctypes structure's cost, and a decode step's
# calls are short enough to notice
_BATCH = struct.Struct("@4i4Q")
_OPTIONS = struct.Struct("@iffiQ")
assert _BATCH.size == ctypes.sizeof(PagedBatchC) and _OPTIONS.size == ctypes.sizeof(PagedOptionsC)


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
    row_start[b + 1] - 1 (int32 [B + 1]) and max_rows bounds the longest.
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
        self._index = k.device.index
        self._one_device = torch.cuda.device_count() == 1
        self.status_word = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = PagedCacheC(n_pages, H, P, D, KV_FORMATS[fmt], k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                              v_scale.data_ptr())
        self._cref = ctypes.byref(self._c)
        self._status_ptr = self.status_word.data_ptr()
        self._lib = lib()
        self._workspaces = {}

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

    # -- marshalling ------------------------------------------------------
    def _batch(self, what, table, lens, n_rows, row_start, max_rows):
        """dvi_paged_batch of a call, as bytes."""
        i32, dev = torch.int32, self._index
        if table.dtype is not i32 or lens.dtype is not i32 or table.dim() != 2:
            raise ValueError(f"{what}: table must be int32 [B, max_pages] and lens int32 [B]")
        B, width = table.shape
        if lens.shape != (B,) or not (table.is_contiguous() and lens.is_contiguous()):
            raise ValueError(f"{what}: table and lens must be contiguous, with one row and one length a sequence")
        if table.get_device() != dev or lens.get_device() != dev:
            raise ValueError(f"{what}: table and lens must be on {self.device}")
        if not 1 <= B <= 1024 or not 1 <= width <= (1 << 30) // self.page_tokens:
            raise ValueError(f"{what}: 1 to 1024 sequences of 1 to {(1 << 30) // self.page_tokens} pages")
        start = 0
        if row_start is None:
            if n_rows % B:
                raise ValueError(f"{what}: {n_rows} rows do not divide into {B} sequences (give row_start)")
            max_rows = n_rows // B
        else:
            if row_start.dtype is not i32 or row_start.shape != (B + 1,) or not row_start.is_contiguous() or \
                    row_start.get_device() != dev:
                raise ValueError(f"{what}: row_start must be contiguous int32 [B + 1] on {self.device}")
            start = row_start.data_ptr()
            max_rows = n_rows if max_rows is None else min(max_rows, n_rows)
            if max_rows < 0:
                raise ValueError(f"{what}: max_rows must not be negative")
        return _BATCH.pack(B, width, n_rows, max_rows, table.data_ptr(), lens.data_ptr(), start, self._status_ptr)

    def _rows(self, what, t, heads, dtype, esz, n_rows):
        """Elements from row to row of t [n_rows, heads, head_dim], whose rows may lie apart, and its address."""
        D = self.head_dim
        if t.dtype is not dtype or t.shape != (n_rows, heads, D):
            raise ValueError(f"{what} must be {dtype} [{n_rows}, {heads}, {D}], got {t.dtype} {tuple(t.shape)}")
        ld, sh, sd = t.stride()
        if n_rows <= 1:
            ld = heads * D
        if sd != 1 or (sh != D and heads > 1) or ld < heads * D:
            raise ValueError(f"{what}: each row's heads must be contiguous")
        if t.get_device() != self._index:
            raise ValueError(f"{what} must be on {self.device}")
        p = t.data_ptr()
        if p % 16 or ld * esz % 16:
            raise ValueError(f"{what}: rows must start on 16-byte boundaries")
        return ld, p

    def _call(self, what, fn, *args):
        """fn(*args) with the cache's device current (the library launches on the current one)."""
        if self._one_device or self._index == torch.cuda.current_device():
            rc = fn(*args)
        else:
            with torch.cuda.device(self._index):
                rc = fn(*args)
        if rc != 0:
            raise DVIError(f"{what}: {STATUS.get(rc, rc)}")

    def _stream(self, stream):
        return (torch.cuda.current_stream(self._index) if stream is None else stream).cuda_stream

    # -- calls ------------------------------------------------------------
    def append(self, table: torch.Tensor, lens: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               q: Optional[torch.Tensor] = None, rotary: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """Write rows k, v [n, H_kv, head_dim] (bf16 or f32) behind lens, the keys rotated by `rotary`
        ([n_pos, rot_dim / 2, 2], see rotary_table) at their positions.  Returns q [n, H_q, head_dim]
        rotated alike (into q_out, which may be q), or None without q."""
        td = k.dtype
        if td not in _TYPES or k.dim() != 3:
            raise ValueError("append: k must be bfloat16 or float32 [n, H_kv, head_dim]")
        code, esz = _TYPES[td]
        n, H = k.shape[0], self.n_kv_heads
        bt = self._batch("append", table, lens, n, row_start, max_rows)
        ld_k, k_p = self._rows("append: k", k, H, td, esz, n)
        ld_v, v_p = self._rows("append: v", v, H, td, esz, n)
        rot_p, rot_dim, n_pos = None, 0, 0
        if rotary is not None:
            if rotary.dtype is not torch.float32 or rotary.dim() != 3 or rotary.shape[2] != 2 or \
                    not rotary.is_contiguous() or rotary.get_device() != self._index or rotary.data_ptr() % 16:
                raise ValueError(f"append: rotary must be contiguous float32 [n_pos, rot_dim / 2, 2] on {self.device}")
            n_pos, rot_dim = rotary.shape[0], 2 * rotary.shape[1]
            if rot_dim % 16 or not 16 <= rot_dim <= self.head_dim or n_pos < 1:
                raise ValueError("append: rot_dim must be a multiple of 16 up to head_dim")
            rot_p = rotary.data_ptr()
        q_p = o_p = None
        ld_q = ld_o = heads = 0
        if q is not None:
            if q.dim() != 3 or q.shape[1] < 1:
                raise ValueError("append: q must be [n, H_q, head_dim]")
            heads = q.shape[1]
            ld_q, q_p = self._rows("append: q", q, heads, td, esz, n)
            if q_out is None:
                q_out = torch.empty((n, heads, self.head_dim), dtype=td, device=self.device)
                ld_o, o_p = heads * self.head_dim, q_out.data_ptr()
            else:
                ld_o, o_p = self._rows("append: q_out", q_out, heads, td, esz, n)
        elif q_out is not None:
            raise ValueError("append: q_out without q")
        self._call("append", self._lib.dvi_paged_append, self._cref, bt, code, k_p, ld_k, v_p, ld_v, rot_p, rot_dim,
                   n_pos, q_p, ld_q, o_p, ld_o, heads, self._stream(stream))
        return q_out

    def attend(self, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None,
               softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of rows q [n, H_q, head_dim] (bf16 or f32), appended before at the same lens: the row at
        position p sees the held positions up to p (the last `window` of them).  scale: head_dim^-0.5 unless
        given; softcap c > 0: scores become c tanh(score / c); slopes f32 [H_q]: + slope (p_key - p)."""
        td = q.dtype
        if td not in _TYPES or q.dim() != 3:
            raise ValueError("attend: q must be bfloat16 or float32 [n, H_q, head_dim]")
        code, esz = _TYPES[td]
        n, heads = q.shape[0], q.shape[1]
        if heads < 1 or heads % self.n_kv_heads:
            raise ValueError(f"attend: {heads} heads do not divide over {self.n_kv_heads} KV heads")
        bt = self._batch("attend", table, lens, n, row_start, max_rows)
        ld_q, q_p = self._rows("attend: q", q, heads, td, esz, n)
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=td, device=self.device)
            ld_o, o_p = heads * self.head_dim, out.data_ptr()
        else:
            ld_o, o_p = self._rows("attend: out", out, heads, td, esz, n)
        slopes_p = 0
        if slopes is not None:
            if slopes.dtype is not torch.float32 or slopes.shape != (heads,) or not slopes.is_contiguous() or \
                    slopes.get_device() != self._index:
                raise ValueError(f"attend: slopes must be contiguous float32 [{heads}] on {self.device}")
            slopes_p = slopes.data_ptr()
        scale = self.head_dim ** -0.5 if scale is None else scale
        if not 0.0 < scale < 1e30 or not 0.0 <= softcap < 1e30 or not 0 <= window < 1 << 31:
            raise ValueError("attend: needs scale > 0, softcap >= 0 and window >= 0")
        s = self._stream(stream)
        ws, ws_p, ws_n = self._workspaces.get(s) or self._workspace(s)
        self._call("attend", self._lib.dvi_paged_attend, self._cref, bt,
                   _OPTIONS.pack(heads, scale, softcap, window, slopes_p), code, q_p, ld_q, o_p, ld_o, ws_p, ws_n, s)
        return out

    def read(self, table: torch.Tensor, lens: torch.Tensor, n_rows: int, row_start: Optional[torch.Tensor] = None,
             max_rows: Optional[int] = None, dtype: torch.dtype = torch.bfloat16,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Values of n_rows cached rows, positions lens[b], lens[b] + 1, ... of each sequence:
        (k, v) [n_rows, H_kv, head_dim] in dtype; zeros where no page is held."""
        if dtype not in _TYPES:
            raise ValueError("read: dtype must be bfloat16 or float32")
        code, esz = _TYPES[dtype]
        H, D = self.n_kv_heads, self.head_dim
        bt = self._batch("read", table, lens, n_rows, row_start, max_rows)
        k = torch.empty((n_rows, H, D), dtype=dtype, device=self.device)
        v = torch.empty((n_rows, H, D), dtype=dtype, device=self.device)
        self._call("read", self._lib.dvi_paged_read, self._cref, bt, code, k.data_ptr(), v.data_ptr(),
                   self._stream(stream))
        return k, v

    def status(self) -> list:
        """Names of the DVI_DEV_* flags set since the last look (waits for the device), then cleared."""
        word = int(self.status_word.item())
        if word:
            self.status_word.zero_()
        return [name for bit, name in DEV_BITS.items() if word & bit]

    def _workspace(self, stream: int):
        """attend's workspace, one for each stream (calls on different streams may overlap): the tensor, its
        address and its size."""
        with torch.cuda.device(self._index):
            n = self._lib.dvi_paged_workspace_bytes(self.head_dim)
            ws = torch.zeros(n, dtype=torch.uint8, device=self.device)
            got = (ws, ws.data_ptr(), n)
            # memory made inside a capture is the graph's: it serves this call only
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream(self._index).synchronize()   # zeroed for whichever stream asks
                self._workspaces[stream] = got
        return got
