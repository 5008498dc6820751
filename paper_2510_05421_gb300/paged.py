"""ctypes binding of the 8-bit paged KV cache (include/dvi.h): argument checks
and marshalling only.  The tensors are the caller's, and every call enqueues
on the caller's current stream (or the one it names)."""
from __future__ import annotations

import ctypes
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
        self.status_word = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = PagedCacheC(n_pages, H, P, D, KV_FORMATS[fmt], k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                              v_scale.data_ptr())
        self._cref = ctypes.byref(self._c)
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
        if table.dtype != torch.int32 or lens.dtype != torch.int32 or table.dim() != 2:
            raise ValueError(f"{what}: table must be int32 [B, max_pages] and lens int32 [B]")
        B, width = table.shape
        if lens.shape != (B,) or not (table.is_contiguous() and lens.is_contiguous()):
            raise ValueError(f"{what}: table and lens must be contiguous, with one row and one length a sequence")
        if table.device != self.device or lens.device != self.device:
            raise ValueError(f"{what}: table and lens must be on {self.device}")
        start = None
        if row_start is None:
            if B < 1 or n_rows % B:
                raise ValueError(f"{what}: {n_rows} rows do not divide into {B} sequences (give row_start)")
            max_rows = n_rows // B
        else:
            if row_start.dtype != torch.int32 or row_start.shape != (B + 1,) or not row_start.is_contiguous() or \
                    row_start.device != self.device:
                raise ValueError(f"{what}: row_start must be contiguous int32 [B + 1] on {self.device}")
            start = row_start.data_ptr()
            max_rows = n_rows if max_rows is None else max_rows
            if max_rows < 0:
                raise ValueError(f"{what}: max_rows must not be negative")
        if not 1 <= B <= 1024 or width < 1 or width * self.page_tokens > 1 << 30:
            raise ValueError(f"{what}: 1 to 1024 sequences of 1 to {(1 << 30) // self.page_tokens} pages")
        return PagedBatchC(B, width, n_rows, max_rows, table.data_ptr(), lens.data_ptr(), start,
                           self.status_word.data_ptr())

    def _rows(self, what, t, heads, dtype, n_rows):
        """Elements from row to row of t [n_rows, heads, head_dim], whose rows may lie apart."""
        if t.dtype != dtype or t.dim() != 3 or t.shape[1] != heads or t.shape[2] != self.head_dim or \
                t.shape[0] != n_rows:
            raise ValueError(f"{what} must be {dtype} [{n_rows}, {heads}, {self.head_dim}], got {t.dtype} "
                             f"{tuple(t.shape)}")
        ld, sh, sd = t.stride()
        if n_rows <= 1:
            ld = heads * self.head_dim
        if sd != 1 or (sh != self.head_dim and heads > 1) or ld < heads * self.head_dim:
            raise ValueError(f"{what}: each row's heads must be contiguous")
        if t.device != self.device:
            raise ValueError(f"{what} must be on {self.device}")
        if t.data_ptr() % 16 or ld * t.element_size() % 16:
            raise ValueError(f"{what}: rows must start on 16-byte boundaries")
        return ld

    def _call(self, what, fn, stream, *args):
        if self._index != torch.cuda.current_device():
            with torch.cuda.device(self._index):
                rc = fn(*args, stream)
        else:
            rc = fn(*args, stream)
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
        if k.dtype not in _TYPES:
            raise ValueError("append: k must be bfloat16 or float32")
        n = k.shape[0]
        bt = self._batch("append", table, lens, n, row_start, max_rows)
        ld_k = self._rows("append: k", k, self.n_kv_heads, k.dtype, n)
        ld_v = self._rows("append: v", v, self.n_kv_heads, k.dtype, n)
        rot_p, rot_dim, n_pos = None, 0, 0
        if rotary is not None:
            if rotary.dtype != torch.float32 or rotary.dim() != 3 or rotary.shape[2] != 2 or \
                    not rotary.is_contiguous() or rotary.device != self.device or rotary.data_ptr() % 16:
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
            ld_q = self._rows("append: q", q, heads, k.dtype, n)
            if q_out is None:
                q_out = torch.empty((n, heads, self.head_dim), dtype=k.dtype, device=self.device)
            ld_o = self._rows("append: q_out", q_out, heads, k.dtype, n)
            q_p, o_p = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise ValueError("append: q_out without q")
        self._call("append", self._lib.dvi_paged_append, self._stream(stream), self._cref, ctypes.byref(bt),
                   _TYPES[k.dtype][0], k.data_ptr(), ld_k, v.data_ptr(), ld_v, rot_p, rot_dim, n_pos, q_p, ld_q, o_p,
                   ld_o, heads)
        return q_out

    def attend(self, table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None,
               softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
               row_start: Optional[torch.Tensor] = None, max_rows: Optional[int] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of rows q [n, H_q, head_dim] (bf16 or f32), appended before at the same lens: the row at
        position p sees the held positions up to p (the last `window` of them).  scale: head_dim^-0.5 unless
        given; softcap c > 0: scores become c tanh(score / c); slopes f32 [H_q]: + slope (p_key - p)."""
        if q.dtype not in _TYPES or q.dim() != 3:
            raise ValueError("attend: q must be bfloat16 or float32 [n, H_q, head_dim]")
        n, heads = q.shape[0], q.shape[1]
        if heads < 1 or heads % self.n_kv_heads:
            raise ValueError(f"attend: {heads} heads do not divide over {self.n_kv_heads} KV heads")
        bt = self._batch("attend", table, lens, n, row_start, max_rows)
        ld_q = self._rows("attend: q", q, heads, q.dtype, n)
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=self.device)
        ld_o = self._rows("attend: out", out, heads, q.dtype, n)
        if slopes is not None and (slopes.dtype != torch.float32 or slopes.shape != (heads,) or
                                   not slopes.is_contiguous() or slopes.device != self.device):
            raise ValueError(f"attend: slopes must be contiguous float32 [{heads}] on {self.device}")
        scale = self.head_dim ** -0.5 if scale is None else scale
        if not 0.0 < scale < 1e30 or not 0.0 <= softcap < 1e30 or not 0 <= window < 1 << 31:
            raise ValueError("attend: needs scale > 0, softcap >= 0 and window >= 0")
        opt = PagedOptionsC(heads, scale, softcap, window, None if slopes is None else slopes.data_ptr())
        s = self._stream(stream)
        ws = self._workspace(s)
        self._call("attend", self._lib.dvi_paged_attend, s, self._cref, ctypes.byref(bt), ctypes.byref(opt),
                   _TYPES[q.dtype][0], q.data_ptr(), ld_q, out.data_ptr(), ld_o, ws.data_ptr(), ws.numel())
        return out

    def read(self, table: torch.Tensor, lens: torch.Tensor, n_rows: int, row_start: Optional[torch.Tensor] = None,
             max_rows: Optional[int] = None, dtype: torch.dtype = torch.bfloat16,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Values of n_rows cached rows, positions lens[b], lens[b] + 1, ... of each sequence:
        (k, v) [n_rows, H_kv, head_dim] in dtype; zeros where no page is held."""
        if dtype not in _TYPES:
            raise ValueError("read: dtype must be bfloat16 or float32")
        bt = self._batch("read", table, lens, n_rows, row_start, max_rows)
        out = torch.empty((2, n_rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device)
        k, v = out[0], out[1]
        self._call("read", self._lib.dvi_paged_read, self._stream(stream), self._cref, ctypes.byref(bt),
                   _TYPES[dtype][0], k.data_ptr(), v.data_ptr())
        return k, v

    def status(self) -> list:
        """Names of the DVI_DEV_* flags set since the last look (waits for the device), then cleared."""
        word = int(self.status_word.item())
        if word:
            self.status_word.zero_()
        return [name for bit, name in DEV_BITS.items() if word & bit]

    def _workspace(self, stream: int) -> torch.Tensor:
        """attend's workspace, one for each stream (calls on different streams may overlap)."""
        ws = self._workspaces.get(stream)
        if ws is None:
            with torch.cuda.device(self._index):
                n = self._lib.dvi_paged_workspace_bytes(self.head_dim)
                ws = torch.zeros(n, dtype=torch.uint8, device=self.device)
                # memory made inside a capture is the graph's: it serves this call only
                if not torch.cuda.is_current_stream_capturing():
                    torch.cuda.current_stream(self._index).synchronize()   # zeroed for whichever stream asks
                    self._workspaces[stream] = ws
        return ws
