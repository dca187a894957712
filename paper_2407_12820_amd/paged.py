"""Paged key/value cache: ctypes marshalling over the pqc_paged_* calls of include/pqcache.h.

A `PagedCache` is a view of a pool of pages that the caller owns: which sequences lie in it, and where, comes with every
call as a page table and lengths, so that one object serves a batch that changes from step to step.

Scratch memory of the attention calls: one workspace and one block of counters per stream, which all caches share, since
what runs on a stream runs in order.  A call that is recorded into a graph has a workspace out of the graph's own memory, and
counters that only the calls recorded on the same stream into the same graph get, so that two graphs share none.
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Optional

import torch

from . import binding
from .binding import PQCacheError

_DTYPES = {"f32": (0, torch.float32), "bf16": (1, torch.bfloat16), "fp8": (2, torch.float8_e4m3fn)}
_STYLES = {"halves": 0, "pairs": 1}


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens", "n_pages", "max_pages",
                                         "io_dtype", "cache_dtype", "out_dtype")] + [("softmax_scale", C.c_float)] + [
                                             (n, C.c_int32) for n in ("rot_dims", "rot_style", "rot_positions")]


class Pages(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_pages", "v_pages", "k_scale", "v_scale", "page_table", "lengths", "counters")]


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = binding.load()
        vp, cfg, pages, i32, i64, size = C.c_void_p, C.POINTER(Config), C.POINTER(Pages), C.c_int32, C.c_int64, C.c_size_t
        lib.pqc_paged_append.restype = C.c_int
        lib.pqc_paged_append.argtypes = [cfg, pages, vp, i64, vp, i64, vp, i64, i32, vp, vp, vp, vp, vp, vp]
        lib.pqc_paged_counter_bytes.restype = size
        lib.pqc_paged_counter_bytes.argtypes = [cfg]
        lib.pqc_paged_workspace_bytes.restype = size
        lib.pqc_paged_workspace_bytes.argtypes = [cfg, i32, i32]
        lib.pqc_paged_attn.restype = C.c_int
        lib.pqc_paged_attn.argtypes = [cfg, pages, vp, i32, vp, vp, vp, size, vp]
        lib.pqc_paged_gather_attn.restype = C.c_int
        lib.pqc_paged_gather_attn.argtypes = [cfg, pages, vp, vp, i32, vp, vp, size, vp]
        lib.hipStreamGetCaptureInfo.restype = C.c_int  # of the HIP runtime that the library is linked to
        lib.hipStreamGetCaptureInfo.argtypes = [vp, C.POINTER(C.c_int), C.POINTER(C.c_uint64)]
        _lib = lib
    return _lib


class _Scratch:
    """Of one stream."""

    def __init__(self, device, words: int):
        self.counters = torch.zeros(words, dtype=torch.int32, device=device)
        self.counters_ptr = self.counters.data_ptr()
        self.workspace, self.ptr, self.size = None, 0, 0

    def grow(self, size: int) -> None:
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.counters.device)
        self.ptr, self.size = self.workspace.data_ptr(), size


class _Device:
    """Scratch memory of a GPU: by raw stream, and counters for recordings."""

    SPARE = 64     # blocks of counters that are made at a time; a recording without one takes a launch more
    WORDS = 512    # counters that a call of up to 512 KV heads needs

    def __init__(self):
        self.streams, self.spare = {}, []
        self.recorded = {}  # by recording and raw stream: its graph's for good, 2 KB each

    def restock(self, device) -> None:
        """Counters for recordings to come, if there are none."""
        if not self.spare:
            self.spare = list(torch.zeros((self.SPARE, self.WORDS), dtype=torch.int32, device=device))
            torch.cuda.current_stream(device).synchronize()  # a graph may run on any stream

    def stream(self, raw: int, device) -> _Scratch:
        """For a call that runs now."""
        self.restock(device)
        found = self.streams.get(raw)
        if found is None:
            found = self.streams[raw] = _Scratch(device, self.WORDS)
        return found

    def recording(self, raw: int, lib) -> Optional[torch.Tensor]:
        """Counters for a call that is being recorded on this stream; None: there are none left."""
        status, at = C.c_int(0), C.c_uint64(0)
        if lib.hipStreamGetCaptureInfo(raw, C.byref(status), C.byref(at)) != 0:
            return None
        key = at.value, raw
        if key not in self.recorded and self.spare:
            self.recorded[key] = self.spare.pop()
        return self.recorded.get(key)


_devices = {}
_lock = threading.Lock()  # from the choice of scratch memory to the launch: another thread may let it grow, which frees it


def rotation_table(n_positions: int, rot_dims: int, base: float = 10000.0, device="cuda:0") -> torch.Tensor:
    """[n_positions][rot_dims] f32: cosines, then sines, of position * base^(-2j / rot_dims); angles in double precision."""
    j = torch.arange(0, rot_dims, 2, device=device, dtype=torch.float64)
    angle = torch.arange(n_positions, device=device, dtype=torch.float64)[:, None] * base ** (-j / rot_dims)
    return torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).contiguous()


# The small calls are shorter than what Python does in front of them, so that each tensor is checked in one expression on the
# quickest of torch's accessors, and what is wrong is worked out by _need and _rows only if something is.
class PagedCache:
    """Pages [n_pages][Hkv][page_tokens][D] of keys and of values, float8_e4m3fn with scales [n_pages][Hkv] f32 (positive; `append` leaves
    powers of two), or bfloat16 (scales None).  `dtype`: "f32" or "bf16", of q, k and v; `out_dtype`: of the attention output; `rotation`: the table of
    rotation_table() or one laid out like it, None for no rotation.  Like a decode context it is not thread-safe.

    Calls run on the current stream, or on `stream`, to which their allocations then belong too.  They may be recorded into
    graphs."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scale: Optional[torch.Tensor], v_scale: Optional[torch.Tensor], *,
                 n_q_heads: int, dtype: str = "bf16", out_dtype: str = "f32", softmax_scale: float = 0.0,
                 rotation: Optional[torch.Tensor] = None, rot_style: str = "halves"):
        self.lib = _load()
        self.device = k_pages.device
        if k_pages.dim() != 4 or k_pages.dtype not in (torch.float8_e4m3fn, torch.bfloat16):
            raise ValueError("pages are [n_pages][Hkv][page_tokens][D] of float8_e4m3fn or bfloat16")
        n_pages, heads, tokens, dim = k_pages.shape
        self.io = _DTYPES[dtype][1]
        self.out = _DTYPES[out_dtype][1]
        self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.rotation = k_pages, v_pages, k_scale, v_scale, rotation
        self._need(k_pages, k_pages.dtype, k_pages.shape, "k_pages")
        self._need(v_pages, k_pages.dtype, k_pages.shape, "v_pages")
        fp8 = k_pages.dtype is torch.float8_e4m3fn
        if fp8:
            self._need(k_scale, torch.float32, (n_pages, heads), "k_scale")
            self._need(v_scale, torch.float32, (n_pages, heads), "v_scale")
        rot_dims = rot_positions = 0
        if rotation is not None:
            rot_positions, rot_dims = rotation.shape
            self._need(rotation, torch.float32, rotation.shape, "rotation")
        self._rotation = None if rotation is None else rotation.data_ptr()
        self.heads, self.dim, self.q_heads = heads, dim, n_q_heads
        self._q_row, self._out_row = n_q_heads * dim * self.io.itemsize, n_q_heads * dim * self.out.itemsize  # bytes of a token
        self.cfg = Config(1, n_q_heads, heads, dim, tokens, n_pages, 1, _DTYPES[dtype][0], 2 if fp8 else 1, _DTYPES[out_dtype][0],
                          softmax_scale, rot_dims, _STYLES[rot_style], rot_positions)
        self.pages = Pages(k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr() if fp8 else None,
                           v_scale.data_ptr() if fp8 else None, None, None, None)
        self._cfg, self._pages = C.byref(self.cfg), C.byref(self.pages)
        self._dev = k_pages.get_device()
        self._scratch = _devices.setdefault(self._dev, _Device())
        self._counted = 0 < self.lib.pqc_paged_counter_bytes(self._cfg) <= 4 * _Device.WORDS
        self._sizes = {}  # workspace bytes by (query tokens, listed tokens, batch, max_pages)
        if self._dev >= 0:
            with _lock, torch.cuda.device(self._dev):
                if not torch.cuda.is_current_stream_capturing():
                    self._scratch.restock(self.device)
        self._set = (1, 1, None, None, None)  # batch, max_pages, page table, lengths and counters as they are in the structures

    @classmethod
    def empty(cls, n_pages: int, n_q_heads: int, n_kv_heads: int, head_dim: int = 128, page_tokens: int = 64, cache_dtype: str = "fp8",
              device="cuda:0", **more) -> "PagedCache":
        """A cache with a pool of its own."""
        shape = (n_pages, n_kv_heads, page_tokens, head_dim)
        k, v = (torch.empty(shape, dtype=_DTYPES[cache_dtype][1], device=device) for _ in range(2))
        ks = vs = None
        if cache_dtype == "fp8":
            ks, vs = (torch.ones((n_pages, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2))
        return cls(k, v, ks, vs, n_q_heads=n_q_heads, **more)

    # -- marshalling helpers
    def _need(self, t, dtype, shape, what: str) -> int:
        if t is None or t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.device != self.device:
            got = "None" if t is None else f"{t.dtype} {tuple(t.shape)} on {t.device}"
            raise ValueError(f"{what}: expected contiguous {dtype} {tuple(shape)} on {self.device}, got {got}")
        return t.data_ptr()

    def _rows(self, t: torch.Tensor, n: int, heads: int, what: str) -> int:
        """Token stride of [n][heads][D] whose heads are adjacent."""
        if t.dtype is not self.io or t.shape != (n, heads, self.dim) or t.get_device() != self._dev:
            raise ValueError(f"{what}: expected {self.io} {(n, heads, self.dim)} on {self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        token, head, one = t.stride()
        if one != 1 or (head != self.dim and heads > 1):
            raise ValueError(f"{what}: the heads of a token must be adjacent")
        return token if n > 1 else heads * self.dim

    def _place(self, page_table: torch.Tensor, lengths: torch.Tensor, offsets: Optional[torch.Tensor], n: int) -> Optional[int]:
        """Sets the batch of a call; returns the address of the offsets."""
        shape = page_table.shape
        if len(shape) != 2:
            raise ValueError("page_table is [B][max_pages]")
        b, most = shape
        if lengths.dtype is not torch.int32 or lengths.shape != (b,) or not lengths.is_contiguous() or lengths.get_device() != self._dev:
            self._need(lengths, torch.int32, (b,), "lengths")
        if page_table.dtype is not torch.int32 or not page_table.is_contiguous() or page_table.get_device() != self._dev:
            self._need(page_table, torch.int32, shape, "page_table")
        was_b, was_most, was_table, was_lengths, counters = self._set
        table, lens = page_table.data_ptr(), lengths.data_ptr()
        if b != was_b or most != was_most:
            self.cfg.batch, self.cfg.max_pages = b, most
        if table != was_table:
            self.pages.page_table = table
        if lens != was_lengths:
            self.pages.lengths = lens
        self._set = b, most, table, lens, counters
        if offsets is not None:
            return self._need(offsets, torch.int32, (b + 1,), "offsets")
        if n != b:
            raise ValueError(f"{n} tokens for {b} sequences: give the offsets")
        return None

    def _own(self, stream) -> None:
        if stream.device != self.device:
            raise ValueError(f"the stream is of {stream.device}, the pages are on {self.device}")

    def _plain(self, t: torch.Tensor, dtype, n: int, heads: int, what: str) -> int:
        """Address of a contiguous [n][heads][D]."""
        if t.dtype is not dtype or t.shape != (n, heads, self.dim) or not t.is_contiguous() or t.get_device() != self._dev:
            self._need(t, dtype, (n, heads, self.dim), what)
        return t.data_ptr()

    def _attend(self, what: str, fn, n: int, n_idx: int, args) -> None:
        """fn(*args, workspace, bytes, stream) on the current stream of the cache's device."""
        dev = self._dev
        if dev < 0:
            raise ValueError(f"{what} runs on a GPU, the pages are on {self.device}")
        if torch._C._cuda_getDevice() != dev:
            with torch.cuda.device(dev):
                return self._attend(what, fn, n, n_idx, args)
        sizes = (n, n_idx, *self._set[:2])
        need = self._sizes.get(sizes)
        if need is None:
            if len(self._sizes) >= 256:
                self._sizes.clear()
            need = self._sizes[sizes] = self.lib.pqc_paged_workspace_bytes(self._cfg, n, n_idx)
        with _lock:
            self._launch(what, fn, need, args)

    def _launch(self, what: str, fn, need: int, args) -> None:
        raw = torch._C._cuda_getCurrentRawStream(self._dev)
        if torch._C._cuda_isCurrentStreamCapturing():
            own = self._scratch.recording(raw, self.lib) if self._counted else None
            counters = None if own is None else own.data_ptr()
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            at, size = workspace.data_ptr(), need
        else:
            scratch = self._scratch.streams.get(raw)
            if scratch is None or not self._scratch.spare:
                scratch = self._scratch.stream(raw, self.device)
            if scratch.size < need:
                scratch.grow(need)
            counters = scratch.counters_ptr if self._counted else None
            at, size = scratch.ptr, scratch.size
        if counters != self._set[4]:
            self.pages.counters = counters
            self._set = (*self._set[:4], counters)
        rc = fn(*args, at, size, raw)
        if rc != 0:
            raise PQCacheError(rc, what)

    # -- entry points (same names as the C ABI)
    def append(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, *, new_offsets=None, q=None,
               positions=None, q_out=None, k_out=None, stream=None):
        """New tokens k, v [n][Hkv][D] (rows of a projection allowed) join their sequences; `lengths` counts them already.
        With q [n][Hq][D] returns its rotated copy (q_out if given); k_out, if given, receives the rotated keys of the tokens that have a
        place in the table.  Outputs over each other, an input or the pages are refused."""
        if stream is not None:
            self._own(stream)
            with torch.cuda.stream(stream):
                return self.append(k, v, page_table, lengths, new_offsets=new_offsets, q=q, positions=positions, q_out=q_out, k_out=k_out)
        n, heads = k.shape[0], self.heads
        off = self._place(page_table, lengths, new_offsets, n)
        k_stride, v_stride = self._rows(k, n, heads, "k"), self._rows(v, n, heads, "v")
        qp = qo = ko = pos = None
        q_stride = 0
        if q is not None:
            q_stride, qp = self._rows(q, n, self.q_heads, "q"), q.data_ptr()
            if q_out is None:
                q_out = torch.empty((n, self.q_heads, self.dim), dtype=self.io, device=self.device)
            qo = self._plain(q_out, self.io, n, self.q_heads, "q_out")
        if k_out is not None:
            ko = self._plain(k_out, self.io, n, heads, "k_out")
        if positions is not None:
            pos = self._need(positions, torch.int32, (n,), "positions")
        if n:
            if self._dev < 0:
                raise ValueError(f"pqc_paged_append runs on a GPU, the pages are on {self.device}")
            if torch._C._cuda_getDevice() != self._dev:
                with torch.cuda.device(self._dev):
                    return self.append(k, v, page_table, lengths, new_offsets=new_offsets, q=q, positions=positions, q_out=q_out, k_out=k_out)
            rc = self.lib.pqc_paged_append(self._cfg, self._pages, qp, q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, n, off, pos,
                                           self._rotation, qo, ko, torch._C._cuda_getCurrentRawStream(self._dev))
            if rc != 0:
                raise PQCacheError(rc, "pqc_paged_append")
        return q_out

    def attn(self, q: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, *, q_offsets=None, out=None, stream=None):
        """Attention of q [n][Hq][D] over all tokens of each sequence, causal; -> out [n][Hq][D]."""
        if stream is not None:
            self._own(stream)
            with torch.cuda.stream(stream):
                return self.attn(q, page_table, lengths, q_offsets=q_offsets, out=out)
        n = q.shape[0]
        off = self._place(page_table, lengths, q_offsets, n)
        qp = self._plain(q, self.io, n, self.q_heads, "q")
        if out is None:
            out = torch.empty((n, self.q_heads, self.dim), dtype=self.out, device=self.device)
        op = self._plain(out, self.out, n, self.q_heads, "out")
        if op < qp + n * self._q_row and qp < op + n * self._out_row:
            raise ValueError("out must not overlap q")
        if n:
            self._attend("pqc_paged_attn", self.lib.pqc_paged_attn, n, 0, (self._cfg, self._pages, qp, n, off, op))
        return out

    def gather_attn(self, q: torch.Tensor, idx: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, *, out=None, stream=None):
        """Attention of q [B][Hq][D] over the tokens idx [B][Hkv][n_idx] int32 of each sequence; -> out [B][Hq][D]."""
        if stream is not None:
            self._own(stream)
            with torch.cuda.stream(stream):
                return self.gather_attn(q, idx, page_table, lengths, out=out)
        b = q.shape[0]
        self._place(page_table, lengths, None, b)
        qp = self._plain(q, self.io, b, self.q_heads, "q")
        n_idx = idx.shape[-1]
        if n_idx < 1 or idx.dtype is not torch.int32 or idx.shape != (b, self.heads, n_idx) or not idx.is_contiguous() or idx.get_device() != self._dev:
            self._need(idx, torch.int32, (b, self.heads, max(n_idx, 1)), "idx")
        if out is None:
            out = torch.empty((b, self.q_heads, self.dim), dtype=self.out, device=self.device)
        op = self._plain(out, self.out, b, self.q_heads, "out")
        if op < qp + b * self._q_row and qp < op + b * self._out_row:
            raise ValueError("out must not overlap q")
        if b:
            self._attend("pqc_paged_gather_attn", self.lib.pqc_paged_gather_attn, b, n_idx, (self._cfg, self._pages, qp, idx.data_ptr(), n_idx, op))
        return out
