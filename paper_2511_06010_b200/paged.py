"""A paged private KV store: pages in bf16 or in 4 bits, the calls that write and read them, and the
host-side book of which pages a request holds.  No arithmetic: every step runs in the CUDA library;
torch owns the memory and the streams.
"""
from __future__ import annotations

import ctypes
import functools
import math
from typing import Optional

import numpy as np
import torch

from . import binding as M

FORMATS = {"bf16": M.KV_BF16, "fp4": M.KV_FP4}
# the C calls themselves: the checks here replace the binding's, and an address is passed once
_append, _gather, _attend = (getattr(M._lib, "moska_" + n) for n in ("kv_append_paged", "kv_gather_paged", "paged_attn"))


def _on(index):
    """The library works on the current device: makes device `index` current for a call."""
    return None if index < 0 or torch._C._cuda_getDevice() == index else torch.cuda.device(index)


def _stream(stream, index):
    """Address of a stream, of the device's current one without `stream`."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index) if index >= 0 else 0
    return stream if isinstance(stream, int) else stream.cuda_stream


def _call(fn, name, index, *args):
    guard = _on(index)
    if guard is None:
        status = fn(*args)
    else:
        with guard:
            status = fn(*args)
    if status != M.OK:
        raise M.MoskaError(status, name)


@functools.lru_cache(maxsize=256)
def _shape(B, Hq, Hkv, D, n_unique_splits, q_len):
    """The shape struct of a call without a shared store (read only)."""
    return M.shape(B, Hq, Hkv, D, 1, 128, 1, n_unique_splits=n_unique_splits, q_len=q_len)


def _dense(t, name, dtype, shape, index):
    """Address of a dense tensor of a call; raises ValueError if it is not what the call needs."""
    if t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the store on device {index}")
    raise ValueError(f"{name} must be contiguous")


def _rows(t, name, shape, index):
    """Address and row stride of [n][heads][D] rows whose heads are dense; rows may lie apart."""
    if t.dtype != torch.bfloat16 or t.shape != shape:
        raise ValueError(f"{name}: expected torch.bfloat16 {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the store on device {index}")
    n, heads, D = shape
    row, head, one = t.stride()
    if n and (one != 1 or (heads > 1 and head != D)):
        raise ValueError(f"{name}: the heads of a row must be dense")
    return t.data_ptr(), (row if n > 1 else heads * D)


class PagedKvStore:
    """Pools of pages holding the private keys and values of many requests.

    bf16: `k_pages`, `v_pages` [n_pages][page_size][Hkv][D].  4-bit ("fp4": E2M1 codes, one f16 scale
    per (token, KV head, 32 dimensions)): `pages4` uint8 [n_pages][Hkv][page_size / 16][18 D].
    A store over existing pools: PagedKvStore(k_pages=.., v_pages=..) or PagedKvStore(pages4=..,
    page_size=..); new ones: PagedKvStore.empty(...).  page_size is a power of two, 16..32768.
    """

    def __init__(self, k_pages=None, v_pages=None, pages4=None, page_size: Optional[int] = None):
        if (pages4 is None) == (k_pages is None) or (k_pages is None) != (v_pages is None):
            raise ValueError("give k_pages and v_pages, or pages4")
        if pages4 is None:
            self.fmt = "bf16"
            self.n_pages, self.page_size, self.Hkv, self.D = k_pages.shape
            if page_size not in (None, self.page_size):
                raise ValueError(f"page_size = {page_size}, the pages hold {self.page_size}")
            self.device, index = k_pages.device, k_pages.get_device()
            shape = (self.n_pages, self.page_size, self.Hkv, self.D)
            pool = [_dense(t, name, torch.bfloat16, shape, index) for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages"))]
            self.k_pages, self.v_pages, self.pages4 = k_pages, v_pages, None
        else:
            self.fmt = "fp4"
            self.n_pages, self.Hkv, blocks, block_bytes = pages4.shape
            self.page_size, self.D = 16 * blocks, block_bytes // 18
            if page_size not in (None, self.page_size):
                raise ValueError(f"page_size = {page_size}, the pages hold {self.page_size}")
            self.device, index = pages4.device, pages4.get_device()
            pool = [_dense(pages4, "pages4", torch.uint8, (self.n_pages, self.Hkv, blocks, 18 * self.D), index), None]
            self.k_pages, self.v_pages, self.pages4 = None, None, pages4
        self._index, self._pool = index, pool
        self._head = (FORMATS[self.fmt], self.page_size, self.n_pages)

    @classmethod
    def empty(cls, n_pages, page_size, Hkv, D, fmt="bf16", device="cuda"):
        """A store of its own memory; the pages hold nothing yet."""
        if page_size < 16 or page_size & (page_size - 1):
            raise ValueError(f"page_size = {page_size} is not a power of two of at least 16")
        if FORMATS[fmt] == M.KV_BF16:
            k, v = (torch.empty(n_pages, page_size, Hkv, D, dtype=torch.bfloat16, device=device) for _ in range(2))
            return cls(k_pages=k, v_pages=v)
        return cls(pages4=torch.empty(n_pages, Hkv, page_size // 16, 18 * D, dtype=torch.uint8, device=device))

    def kv(self, page_table, kv_len) -> M.MoskaPagedKv:
        """The store seen through a page table int32 [R][max_pages] and context lengths int32 [R]."""
        if page_table.dim() != 2:
            raise ValueError(f"page_table: expected [requests][pages], got {tuple(page_table.shape)}")
        R, max_pages = shape = page_table.shape
        return M.MoskaPagedKv(*self._head, max_pages, *self._pool,
                              _dense(page_table, "page_table", torch.int32, shape, self._index),
                              _dense(kv_len, "kv_len", torch.int32, (R,), self._index))

    def _row_start(self, n_requests, n_rows, row_start, q_len):
        if row_start is not None:
            return _dense(row_start, "row_start", torch.int32, (n_requests + 1,), self._index)
        if n_rows != n_requests * q_len:
            raise ValueError(f"{n_rows} rows for {n_requests} requests of {q_len} each: give row_start")
        return None

    def append(self, q, k, v, page_table, kv_len, positions=None, cos_sin=None, row_start=None, interleaved=False,
               q_out=None, q_len=1, stream=None):
        """Writes the new rows k, v [N][Hkv][D] into the pages, keys rotated, and returns the rotated
        queries (q [N][Hq][D], or None).  kv_len counts the tokens after the call.  Request r has rows
        row_start[r] .. row_start[r+1] - 1, or q_len each without row_start.  cos_sin float
        [positions][rot_dim] (cos, then sin; None: no rotation), positions int32 [N].  q, k and v may be
        columns of one projection's output."""
        index, Hkv, D = self._index, self.Hkv, self.D
        n, n_requests = k.shape[0], page_table.shape[0]
        kv = self.kv(page_table, kv_len)
        first = self._row_start(n_requests, n, row_start, q_len)
        kp, ks = _rows(k, "k", (n, Hkv, D), index)
        vp, vs = _rows(v, "v", (n, Hkv, D), index)
        Hq, qp, qs, to = Hkv, None, 0, None
        if q is not None:
            shape = q.shape
            if len(shape) != 3 or shape[0] != n or shape[2] != D:
                raise ValueError(f"q: expected ({n}, heads, {D}), got {tuple(shape)}")
            Hq = shape[1]
            qp, qs = _rows(q, "q", shape, index)
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                to = q_out.data_ptr()
            else:
                to = _dense(q_out, "q_out", torch.bfloat16, shape, index)
        elif q_out is not None:
            raise ValueError("q_out without q")
        rot_dim, n_positions, at, table = 0, 0, None, None
        if cos_sin is not None:
            if positions is None or cos_sin.dim() != 2:
                raise ValueError("cos_sin is [positions][rot_dim] and comes with positions")
            n_positions, rot_dim = cos_sin.shape
            table = _dense(cos_sin, "cos_sin", torch.float32, cos_sin.shape, index)
            at = _dense(positions, "positions", torch.int32, (n,), index)
        if n:
            _call(_append, "moska_kv_append_paged", index, qp, qs, kp, ks, vp, vs, at, table, n_positions, rot_dim,
                  interleaved, first, n_requests, to, ctypes.byref(kv),
                  ctypes.byref(_shape(n, Hq, Hkv, D, 1, 1 if first else q_len)), _stream(stream, index))
        return q_out

    def gather(self, page_table, kv_len, n_rows, row_start=None, q_len=1, k_out=None, v_out=None, stream=None):
        """The last rows of the contexts as bf16 [n_rows][Hkv][D] keys and values; rows as in append.
        Rows behind the last request keep what k_out and v_out hold."""
        index, shape, n_requests = self._index, (n_rows, self.Hkv, self.D), page_table.shape[0]
        kv = self.kv(page_table, kv_len)
        first = self._row_start(n_requests, n_rows, row_start, q_len)
        if k_out is None:
            k_out = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        if v_out is None:
            v_out = torch.empty_like(k_out)
        kp, vp = _dense(k_out, "k_out", torch.bfloat16, shape, index), _dense(v_out, "v_out", torch.bfloat16, shape, index)
        if n_rows:
            _call(_gather, "moska_kv_gather_paged", index, first, n_requests, kp, vp, ctypes.byref(kv),
                  ctypes.byref(_shape(n_rows, self.Hkv, self.Hkv, self.D, 1, 1 if first else q_len)), _stream(stream, index))
        return k_out, v_out


class PagedAttention:
    """Attention of a batch over its paged private contexts alone (no shared store): owns the scratch
    and the result buffers for one shape.  Calls share them: give every stream its own instance."""

    def __init__(self, B, Hq, Hkv, D, max_len, fmt="bf16", q_len=1, n_unique_splits=None, device="cuda"):
        """B counts batch rows: B / q_len requests of q_len query tokens; max_len: longest context."""
        self.fmt = fmt
        if n_unique_splits is None:
            n_unique_splits = M.default_paged_splits(FORMATS[fmt], B // max(1, q_len), Hkv, D, max(1, max_len))
        self.shape = _shape(B, Hq, Hkv, D, n_unique_splits, q_len)
        self.scale = 1.0 / math.sqrt(D)
        self.out = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=device)
        self.lse = torch.empty(B, Hq, dtype=torch.float32, device=device)
        ws_bytes = M.paged_attn_workspace_bytes(self.shape)
        self.ws = torch.empty(max(256, ws_bytes), dtype=torch.uint8, device=device)
        self._index, self._requests, self._heads = self.out.get_device(), B // max(1, q_len), (Hkv, D)
        self._results = (self.out.data_ptr(), self.lse.data_ptr(), self.scale, ctypes.byref(self.shape),
                         self.ws.data_ptr(), self.ws.numel())

    def __call__(self, q, store, page_table, kv_len, stream=None):
        """q bf16 [B][Hq][D] -> (out bf16 [B][Hq][D], lse float [B][Hq]), this object's buffers."""
        index = self._index
        if store.fmt != self.fmt or (store.Hkv, store.D) != self._heads:
            raise ValueError("the store's format or heads are not this attention's")
        if store._index != index:
            raise ValueError(f"the store is on {store.device}, the results on {self.out.device}")
        kv = store.kv(page_table, kv_len)
        if not self._requests:
            return self.out, self.lse
        if page_table.shape[0] != self._requests:
            raise ValueError(f"{page_table.shape[0]} page-table rows for {self._requests} requests")
        _call(_attend, "moska_paged_attn", index, _dense(q, "q", torch.bfloat16, self.out.shape, index),
              ctypes.byref(kv), *self._results, _stream(stream, index))
        return self.out, self.lse


class PageTable:
    """Which pages every request slot holds: a free list on the host and the int32 table [slots][max_pages]
    on the device.  Entries of pages that a slot does not hold are -1."""

    def __init__(self, n_pages, page_size, slots, max_pages, device="cuda"):
        self.page_size = page_size
        self.host = np.full((slots, max_pages), -1, dtype=np.int32)
        self.held = np.zeros(slots, dtype=np.int64)  # pages of each slot
        self.free = list(range(n_pages - 1, -1, -1))
        self.device_table = torch.full((slots, max_pages), -1, dtype=torch.int32, device=device)
        self._changed = False

    def reserve(self, slot: int, tokens: int) -> None:
        """Gives the slot pages for a context of `tokens`; raises (and changes nothing) if there are too few."""
        need = -(-int(tokens) // self.page_size)
        more = need - int(self.held[slot])
        if more <= 0:
            return
        if need > self.host.shape[1]:
            raise ValueError(f"{tokens} tokens need {need} pages, a table row has {self.host.shape[1]}")
        if more > len(self.free):
            raise RuntimeError(f"{more} pages wanted, {len(self.free)} free")
        for i in range(int(self.held[slot]), need):
            self.host[slot, i] = self.free.pop()
        self.held[slot] = need
        self._changed = True

    def release(self, slot: int) -> None:
        """Takes the slot's pages back."""
        n = int(self.held[slot])
        self.free.extend(int(p) for p in self.host[slot, :n][::-1])
        self.host[slot, :n] = -1
        self.held[slot] = 0
        self._changed = True

    def table(self) -> torch.Tensor:
        """The device table, brought up to date on the current stream."""
        if self._changed:
            self.device_table.copy_(torch.from_numpy(self.host))
            self._changed = False
        return self.device_table
