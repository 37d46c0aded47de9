"""A paged private KV store: pages in bf16 or in 4 bits, the calls that write and read them, and the
host-side book of which pages a request holds.  No arithmetic: every step runs in the CUDA library;
torch owns the memory and the streams.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional

import numpy as np
import torch

from . import binding as M

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_paged_call.so")):
    raise ImportError("_paged_call.so is missing: build it with `python -m paper_2511_06010_b200.build`")
from . import _paged_call as _call  # noqa: E402

if _call.built_for != f"torch {torch.__version__};":  # it reads torch's tensors by that torch's layout
    raise ImportError(f"_paged_call.so was built for {_call.built_for} this is {torch.__version__}: build it again with "
                      "`python -m paper_2511_06010_b200.build`")

FORMATS = {"bf16": M.KV_BF16, "fp4": M.KV_FP4}
_call.bind(*(ctypes.cast(getattr(M._lib, "moska_" + n), ctypes.c_void_p).value
             for n in ("kv_append_paged", "kv_gather_paged", "paged_attn")), M.MoskaError)


def _settled(device) -> None:
    """Waits until the device's current stream is done: fresh memory of the allocator may be what that stream was
    still using, and the calls may run on another one."""
    if device.type == "cuda" and not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(device).synchronize()


def _address(stream):
    """None (the current stream of the store's device), a stream object or a raw address -> what the calls take."""
    return stream if stream is None or isinstance(stream, int) else stream.cuda_stream


class PagedKvStore:
    """Pools of pages holding the private keys and values of many requests.

    bf16: `k_pages`, `v_pages` [n_pages][page_size][Hkv][D].  4-bit ("fp4": E2M1 codes, one f16 scale
    per (token, KV head, 32 dimensions)): `pages4` uint8 [n_pages][Hkv][page_size / 16][18 D].
    A store over existing pools: PagedKvStore(k_pages=.., v_pages=..) or PagedKvStore(pages4=..,
    page_size=..); new ones: PagedKvStore.empty(...).  page_size is a power of two, 16..32768.

    Calls run on the current stream, or on `stream`: their inputs have to be ready there, and their results are.
    Results that a call makes, its inputs and the pools may be dropped at any time, on either stream.
    """

    def __init__(self, k_pages=None, v_pages=None, pages4=None, page_size: Optional[int] = None):
        if (pages4 is None) == (k_pages is None) or (k_pages is None) != (v_pages is None):
            raise ValueError("give k_pages and v_pages, or pages4")
        pool = k_pages if pages4 is None else pages4
        if pool.dim() != 4:
            raise ValueError(f"a pool has four dimensions, got {tuple(pool.shape)}")
        if pages4 is None:
            self.fmt = "bf16"
            self.n_pages, self.page_size, self.Hkv, self.D = pool.shape
        else:
            self.fmt = "fp4"
            self.n_pages, self.Hkv, blocks, block_bytes = pool.shape
            self.page_size, self.D = 16 * blocks, block_bytes // 18
        if page_size not in (None, self.page_size):
            raise ValueError(f"page_size = {page_size}, the pages hold {self.page_size}")
        self.device, self.k_pages, self.v_pages, self.pages4 = pool.device, k_pages, v_pages, pages4
        self._pools = (pool, v_pages)  # what the handle points into
        self._handle = _call.store(FORMATS[self.fmt], self.page_size, self.n_pages, self.Hkv, self.D, pool, v_pages)

    @classmethod
    def empty(cls, n_pages, page_size, Hkv, D, fmt="bf16", device="cuda"):
        """A store of its own memory; the pages hold nothing yet."""
        if fmt not in FORMATS:
            raise ValueError(f"fmt = {fmt!r} is not one of {sorted(FORMATS)}")
        if page_size < 16 or page_size & (page_size - 1):
            raise ValueError(f"page_size = {page_size} is not a power of two of at least 16")
        if FORMATS[fmt] == M.KV_BF16:
            k, v = (torch.empty(n_pages, page_size, Hkv, D, dtype=torch.bfloat16, device=device) for _ in range(2))
            st = cls(k_pages=k, v_pages=v)
        else:
            st = cls(pages4=torch.empty(n_pages, Hkv, page_size // 16, 18 * D, dtype=torch.uint8, device=device))
        _settled(st.device)
        return st

    def kv(self, page_table, kv_len) -> M.MoskaPagedKv:
        """The store seen through a page table int32 [R][max_pages] and context lengths int32 [R]."""
        return M.MoskaPagedKv(*_call.view(self._handle, page_table, kv_len))

    def append(self, q, k, v, page_table, kv_len, positions=None, cos_sin=None, row_start=None, interleaved=False,
               q_out=None, q_len=1, stream=None):
        """Writes the new rows k, v [N][Hkv][D] into the pages, keys rotated, and returns the rotated
        queries (q [N][Hq][D], or None).  kv_len counts the tokens after the call.  Request r has rows
        row_start[r] .. row_start[r+1] - 1, or q_len each without row_start.  cos_sin float
        [positions][rot_dim] (cos, then sin; None: no rotation), positions int32 [N].  q, k and v may be
        columns of one projection's output.  Padding rows (behind the last request, or of no token of a context)
        are not written: they keep what q_out held, and in a result made here they hold anything."""
        return _call.append(self._handle, q, k, v, page_table, kv_len, positions, cos_sin, row_start, interleaved, q_out,
                            q_len, _address(stream))

    def gather(self, page_table, kv_len, n_rows, row_start=None, q_len=1, k_out=None, v_out=None, stream=None):
        """The last rows of the contexts as bf16 [n_rows][Hkv][D] keys and values; rows as in append.
        Padding rows keep what k_out and v_out held, as in append."""
        return _call.gather(self._handle, page_table, kv_len, n_rows, row_start, q_len, k_out, v_out, _address(stream))


class PagedAttention:
    """Attention of a batch over its paged private contexts alone (no shared store): owns the scratch
    and the result buffers for one shape.  Calls share them: give every stream its own instance."""

    def __init__(self, B, Hq, Hkv, D, max_len, fmt="bf16", q_len=1, n_unique_splits=None, device="cuda"):
        """B counts batch rows: B / q_len requests of q_len query tokens; max_len: longest context."""
        self.fmt = fmt
        if n_unique_splits is None:
            n_unique_splits = M.default_paged_splits(FORMATS[fmt], B // max(1, q_len), Hkv, D, max(1, max_len))
        self.shape = M.shape(B, Hq, Hkv, D, 1, 128, 1, n_unique_splits=n_unique_splits, q_len=q_len)
        self.scale = 1.0 / math.sqrt(D)
        self.out = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=device)
        self.lse = torch.empty(B, Hq, dtype=torch.float32, device=device)
        self.ws = torch.empty(M.paged_attn_workspace_bytes(self.shape), dtype=torch.uint8, device=device)
        _settled(self.out.device)

    def __call__(self, q, store, page_table, kv_len, stream=None):
        """q bf16 [B][Hq][D] -> (out bf16 [B][Hq][D], lse float [B][Hq]), this object's buffers."""
        if store.fmt != self.fmt or store.Hkv != self.shape.Hkv:
            raise ValueError("the store's format or heads are not this attention's")
        _call.attend(store._handle, q, page_table, kv_len, self.out, self.lse, self.scale, self.shape.q_len,
                     self.shape.n_unique_splits, self.ws, _address(stream))
        return self.out, self.lse


class PageTable:
    """Which pages every request slot holds: a free list on the host and the int32 table [slots][max_pages]
    on the device.  Entries of pages that a slot does not hold are -1.

    There is one device table, at one address (a captured graph finds the pages of each replay in it).  It is
    rewritten by table(), so that calls reading it and table() have to follow one another on a stream: pass
    table() the stream that the calls run on."""

    def __init__(self, n_pages, page_size, slots, max_pages, device="cuda"):
        self.page_size = page_size
        self.host = np.full((slots, max_pages), -1, dtype=np.int32)
        self.held = np.zeros(slots, dtype=np.int64)  # pages of each slot
        self.free = list(range(n_pages - 1, -1, -1))
        self.device_table = torch.full((slots, max_pages), -1, dtype=torch.int32, device=device)
        _settled(self.device_table.device)
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

    def table(self, stream=None) -> torch.Tensor:
        """The device table, brought up to date on `stream` (the current one of its device without): after the calls
        queued there, before those to come.  Returns when the copy is done."""
        if self._changed:
            with self._on(stream):
                self.device_table.copy_(torch.from_numpy(self.host))
            self._changed = False
        return self.device_table

    def _on(self, stream):
        if stream is None or self.device_table.device.type != "cuda":
            return contextlib.nullcontext()
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=self.device_table.device)
        return torch.cuda.stream(stream)
