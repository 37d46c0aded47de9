"""Speculative decoding over a paged private KV store: attention of drafted trees, and verification of the drafts.

A request's drafted tokens are a tree whose nodes are consecutive batch rows, a parent before its children; `parents`
int32 [rows] holds the index, within the request, of each node's parent (-1: none).  Node 0 is the token that the last step
sampled.  A step over a paged.PagedKvStore is

    store.append(q, k, v, table, kv_len, positions, cos_sin, ...)      # all nodes, at committed tokens + depth
    out, lse = attention(q, store, table, kv_len, parents)              # or engine.MoskaLayer.step_paged(..., parents=)
    path, n_path, next_token = verify(target_probs, tokens, parents, u_accept, u_next, draft_probs)
    kv_len = store.commit(table, kv_len, path, n_path, max_nodes)

No arithmetic here: every step runs in the CUDA library; torch owns the memory and the streams.
"""
from __future__ import annotations

import math

import torch

from . import binding as M
from .paged import FORMATS, _address, _call, _settled

MAX_NODES = M.TREE_MAX_NODES


class TreeAttention:
    """Attention of drafted trees over the paged contexts that they end: owns the scratch and the result
    buffers for one shape.  Calls share them: give every stream its own instance."""

    def __init__(self, B, Hq, Hkv, D, max_len, n_requests, max_nodes, fmt="bf16", n_unique_splits=None, device="cuda"):
        """B counts batch rows (nodes of n_requests trees of at most max_nodes, and padding rows behind them);
        max_len: longest context, the nodes included.  n_unique_splits: parts that a context may be cut into."""
        if fmt not in FORMATS:
            raise ValueError(f"fmt = {fmt!r} is not one of {sorted(FORMATS)}")
        if not 1 <= max_nodes <= MAX_NODES:
            raise ValueError(f"max_nodes = {max_nodes}, 1..{MAX_NODES} are possible")
        self.fmt, self.n_requests, self.max_nodes = fmt, n_requests, max_nodes
        if n_unique_splits is None:
            n_unique_splits = 64 if max_len > 128 else 1  # (a cut is a multiple of 128 tokens)
        self.shape = M.shape(B, Hq, Hkv, D, 1, 128, 1, n_unique_splits=n_unique_splits, q_len=max_nodes)
        self.scale = 1.0 / math.sqrt(D)
        self.out = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=device)
        self.lse = torch.empty(B, Hq, dtype=torch.float32, device=device)
        self.ws = torch.empty(M.tree_attn_workspace_bytes(self.shape), dtype=torch.uint8, device=device)
        _settled(self.out.device)

    def __call__(self, q, store, page_table, kv_len, parents=None, row_start=None, stream=None):
        """q bf16 [B][Hq][D] -> (out bf16 [B][Hq][D], lse float [B][Hq]), this object's buffers.  Every node sees its
        request's committed tokens, its ancestors and itself; without parents trees are chains.  Request r's nodes are rows
        row_start[r] .. row_start[r+1] - 1, or max_nodes each without row_start; padding rows behind the last request
        keep what the buffers held."""
        if store.fmt != self.fmt or store.Hkv != self.shape.Hkv:
            raise ValueError("the store's format or heads are not this attention's")
        if page_table.shape[0] != self.n_requests:
            raise ValueError(f"{page_table.shape[0]} page-table rows for {self.n_requests} requests")
        _call.tree_attend(store._handle, q, page_table, kv_len, parents, row_start, self.out, self.lse, self.scale,
                          self.max_nodes, self.shape.n_unique_splits, self.ws, _address(stream))
        return self.out, self.lse


def verify(target_probs, tokens, parents, u_accept, u_next, draft_probs=None, row_start=None, max_nodes=None, out=None,
           stream=None):
    """Which drafted tokens the target takes: (path int32 [R][max_nodes], n_path int32 [R], next_token int32 [R]).

    target_probs, draft_probs float or bf16 [rows][V] (rows may lie apart): row i is the distribution behind node i; in
    draft_probs the one that its children were drawn from, each independently of its siblings (for siblings drawn without
    replacement what is emitted does not follow the target).  None: they were picked without chance, the likeliest ones for
    instance.  tokens int32 [rows]: a node
    whose token is outside the vocabulary is not tried.  u_accept float [rows] and u_next float [R]: random numbers
    in [0, 1).  path[r]: the accepted nodes, 0 first, then -1.  Rows as in TreeAttention; max_nodes may be left out where
    all requests have as many.  The same inputs always give the same result.  `out`: the three results' tensors."""
    if max_nodes is None:
        if row_start is not None or u_next.shape[0] == 0:
            raise ValueError("give max_nodes")
        max_nodes = target_probs.shape[0] // u_next.shape[0]
    path, n_path, next_token = (None, None, None) if out is None else out
    return _call.verify(target_probs, draft_probs, tokens, parents, u_accept, u_next, row_start, max_nodes, path, n_path,
                        next_token, _address(stream))
