"""Host-side sequencing of the attention calls: the half of a transformer layer that stands beside SparseFFN.

Only call ordering and buffer ownership live here; every arithmetic step is a libs24 kernel.  In training, Attention owns what one layer keeps
between its passes.  In sampling, PagedKV holds the keys and values of the sequences that are being sampled, in 16 or 8 bits: the tokens of a
prompt are written to it as they come, each new token attends over it, and whole sequences are read back where the next chunk of a
prompt attends to the earlier ones.
"""
from __future__ import annotations

import threading

import torch

from . import binding as s24


class _Buffers(threading.local):
    """A thread's workspaces, one for each device and stream."""

    def __init__(self):
        self.held = {}


_buffers = _Buffers()


def _workspace(n, beside):
    """n bytes for a call on the current stream, on the device of the tensor `beside`.  A workspace holds nothing between calls, and those of a stream follow each other: they
    all have one, as large as the largest of them needs (two threads may launch on one stream in between each other: each has its own).  A call that goes
    into a graph has one from the graph's memory: graphs that were captured on one stream may be replayed on several at the same time, and outlive a
    buffer that is outgrown."""
    if n == 0:
        return None
    stream, held = s24._stream(), _buffers.held
    if stream != 0 and torch.cuda.is_current_stream_capturing():   # (the default stream cannot be captured)
        return s24.Workspace(n, beside.device)
    key = (beside.get_device(), stream)
    work = held.get(key)
    if work is None or work.bytes < n:
        work = held[key] = s24.Workspace(n, beside.device)
    return work


class Attention:
    """Buffers and call sequence of one attention layer: hq query heads on hkv key-value heads of d values, up to tokens_q query rows
    (in the backward pass up to tokens_k key rows; None: as many) of packed sequences.  dtype: torch.bfloat16 or torch.float16.  lse [hq, rows] is that of the last
    forward pass."""

    def __init__(self, hq: int, hkv: int, d: int, tokens_q: int, tokens_k: int | None = None, dtype=torch.bfloat16, device="cuda", causal: bool = True,
                 scale: float | None = None):
        self.hq, self.hkv, self.d, self.tokens_q = hq, hkv, d, tokens_q
        self.tokens_k = tokens_q if tokens_k is None else tokens_k
        self.causal, self.scale = causal, scale
        self.dtype, self.device = dtype, device
        self.O = torch.empty((tokens_q, hq, d), dtype=dtype, device=device)
        self.rest = torch.empty((tokens_q, hq, d), dtype=torch.int8, device=device)   # what the rounding of O took away: the backward pass takes delta from both
        self._rest = self.rest.data_ptr()
        self.lse = self._lse = torch.empty((hq, tokens_q), dtype=torch.float32, device=device)
        self.dQ = self.dK = self.dV = None   # allocated by the first backward pass
        self.need = {}   # bytes of workspace that a pass over so many rows and sequences takes

    def _workspace(self, need, tokens_q, tokens_k, cu_q):
        key = (need, tokens_q, tokens_k, cu_q.shape[0])
        n = self.need.get(key)
        if n is None:
            if len(self.need) >= 1024:   # (batches of ever new sizes)
                self.need.clear()
            n = self.need[key] = need(tokens_q, tokens_k, self.hq, self.hkv, self.d, cu_q.shape[0] - 1)
        return _workspace(n, self.O)

    def forward(self, Q, K, V, cu_q, cu_k=None):
        """O [rows of Q, hq, d].  Q, K, V may be views of one projection's result; cu_q, cu_k: int32 offsets of the sequences."""
        n, O, self.lse = Q.shape[0], self.O, self._lse
        if n < self.tokens_q:
            O, self.lse = O[:n], self._lse.view(-1)[:self.hq * n].view(self.hq, n)
        return s24.attn_fwd(Q, K, V, O, self.lse, self._workspace(s24.attn_fwd_workspace, n, K.shape[0], cu_q), cu_q, cu_k, self.causal, self.scale, self._rest)

    def backward(self, Q, K, V, dO, cu_q, cu_k=None):
        """dQ, dK, dV of the last forward pass, whose operands are given again."""
        nq, nk = Q.shape[0], K.shape[0]
        work = self._workspace(s24.attn_bwd_workspace, nq, nk, cu_q)
        if self.dQ is None:
            # the layout of the projection's gradient: dQ, dK and dV are its parts
            if self.tokens_q == self.tokens_k:
                self.dQKV = torch.empty((self.tokens_q, self.hq + 2 * self.hkv, self.d), dtype=self.dtype, device=self.device)
                self.dQ, self.dK, self.dV = self.dQKV[:, :self.hq], self.dQKV[:, self.hq:self.hq + self.hkv], self.dQKV[:, self.hq + self.hkv:]
            else:
                self.dQKV = None
                self.dQ = torch.empty((self.tokens_q, self.hq, self.d), dtype=self.dtype, device=self.device)
                self.dK, self.dV = (torch.empty((self.tokens_k, self.hkv, self.d), dtype=self.dtype, device=self.device) for _ in range(2))
        O, dQ, dK, dV = self.O, self.dQ, self.dK, self.dV
        if nq < self.tokens_q:
            O, dQ = O[:nq], dQ[:nq]
        if nk < self.tokens_k:
            dK, dV = dK[:nk], dV[:nk]
        return s24.attn_bwd(Q, K, V, O, dO, self.lse, dQ, dK, dV, work, cu_q, cu_k, self.causal, self.scale, self._rest)


class PagedKV:
    """Keys and values of many sequences in pages of `page` tokens, in 16 bits (the values as they are) or 8 (whole numbers and a step for each token
    and head).  Which page belongs to whom is the caller's: a table [sequences, pages of the longest] of page numbers."""

    def __init__(self, pages: int, page: int, hkv: int, d: int, dtype=torch.bfloat16, bits: int = 16, device="cuda"):
        if bits not in (16, 8):
            raise ValueError(f"a cache of 16 or 8 bits, not {bits}")
        self.pages, self.page, self.hkv, self.d, self.dtype, self.bits = pages, page, hkv, d, dtype, bits
        shape = (pages, hkv, page, d)
        self.K, self.V = (torch.empty(shape, dtype=dtype if bits == 16 else torch.uint8, device=device) for _ in range(2))
        self.k_step, self.v_step = (torch.empty(shape[:3], dtype=torch.float32, device=device) if bits == 8 else None for _ in range(2))
        self.buffers = s24.KVBuffers(self.K, self.V, dtype, self.k_step, self.v_step)
        self.need = {}   # bytes of workspace that queries of a shape take

    def write(self, K, V, places):
        """Rows of K and V [tokens, hkv, d] to their places: page number * page + position in the page (int64; negative ones are skipped)."""
        s24.kv_write(self.buffers, K, V, places)

    def read(self, table, cu, K, V):
        """The sequences, one after the other from the offsets cu on, into K and V [tokens, hkv, d]: as Attention.forward takes them."""
        return s24.kv_read(self.buffers, table, cu, K, V)

    def attend(self, Q, table, lengths, O, scale=None):
        """O [sequences, hq, d]: attention of one new token of each sequence over its first lengths[i] positions."""
        n = self.need.get(Q.shape)
        if n is None:
            n = self.need[Q.shape] = s24.attn_decode_workspace(self.buffers, Q.shape[0], Q.shape[1])
        return s24.attn_decode(self.buffers, Q, table, lengths, O, _workspace(n, self.K), scale)
