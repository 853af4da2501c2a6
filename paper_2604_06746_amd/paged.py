"""Buffer management for a cache held in 8 bits, in pages: a layer's, for a batch of sequences that take pages as they grow.

Owns the torch buffers and the list of free pages and calls the C ABI, on the current stream; no arithmetic happens here.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding as B


class PagedCache:
    """One layer's keys and values as 8-bit floats with a scale for each page and KV head, and the mass that each page has gathered.

    A sequence takes pages before its rows come (`reserve`, which is host work: keep it out of captured steps) and gives them back (`drop`,
    `release`).  append reads one array of lengths and writes the other, which is the current one from then on (`lens`): a captured step that
    is replayed has to make an even number of appends.  The calls of one PagedCache share its workspace and lengths, so they belong on one
    stream, or in order.  A sequence whose reserved pages do not hold what is appended stays as it was, and `missed` (int32 [batch] on the
    device) has a 1 for it: until the program sets that back to 0, attend gives the sequence's rows zeros.
    dtype: of new rows, queries and outputs.  max_pages: most pages of a sequence.  max_new: most fresh tokens in all of an attend call.
    workspace: another PagedCache's, where the calls of both follow each other (as those of a model's layers do)."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, n_pages: int, page_size: int, batch: int,
                 max_pages: int, max_new: Optional[int] = None, device="cuda", workspace: Optional[torch.Tensor] = None):
        self.Hq, self.G, self.d, self.dtype = n_q_heads, n_kv_heads, head_dim, dtype
        self.n_pages, self.page_size, self.batch, self.max_pages = n_pages, page_size, batch, max_pages
        dev = torch.device(device)
        self.k = torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
        self.v = torch.zeros_like(self.k, dtype=torch.uint8).view(torch.float8_e4m3fn)
        self.k_scale, self.v_scale = (torch.ones(n_pages, n_kv_heads, device=dev) for _ in range(2))
        self.pages = torch.full((batch, max_pages), -1, dtype=torch.int32, device=dev)
        self.mass = torch.zeros(batch, max_pages, device=dev)
        self.missed = torch.zeros(batch, dtype=torch.int32, device=dev)
        self._lens = [torch.zeros(batch, dtype=torch.int32, device=dev) for _ in range(2)]
        self._handles = [B.make_paged(self.k, self.v, self.k_scale, self.v_scale, self.pages, x, dtype, self.mass, self.missed) for x in self._lens]
        self._now = 0
        self._free: List[int] = list(range(n_pages - 1, -1, -1))
        self._table: List[List[int]] = [[] for _ in range(batch)]
        size = B.structkv_paged_workspace_bytes(self._handles[0], n_q_heads, batch if max_new is None else max_new)
        if size == 0:
            raise B.StructKVError(B.STRUCTKV_ERR_INVALID_ARG, B.structkv_last_error())
        if workspace is not None and (workspace.numel() * workspace.element_size() < size or workspace.device != self.k.device):
            raise B.StructKVError(B.STRUCTKV_ERR_WORKSPACE, "the workspace must have %d bytes, on the cache's GPU" % size)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=dev) if workspace is None else workspace

    @property
    def lens(self) -> torch.Tensor:
        """Slots in use, int32 [batch] on the device."""
        return self._lens[self._now]

    @property
    def handle(self) -> B.structkv_paged:
        return self._handles[self._now]

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def _put(self, b: int, first: int, ids: Sequence[int]) -> None:
        self.pages[b, first:first + len(ids)] = torch.tensor(ids, dtype=torch.int32, device=self.pages.device)

    def reserve(self, b: int, tokens: int) -> None:
        """Pages for `tokens` slots of sequence b in all, those that it has among them; nothing is taken where the pool cannot give them."""
        have, need = len(self._table[b]), -(-tokens // self.page_size)
        if need <= have:
            return
        if need > self.max_pages or need - have > len(self._free):
            raise B.StructKVError(B.STRUCTKV_ERR_INVALID_ARG, "sequence %d needs %d pages: it may have %d, and %d are free" % (
                b, need, self.max_pages, len(self._free)))
        new = [self._free.pop() for _ in range(need - have)]
        self._table[b] += new
        self._put(b, have, new)
        self.mass[b, have:need] = 0.0

    def drop(self, b: int, entries: Sequence[int]) -> None:
        """The pages of these table entries go back to the pool: nobody sees their tokens from then on.  The page that the next token goes to
        must not be among them."""
        entries = [int(j) for j in entries]
        if any(not 0 <= j < len(self._table[b]) for j in entries):
            raise B.StructKVError(B.STRUCTKV_ERR_INVALID_ARG, "sequence %d has %d table entries" % (b, len(self._table[b])))
        for j in entries:
            if self._table[b][j] >= 0:
                self._free.append(self._table[b][j])
                self._table[b][j] = -1
        if entries:
            self.pages[b, torch.tensor(entries, device=self.pages.device)] = -1

    def release(self, b: int) -> None:
        """All pages of sequence b go back to the pool, and its length to zero."""
        self._free += [p for p in self._table[b] if p >= 0]
        self._put(b, 0, [-1] * len(self._table[b]))
        self._table[b] = []
        self.lens[b] = 0
        self.missed[b] = 0

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: Sequence[int], rotary: Optional[B.structkv_rotary] = None,
               pos_new: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Rows behind those in use, keys rotated on the way where rotary is given; returns q rotated, where given.  Arguments as
        structkv_paged_append."""
        q_out = None if q is None else torch.empty(q.shape, dtype=q.dtype, device=q.device)
        B.structkv_paged_append(self.handle, k_new, v_new, cu_new, self._lens[1 - self._now], rotary, pos_new, q, q_out)
        self._now = 1 - self._now
        return q_out

    def attend(self, q: torch.Tensor, cu_new: Sequence[int], lam: float = 0.0, scale: float = 0.0, softcap: float = 0.0):
        """Attention of the tokens appended last: (out [new, H_q, d], lse [new, H_q]).  lam > 0, single tokens: their weights are gathered by
        page.  (Chains and a prompt's chunks leave `mass` as it is: pages are chosen by it after some tokens.)"""
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        B.structkv_paged_attend(self.handle, self.Hq, q, cu_new, out, lse, self.workspace, scale, softcap, lam)
        return out, lse
