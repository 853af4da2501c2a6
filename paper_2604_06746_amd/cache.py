"""Buffer management for a layer's cache in use: what follows a prefill's sweep, token by token.

Owns the torch buffers and calls the C ABI, on the current stream; no arithmetic happens here.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as B


class LayerCache:
    """One layer's keys and values for a batch of sequences, with the mass and the positions of the tokens they belong to.

    planes: 1 where all KV heads keep the same tokens, n_kv_heads where each evicts by its own mass.  Calls that change the lengths
    read one array of them and write the other, which is the current one from then on (`lens`): a captured step that is replayed has to
    make an even number of such calls.  The calls of one LayerCache share its workspace and lengths, so they belong on one stream, or in order.
    A sequence that has no room for what is appended stays as it was, and `missed` (int32 [batch] on the device) has a 1 for it: until the
    program sets that back to 0, attend gives the sequence's rows zeros and accept leaves its tokens as they are.
    max_new: most fresh tokens of a sequence in an attend call.  workspace: another LayerCache's, where the calls of both follow each other (as
    those of a model's layers do: it holds 34 MB and more for 64 sequences of 64 drafts); by default each has its own."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, capacities: Sequence[int], planes: int = 1,
                 max_new: int = B.STRUCTKV_MAX_DRAFTS, device="cuda", workspace: Optional[torch.Tensor] = None):
        self.Hq, self.G, self.d, self.planes = n_q_heads, n_kv_heads, head_dim, planes
        self.batch = len(capacities)
        self.cu = [0]
        for n in capacities:
            self.cu.append(self.cu[-1] + int(n))
        total, dev = self.cu[-1], torch.device(device)
        self.k = torch.empty(n_kv_heads, total, head_dim, dtype=dtype, device=dev)
        self.v = torch.empty_like(self.k)
        self.mass = torch.zeros(planes, total, device=dev)
        self.pos = torch.zeros(planes, total, dtype=torch.int32, device=dev)
        self._lens = [torch.zeros(self.batch, dtype=torch.int32, device=dev) for _ in range(2)]
        self.missed = torch.zeros(self.batch, dtype=torch.int32, device=dev)
        self._handles = [B.make_cache(self.k, self.v, self.cu, x, self.mass, self.pos, self.missed) for x in self._lens]
        self._now = 0
        size = B.structkv_cache_workspace_bytes(self._handles[0], n_q_heads, max_new * self.batch)
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
    def handle(self) -> B.structkv_cache:
        return self._handles[self._now]

    def reset(self) -> None:
        self.lens.zero_()
        self.missed.zero_()

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: Sequence[int], pos_new: torch.Tensor,
               mass_new: Optional[torch.Tensor] = None) -> None:
        """Rows behind those in use: a prefill's compact cache, or a step's tokens.  Arguments as structkv_cache_append."""
        B.structkv_cache_append(self.handle, k_new, v_new, cu_new, self._lens[1 - self._now], pos_new, mass_new)
        self._now = 1 - self._now

    def attend(self, q: torch.Tensor, cu_new: Sequence[int], tree_mask: Optional[torch.Tensor] = None, lam: float = 0.0,
               scale: float = 0.0, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None):
        """Attention of the tokens appended last: (out [new, H_q, d], lse [new, H_q]).  lam > 0, single tokens: their weights are gathered."""
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        B.structkv_cache_attend(self.handle, self.Hq, q, cu_new, out, lse, self.workspace, tree_mask, scale, softcap, slopes, lam)
        return out, lse

    def accept(self, cu_new: Sequence[int], path: Optional[torch.Tensor] = None, n_accept: Optional[torch.Tensor] = None,
               q: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None,
               lam: float = 0.0, scale: float = 0.0, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None) -> None:
        """The verified path of the drafts appended last stays; lam > 0: its weights are gathered (q, lse and the rest as in attend), the mass
        decayed once for all of them, where single tokens' attend decays it with each."""
        B.structkv_cache_accept(self.handle, self.Hq, q, lse, cu_new, self._lens[1 - self._now], path, n_accept, tree_mask, scale, softcap,
                                slopes, lam)
        self._now = 1 - self._now

    def evict(self, budget: Sequence[int], keep_tail: int, scores: Optional[torch.Tensor] = None) -> None:
        """Back to `budget` slots a sequence, by the mass (or `scores`), the recent ones kept."""
        B.structkv_cache_evict(self.handle, scores, budget, keep_tail, self._lens[1 - self._now], self.workspace)
        self._now = 1 - self._now
