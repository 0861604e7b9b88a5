"""Cross attention to an encoder's states, the operator after the self
attention in a DiT block.  All work runs in the HIP kernels behind the C ABI;
this module owns the workspace and the outputs.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import api

# elements between tokens: any number for queries, below 2^24 for keys and values
_FAR, _KEYS_APART = 1 << 62, (1 << 24) - 1


def _rows(x: torch.Tensor, most: int) -> torch.Tensor:
    """``x`` itself where the kernels read it in place (rows of contiguous
    elements, addresses and strides of 16 bytes, tokens at most ``most``
    elements apart), or a dense copy."""
    e = x.element_size()
    s0, s1, s2, s3 = x.stride()
    if s3 == 1 and s1 <= most and not (x.data_ptr() | s0 * e | s1 * e | s2 * e) & 15:
        return x
    return x.clone(memory_format=torch.contiguous_format)


class CrossAttention:
    """Attention of query blocks to encoder states, with the workspace kept
    across calls (one of each device, which only grows).  The calls of one
    instance share it: order them on one stream, or across streams by events.  A
    workspace that became too small stays allocated, for graphs captured with
    it."""

    def __init__(self, scale: float):
        self.scale = float(scale)
        self._ws: Dict[torch.device, torch.Tensor] = {}
        self._kept = []
        self._bytes = {}

    def _workspace(self, q, k, masked: bool) -> Optional[torch.Tensor]:
        key = (q.device, q.dtype, q.shape, k.shape, masked)
        n = self._bytes.get(key)
        if n is None:
            if len(self._bytes) >= 4096:
                self._bytes.clear()
            n = self._bytes[key] = api.cross_attn_workspace_bytes(
                q.dtype, q.shape[0], q.shape[2], k.shape[2], q.shape[3], q.shape[1], k.shape[1], masked)
        if n == 0:
            return None
        ws = self._ws.get(q.device)
        if ws is None or ws.numel() < n:
            if ws is not None:
                self._kept.append(ws)
                n = max(n, 2 * ws.numel())           # what is kept stays below what is in use
            ws = self._ws[q.device] = torch.empty(n, dtype=torch.uint8, device=q.device)
        return ws

    def __call__(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kv_lens: Optional[torch.Tensor] = None,
                 key_mask: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(OUT [B, q_len, H, D], LSE [B, H, q_len]) of q [B, q_len, H, D] over the
        live keys of k, v [B, kv_len, Hk, D].  Tensors that the kernels cannot
        read in place are copied first."""
        q, k, v = _rows(q, _FAR), _rows(k, _KEYS_APART), _rows(v, _KEYS_APART)
        B, q_len, H, D = q.shape
        out = q.new_empty((B, q_len, H, D))
        lse = q.new_empty((B, H, q_len), dtype=torch.float32)
        api.cross_attn(q, k, v, self.scale, out, lse, kv_lens, key_mask, self._workspace(q, k, key_mask is not None))
        return out, lse
