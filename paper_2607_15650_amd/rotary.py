"""Rotary positions of queries and keys, and the root-mean-square norm before
them: what makes the attention's inputs from those of the projections.  The
kernel is behind the C ABI (ditango_rotary); this module computes the
frequencies, which depend on the configuration only.
"""
from __future__ import annotations

import math
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import _lib, api

_LAYOUT = {"interleaved": _lib.ROTARY_INTERLEAVED, "half": _lib.ROTARY_HALF}
_NORM = {"none": _lib.NORM_NONE, "head": _lib.NORM_HEAD, "row": _lib.NORM_ROW}


def axis_frequencies(dim: int, theta: float = 10000.0, scaling: Optional[Dict] = None) -> Tuple[List[float], float]:
    """Radians per position of the dim / 2 pairs of one axis, and the factor of
    cosine and sine.  theta^(-2i / dim), scaled for positions beyond those of
    the training (``scaling``: {"kind", "factor": s, ...}):
      linear  every frequency by 1 / s;
      ntk     theta by s^(dim / (dim - 2)): the lowest by 1 / s, the highest kept;
      yarn    (arXiv 2309.00071) by how often a pair turns over the ``original``
              positions: kept from ``beta`` turns on (32), by 1 / s up to
              ``alpha`` (1), linear between; cosine and sine by 0.1 ln s + 1.
    """
    if dim < 2 or dim % 2:
        raise ValueError("an axis takes an even number of dims, 2 at least")
    s, kind, factor = 1.0, "none", 1.0
    if scaling is not None:
        kind, s = scaling["kind"], float(scaling["factor"])
        if kind not in ("linear", "ntk", "yarn"):
            raise ValueError(f"unknown scaling {kind!r}; use linear, ntk or yarn")
        if not s >= 1.0 or not math.isfinite(s):
            raise ValueError("a scaling's factor is 1 at least")
    if kind == "ntk":
        if dim < 4:
            raise ValueError("ntk scaling needs 4 dims at least")
        theta = theta * s ** (dim / (dim - 2))
    freqs = [theta ** (-2.0 * i / dim) for i in range(dim // 2)]
    if kind == "linear":
        freqs = [f / s for f in freqs]
    elif kind == "yarn":
        alpha, beta = float(scaling.get("alpha", 1.0)), float(scaling.get("beta", 32.0))
        original = float(scaling["original"])
        if not beta > alpha or not original > 0:
            raise ValueError("yarn scaling needs beta above alpha and the original number of positions")
        keep = [min(1.0, max(0.0, (original * f / (2 * math.pi) - alpha) / (beta - alpha))) for f in freqs]
        freqs = [f * (g + (1.0 - g) / s) for f, g in zip(freqs, keep)]
        factor = 0.1 * math.log(s) + 1.0
    return freqs, factor


def grid_positions(frames: int, rows: int, cols: int, first: int = 0, count: Optional[int] = None,
                   device="cuda") -> torch.Tensor:
    """Positions [1, count, 3] (frame, row, column) of tokens [first, first +
    count) of a latent grid, flattened frame by frame."""
    total = frames * rows * cols
    count = total - first if count is None else count
    if first < 0 or count < 0 or first + count > total:
        raise ValueError("the tokens must lie inside the grid")
    n = torch.arange(first, first + count, device=device)
    return torch.stack([n // (rows * cols), n // cols % rows, n % cols], dim=-1).to(torch.int32)[None].contiguous()


class Rotary:
    """Rotary positions of a layer's queries and keys.

    ``axes``: the rotated dims of every axis of the positions (frame, row and
    column of a latent grid, say), together at most ``head_dim``; the dims after
    them are left as they are.  ``layout``: a pair's two elements are neighbours
    ("interleaved") or half of the rotated dims apart ("half").  ``norm``: the
    root-mean-square norm before the rotation, over each head ("head"), over all
    heads of a token ("row"), or "none".  ``scaling`` as axis_frequencies takes
    it, for every axis.
    """

    def __init__(self, head_dim: int, axes: Optional[Sequence[int]] = None, theta: float = 10000.0,
                 layout: str = "interleaved", scaling: Optional[Dict] = None, norm: str = "none", eps: float = 1e-6):
        axes = [head_dim] if axes is None else [int(a) for a in axes]
        if layout not in _LAYOUT or norm not in _NORM:
            raise ValueError("layout is interleaved or half; norm is none, head or row")
        if not axes or sum(axes) > head_dim:
            raise ValueError("the axes' dims must fit the head")
        self.head_dim, self.axes = head_dim, axes
        self.rot_dim, self.factor = sum(axes), 1.0
        self.freqs: List[float] = []
        self.axis: List[int] = []
        for i, dim in enumerate(axes):
            f, self.factor = axis_frequencies(dim, theta, scaling)
            self.freqs += f
            self.axis += [i] * (dim // 2)
        self.layout, self.norm, self.eps = layout, norm, float(eps)
        self._tables = api.rotary_tables(self.freqs, self.axis)

    def __call__(self, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """(q, k) rotated, or q alone where k is None: new dense tensors, or the
        ones given (``q`` and ``k`` themselves to work in place).  q, k [B, S,
        heads, head_dim] are the same tokens, at ``positions`` int32 [1 or B, S,
        len(axes)]."""
        if q.shape[-1] != self.head_dim:
            raise ValueError(f"the rows must have {self.head_dim} elements")
        if positions.dim() != 3 or positions.shape[2] != len(self.axes):
            raise ValueError("positions must be int32 [1 or B, S, axes]")
        if q_out is None:
            q_out = q.new_empty(q.shape)
        xs, ys = (q,), (q_out,)
        if k is not None:
            if k_out is None:
                k_out = k.new_empty(k.shape)
            xs, ys = (q, k), (q_out, k_out)
        api.rotary(xs, ys, positions, self._tables, self.rot_dim, _LAYOUT[self.layout], self.factor, _NORM[self.norm],
                   (q_weight, k_weight), self.eps)
        return (q_out, k_out) if k is not None else q_out


class RotatedInputs:
    """The rotated query block and keys of an engine's steps, in buffers of its
    own that the steps share.  Only the rows that a step reads are rotated: the
    block, and the keys of the partitions computed fresh (those of the block's
    own partition in the same call as its queries)."""

    def __init__(self, rotary: Rotary, offsets: Sequence[int]):
        self.rotary = rotary
        self.offsets = [int(o) for o in offsets]
        self.most = max(e - a for a, e in zip(self.offsets, self.offsets[1:]))
        self._buffers: Dict[Tuple, torch.Tensor] = {}
        self._kept = []                # buffers that were replaced: captured graphs may hold them

    def _buffer(self, name: str, x: torch.Tensor, rows: int) -> torch.Tensor:
        """Room for ``rows`` rows of ``x`` [B, S, H, D]: one buffer for each type and
        device, the old one where it fits."""
        n = x.shape[0] * rows * x.shape[2] * x.shape[3]
        key = (name, x.dtype, x.device)
        old = self._buffers.get(key)
        if old is None or old.numel() < n:
            if old is not None:
                self._kept.append(old)
                n = max(n, 2 * old.numel())          # what is kept stays below what is in use
            old = self._buffers[key] = x.new_empty(n)
        return old

    def begin(self, qb: int, q_all: torch.Tensor, k: torch.Tensor, positions: torch.Tensor,
              q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor]) -> torch.Tensor:
        """Starts a step of query block ``qb`` with its tensors ([B, S, H, D],
        positions [1 or B, S, axes]): returns the rotated block [B, L, H, D].
        The block's own keys are rotated with it."""
        a, e = self.offsets[qb], self.offsets[qb + 1]
        if positions is None or positions.dim() != 3 or positions.shape[1] != k.shape[1] or \
                k.shape[1] != self.offsets[-1]:
            raise ValueError("an engine with rotary positions needs positions [1 or B, S, axes] of the whole sequence")
        block = q_all[:, a:e]
        q = self._buffer("q", q_all, self.most)[:block.numel()].view(block.shape)
        self._k = self._buffer("k", k, k.shape[1])[:k.numel()].view(k.shape)
        self._src, self._pos, self._kw = k, positions, k_weight
        self._done = {qb}
        if e > a:
            self.rotary(block, k[:, a:e], positions[:, a:e].contiguous(), q_weight, k_weight, q, self._k[:, a:e])
        return q

    def keys(self, select: Sequence[int]) -> torch.Tensor:
        """K [B, S, H, D] with the rows of the selected partitions rotated."""
        P = len(self.offsets) - 1
        j = 0
        while j < P:
            if not select[j] or j in self._done:
                j += 1
                continue
            i = j
            while j < P and select[j] and j not in self._done:
                self._done.add(j)
                j += 1
            a, e = self.offsets[i], self.offsets[j]
            if e > a:
                self.rotary(self._src[:, a:e], None, self._pos[:, a:e].contiguous(), self._kw, q_out=self._k[:, a:e])
        return self._k


def check_rotary_args(rotary: Optional[Rotary], positions, q_weight, k_weight) -> None:
    if rotary is None and (positions is not None or q_weight is not None or k_weight is not None):
        raise ValueError("positions and norm weights belong to an engine with rotary positions")
