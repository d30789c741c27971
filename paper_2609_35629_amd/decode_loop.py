"""A multi-layer decode loop over the library: per layer a team table of the
prompt and a growing exact suffix (the paragraph "Cache state and budget"
and Alg. "SANTA++ attention for one query head": the generated rows
E = {N+1, .., N+t} are attended exactly, and E is empty at the first sparse
prediction).

Each step decodes every layer with the suffix rows generated so far, then
appends the step's new key/value row of each (b, kv) to that layer's suffix
cache.  The caches, tables and workspaces are allocated once, for the loop's
capacity; a step allocates nothing on the device beyond what the caller's
row copies need.

Given a :class:`Rotary`, a step takes queries and keys as the projections leave
them and turns them by their positions on the way (the prompt's K is given
rotated); a dense loop may carry several continuations of every prompt.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Sequence

import torch

from . import (SantappError, Teams, _lib, build_teams, decode, decode_workspace, dense_decode, dense_workspace,
               prefix_decode, prefix_workspace, rope_append)


class Rotary(NamedTuple):
    """How queries and keys are rotated (see :func:`rope`)."""
    freqs: torch.Tensor
    interleaved: bool = False
    magnitude: float = 1.0


class LayerCache:
    """One layer: its team table (or, for the dense baseline, its prompt
    K/V) and its suffix cache [B, Hkv, capacity, d] of which the first T rows
    are filled.  With ``continuations`` S > 1 (dense only) every prompt has S
    sequences, b = prompt * S + continuation, with suffixes of their own."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, capacity: int, Hq: int, budget: int,
                 P: int, R: int, dense: bool = False, continuations: int = 1):
        prompts, Hkv, N, d = K.shape
        if continuations < 1 or (continuations > 1 and not dense):
            raise SantappError(_lib.EINVAL, "several continuations of a prompt need a dense loop")
        B = prompts * continuations
        self.continuations = continuations
        self.B, self.Hkv, self.N, self.d, self.Hq = B, Hkv, N, d, Hq
        self.capacity = capacity
        self.budget = budget
        self.dense = dense
        self.T = 0
        self.sK = torch.zeros((B, Hkv, capacity, d), dtype=K.dtype, device=K.device)
        self.sV = torch.zeros_like(self.sK)
        self.out = torch.empty((B, Hq, d), dtype=torch.float32, device=K.device)
        self.q: Optional[torch.Tensor] = None
        if dense:
            self.K, self.V = K, V
            self.teams = None
            if continuations > 1:
                self.ws = prefix_workspace(prompts, continuations, Hq, Hkv, N, capacity, d, K.dtype, K.device)
            else:
                self.ws = dense_workspace(B, Hq, Hkv, N, capacity, d)
        else:
            self.teams: Optional[Teams] = build_teams(K, V, P, R)
            self.ws = decode_workspace(self.teams, Hq, capacity, budget)

    def attend(self, q: torch.Tensor, seed: int, step: int, scale: float = 0.0, debug=None,
               T: Optional[int] = None) -> torch.Tensor:
        """The layer's attention output for queries q [B, Hq, d] over the
        prompt (sampled, or dense) and the first T suffix rows (default: those
        generated so far)."""
        T = self.T if T is None else T
        if self.continuations > 1:
            return prefix_decode(q, self.K, self.V, self.sK, self.sV, T=T, scale=scale, out=self.out, workspace=self.ws)
        if self.dense:
            return dense_decode(q, self.K, self.V, self.sK, self.sV, scale=scale, out=self.out, workspace=self.ws, T=T)
        return decode(self.teams, q, self.sK, self.sV, self.budget, seed=seed, step=step, scale=scale,
                      out=self.out, workspace=self.ws, debug=debug, T=T)

    def append(self, k: torch.Tensor, v: torch.Tensor) -> None:
        """Append one generated row per (b, kv): k, v [B, Hkv, d]."""
        if self.T >= self.capacity:
            raise ValueError(f"suffix cache full ({self.capacity} rows)")
        self.sK[:, :, self.T].copy_(k)
        self.sV[:, :, self.T].copy_(v)
        self.T += 1

    def rotate_append(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rotary: Rotary) -> torch.Tensor:
        """Append one generated row per (b, kv) from unrotated k and v [B, Hkv, d]
        and return the queries q [B, Hq, d] of the same token rotated (fp32; the
        layer's buffer, valid until the next call), in one launch."""
        if self.T >= self.capacity:
            raise ValueError(f"suffix cache full ({self.capacity} rows)")
        if self.q is None:
            self.q = torch.empty((self.B, self.Hq, self.d), dtype=torch.float32, device=self.sK.device)
        rope_append(q, k, v, self.sK, self.sV, rotary.freqs, self.T, first=self.N, interleaved=rotary.interleaved,
                    magnitude=rotary.magnitude, q_out=self.q)
        self.T += 1
        return self.q

    def close(self) -> None:
        if self.teams is not None:
            self.teams.close()
            self.teams = None


class DecodeLoop:
    """Layers decoded in order at every step; layer l draws its sampling
    noise with seed `seed + l` (each layer's noise stream is its own).  With
    ``rotary``, the steps' queries and keys come unrotated.  ``continuations``:
    sequences per prompt of a dense loop."""

    def __init__(self, prompts: Sequence[tuple], capacity: int, Hq: int, budget: int, P: int, R: int,
                 seed: int = 0, dense: bool = False, rotary: Optional[Rotary] = None, continuations: int = 1):
        self.layers: List[LayerCache] = [LayerCache(K, V, capacity, Hq, budget, P, R, dense, continuations)
                                         for K, V in prompts]
        self.rotary = rotary
        self.seed = seed
        self.step_id = 0

    def step(self, qs: Sequence[torch.Tensor], ks: Sequence[torch.Tensor], vs: Sequence[torch.Tensor],
             scale: float = 0.0, debugs=None) -> List[torch.Tensor]:
        """One decode step: layer l attends with qs[l], then appends ks[l],
        vs[l].  Returns each layer's output (views of the layer's buffer,
        valid until the next step)."""
        outs = []
        for li, layer in enumerate(self.layers):
            dbg = debugs[li] if debugs is not None else None
            if self.rotary is not None:
                T = layer.T
                q = layer.rotate_append(qs[li], ks[li], vs[li], self.rotary)
                outs.append(layer.attend(q, self.seed + li, self.step_id, scale, dbg, T=T))
                continue
            outs.append(layer.attend(qs[li], self.seed + li, self.step_id, scale, dbg))
            layer.append(ks[li], vs[li])
        self.step_id += 1
        return outs

    def close(self) -> None:
        for layer in self.layers:
            layer.close()
