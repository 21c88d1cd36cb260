"""The norm over a set of gradients and their clipping (dgnn_grad_norm, dgnn_grad_clip), between the gradients that a trainer leaves
(Section "Gradient Checkpoint") and the update of the weights.  A table of the tensors and a workspace; the arithmetic is in the HIP kernels."""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding as B
from .batch import Table, _data_ptr, _is_contiguous, _numel


class Gradients:
    """Gradient tensors (float32 or bfloat16, contiguous, any shapes, on one GPU) that are looked at together, where they lie: the table
    holds their addresses and sizes, so they are bound once and refilled by every step; a tensor that was given other memory since is bound()
    anew ahead of the next call.  `out`: tensors of the same shapes and types that receive the clipped gradients (left out: the gradients
    themselves)."""

    G, OUT, COUNT, DT = range(4)                     # dgnn_grad_item

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        self.grads, self.out = list(grads), list(grads) if out is None else list(out)
        if not self.grads or len(self.out) != len(self.grads):
            raise ValueError("Gradients takes one tensor at least, and as many outputs")
        dev = self.grads[0].device
        if dev.type != "cuda":
            raise ValueError("Gradients takes tensors on the GPU")
        for g, o in zip(self.grads, self.out):
            if o.shape != g.shape or o.dtype != g.dtype or g.device != dev or o.device != dev:
                raise ValueError("shape, dtype or device mismatch in Gradients")
        self.in_place = all(o is g for o, g in zip(self.out, self.grads))
        self.counts, self.index = list(map(_numel, self.grads)), self.grads[0].get_device()
        self.table = Table(len(self.grads), 4)
        self.bind()
        self.table.column(self.COUNT, self.counts)
        self.table.column(self.DT, [B._dtype_code(g) for g in self.grads])
        self.result = torch.zeros(1, dtype=torch.float32, device=dev)
        self.scalar = self.result[0]
        self.ws = torch.empty(B.grad_clip_workspace(len(self.grads)), dtype=torch.uint8, device=dev)

    def bind(self) -> None:
        """The addresses as they are now, after a tensor was given other memory (which is rare) of the same size."""
        self.table.column(self.G, self._addresses(self.grads))
        self.table.column(self.OUT, self.table.words[:, self.G] if self.in_place else self._addresses(self.out))

    def _addresses(self, tensors: List[torch.Tensor]) -> List[int]:
        if list(map(_numel, tensors)) != self.counts or any(t.get_device() != self.index for t in tensors):
            raise ValueError("a tensor of Gradients has another size or device than it was bound with")
        if not all(map(_is_contiguous, tensors)):
            raise AssertionError("dgnn takes contiguous tensors")
        return list(map(_data_ptr, tensors))

    def norm(self) -> torch.Tensor:
        """sqrt(sum g^2) over all of them: a scalar on the device, overwritten by the next call."""
        B.grad_norm(len(self.grads), self.table.at(), self.result, self.ws)
        return self.scalar

    def clip(self, max_norm: float) -> torch.Tensor:
        """out = g min(1, max_norm / (norm + 1e-6)); returns the norm from before, the same scalar as norm().  A norm that is no finite number
        changes nothing."""
        B.grad_clip(len(self.grads), self.table.at(), max_norm, self.result, self.ws)
        return self.scalar


class ClipsGradients:
    """What a trainer has to do with its gradients before they are applied: clip_gradients() between backward() and the update."""

    _clipped = None

    def parameter_gradients(self) -> List[torch.Tensor]:
        """The gradients that backward() leaves."""
        raise NotImplementedError

    def clip_gradients(self, max_norm: float) -> torch.Tensor:
        """Scales them, where they lie, so that the norm over all of them is at most max_norm; returns the norm from before, a scalar on
        the device that the next call overwrites.  A norm that is no finite number changes nothing."""
        grads = self.parameter_gradients()
        bound = self._clipped
        if bound is None or len(bound.grads) != len(grads) or any(a is not b for a, b in zip(bound.grads, grads)):
            bound = self._clipped = Gradients(grads)
        else:
            try:
                bound.bind()
            except ValueError:                       # a gradient of another size
                bound = self._clipped = Gradients(grads)
        return bound.clip(max_norm)


class ClipsBlockGradients(ClipsGradients):
    """The same for a trainer over a block: `dw`, or dw_t[timestep][layer] where every timestep has weights of its own.  Those are either
    parameters themselves, or come out of EvolvingWeights, whose backward() forms the parameters' gradients from dw_t: then it is its
    gradients that are clipped, afterwards, and it refuses a dw_t that was scaled ahead of it."""

    _timesteps_clipped = False

    def parameter_gradients(self) -> List[torch.Tensor]:
        return self.dw if self.dw_t is None else [g for t in range(self.blk.T) for g in self.dw_t[t]]

    def clip_gradients(self, max_norm: float) -> torch.Tensor:
        norm = super().clip_gradients(max_norm)
        if self.dw_t is not None:
            self._mark_timesteps(True)
        return norm

    def _mark_timesteps(self, clipped: bool) -> None:
        """backward() takes the mark off again."""
        if clipped or self._timesteps_clipped:
            for layers in self.dw_t:
                for g in layers:
                    g.clipped = clipped
        self._timesteps_clipped = clipped
