"""Caller-side plumbing for a state-space layer over a block of timesteps, forward, backward and one timestep at a time: what may take the
LSTM's place over the frames of a GCN (Section "CD-GCN" aggregates over time per vertex; here the recurrence is linear and gated by its
input).  With frames x [T, n, f] and an inner width d,

    u0 = x W_in,  z = x W_z            dgnn_feature_transform        u = silu(conv(u0))             dgnn_causal_conv
    delta = u W_dt,  bc = u W_bc       dgnn_feature_transform        y = scan(u, delta, bc, z)      dgnn_selective_scan
    out = y W_out                      dgnn_feature_transform

Sequences are vertices; `lengths` says how many timesteps of the block each has (frames and gradients behind them may hold anything).  A series in blocks (Section "Gradient Checkpoint"): the
layer holds the last frames and the state between calls, and backward() takes and leaves their gradients.  Buffers and call order only;
the arithmetic is in the HIP kernels."""
from __future__ import annotations

from typing import Dict, List, Optional

import torch

from . import binding as B
from .gradients import ClipsGradients

WEIGHTS = ("w_in", "w_z", "w_dt", "w_bc", "w_out")
PARAMETERS = ("taps", "conv_bias", "a", "d", "dt_bias")


class StateSpaceLayer(ClipsGradients):
    """`weights`: w_in, w_z [f, d], w_dt [d, d], w_bc [d, 2 N], w_out [d, f] in the frames' type; taps [w, d], conv_bias [d], a [d, N],
    d [d], dt_bias [d] in float32.  f, d and 2 N are feature widths of the dense transform.  Gradients (float32) are in `grads`."""

    def __init__(self, n: int, T: int, weights: Dict[str, torch.Tensor], lengths: Optional[torch.Tensor] = None):
        self.n, self.T, self.weights, self.lengths = n, T, weights, lengths
        w_in, taps, a = weights["w_in"], weights["taps"], weights["a"]
        (f, d), (w, _), (_, states) = w_in.shape, taps.shape, a.shape
        self.f, self.d, self.states, self.dtype = f, d, states, w_in.dtype
        shapes = dict(w_in=(f, d), w_z=(f, d), w_dt=(d, d), w_bc=(d, 2 * states), w_out=(d, f), taps=(w, d), conv_bias=(d,), a=(d, states), d=(d,), dt_bias=(d,))
        for name, shape in shapes.items():
            if tuple(weights[name].shape) != shape or weights[name].dtype != (w_in.dtype if name in WEIGHTS else torch.float32):
                raise ValueError(f"{name}: expected {shape}")
        dev = w_in.device
        self.dev = dev
        empty = lambda *shape: torch.empty(shape, dtype=self.dtype, device=dev)  # noqa: E731
        self.u0, self.u, self.z, self.delta, self.y = (empty(T, n, d) for _ in range(5))
        self.bc, self.out = empty(T, n, 2 * states), empty(T, n, f)
        self.frames = torch.zeros((w - 1, n, d), dtype=self.dtype, device=dev)         # the last frames of u0, the state: ahead of the next block
        self.state = torch.zeros((n, d, states), device=dev)
        self.frames_before = torch.empty_like(self.frames)                             # ... and ahead of the block that backward() is for
        self.ws = torch.empty(B.selective_scan_workspace(T, n, d, states), dtype=torch.uint8, device=dev)
        self.one = [empty(1, n, width) for width in (d, d, d, d, d, 2 * states, f)]    # the same of one timestep: step() leaves the block's alone
        self.checkpoints = self.grads = self.x = None

    def reset(self) -> None:
        """The start of a series: no frames, no state."""
        self.frames.zero_()
        self.state.zero_()

    def _project(self, x: torch.Tensor, name: str, to: torch.Tensor) -> None:
        B.feature_transform(x.reshape(-1, x.shape[-1]), self.weights[name], to.view(-1, to.shape[-1]))

    def _run(self, x: torch.Tensor, buffers, lengths, checkpoints) -> torch.Tensor:
        p, (u0, u, z, delta, y, bc, out) = self.weights, buffers
        self._project(x, "w_in", u0)
        self._project(x, "w_z", z)
        B.causal_conv(u0, p["taps"], p["conv_bias"], u, silu=True, x_before=self.frames, x_after=self.frames, lengths=lengths)
        self._project(u, "w_dt", delta)
        self._project(u, "w_bc", bc)
        B.selective_scan(u, delta, bc, p["a"], y, self.ws, z=z, d=p["d"], dt_bias=p["dt_bias"], h_before=self.state, h_after=self.state, checkpoints=checkpoints,
                         lengths=lengths)
        self._project(y, "w_out", out)
        return out

    def _check(self, x: torch.Tensor, shape) -> None:
        if tuple(x.shape) != shape or x.dtype != self.dtype or x.device != self.dev:
            raise ValueError(f"StateSpaceLayer: expected {self.dtype} frames of shape {shape} on {self.dev}")

    def forward(self, x: torch.Tensor, train: bool = False) -> torch.Tensor:
        """The block's output frames [T, n, f] (a buffer of the layer's) from the state as it stands, which moves on to the block's end.
        train: backward() may follow, and looks at x once more."""
        self._check(x, (self.T, self.n, self.f))
        if x.untyped_storage().data_ptr() == self.out.untyped_storage().data_ptr():
            raise ValueError("StateSpaceLayer: the frames are the layer's own output buffer")
        self.x = None
        if train:
            if self.checkpoints is None:
                self.checkpoints = torch.empty(B.selective_scan_checkpoints(self.T, self.n, self.d, self.states), device=self.dev)
            self.frames_before.copy_(self.frames)
        out = self._run(x, (self.u0, self.u, self.z, self.delta, self.y, self.bc, self.out), self.lengths, self.checkpoints if train else None)
        if train:
            self.x = x                                                                 # not ahead of a call that is refused half way
        return out

    def step(self, x: torch.Tensor, lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One timestep further: frames [n, f] in and out (a buffer of the layer's, which the next step may take in).  lengths [n] int32, 1 or 0: a
        sequence of 0 keeps its frames and its state, its output is zero.  Without them every sequence moves on, those too that ended inside
        of the block."""
        self._check(x, (self.n, self.f))
        return self._run(x[None], self.one, lengths, None)[0]

    def _training_buffers(self) -> None:
        empty = lambda like: torch.empty_like(like)  # noqa: E731
        self.grads = {k: torch.zeros(self.weights[k].shape, device=self.dev) for k in WEIGHTS + PARAMETERS}
        self.g_y, self.dz, self.du, self.ddelta, self.du0, self.more = (empty(self.y) for _ in range(6))
        self.dbc, self.dx, self.dx_more = empty(self.bc), empty(self.out), empty(self.out)
        self.dframes, self.dstate = empty(self.frames), empty(self.state)
        self.as_it_is = torch.zeros((2, self.f), device=self.dev)                      # the taps of a convolution that changes nothing
        self.as_it_is[0] = 1.0
        need = [B.selective_scan_backward_workspace(self.T, self.n, self.d, self.states),
                B.causal_conv_backward_workspace(self.T, self.n, self.d, self.weights["taps"].shape[0])]
        need += [B.weight_grad_workspace(*self.weights[k].shape) for k in WEIGHTS]
        self.ws_back = torch.empty(max(need), dtype=torch.uint8, device=self.dev)

    def _there(self, t: torch.Tensor) -> torch.Tensor:
        """Frames [T, n, f] with zeros behind the sequences' ends, in dx_more: a weight gradient sums over all rows, where what lies there (anything)
        meets zeros, and zero times NaN or infinity is NaN."""
        if self.lengths is None:
            return t
        B.causal_conv(t.contiguous(), self.as_it_is, None, self.dx_more, lengths=self.lengths)
        return self.dx_more

    def backward(self, g_out: torch.Tensor, behind=None, accumulate: bool = False) -> torch.Tensor:
        """g_out [T, n, f] = dL/d(output frames) of the last forward(), which was one with train; returns dL/dx [T, n, f].  behind = (gradient of the frames,
        gradient of the state) that the block behind leaves in (dframes, dstate); this one's are there afterwards (pass copies of them
        on to the block ahead of this one, or this layer's own where the blocks share it).  accumulate adds to grads."""
        self._check(g_out, (self.T, self.n, self.f))
        if self.x is None:
            raise ValueError("StateSpaceLayer: backward() follows forward(train=True)")
        if self.grads is None:
            self._training_buffers()
        if behind is not None:
            behind = tuple(t.clone() if t is mine else t for t, mine in zip(behind, (self.dframes, self.dstate)))
        dframes, dstate = behind or (None, None)
        p, g, ws, flat = self.weights, self.grads, self.ws_back, lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        wgrad = lambda x, gy, name: B.weight_grad(flat(x), flat(gy), g[name], ws, accumulate=accumulate)  # noqa: E731
        wgrad(self.y, self._there(g_out), "w_out")
        B.input_grad(flat(g_out), p["w_out"], flat(self.g_y))
        B.selective_scan_backward(self.u, self.delta, self.bc, p["a"], self.g_y, self.checkpoints, self.du, self.ddelta, self.dbc, g["a"], ws, z=self.z, dz=self.dz,
                                  d=p["d"], dd=g["d"], dt_bias=p["dt_bias"], ddt_bias=g["dt_bias"], dh_after=dstate, dh_before=self.dstate, lengths=self.lengths,
                                  accumulate=accumulate)
        for grad, name in ((self.ddelta, "w_dt"), (self.dbc, "w_bc")):
            wgrad(self.u, grad, name)
            B.input_grad(flat(grad), p[name], flat(self.more))
            B.add(flat(self.du), flat(self.more), flat(self.du))
        B.causal_conv_backward(self.u0, p["taps"], p["conv_bias"], self.du, self.du0, g["taps"], g["conv_bias"], ws, silu=True, x_before=self.frames_before,
                               dx_after=dframes, dx_before=self.dframes, lengths=self.lengths, accumulate=accumulate)
        x = self._there(self.x)
        wgrad(x, self.du0, "w_in")
        wgrad(x, self.dz, "w_z")
        B.input_grad(flat(self.du0), p["w_in"], flat(self.dx))
        B.input_grad(flat(self.dz), p["w_z"], flat(self.dx_more))
        B.add(flat(self.dx), flat(self.dx_more), flat(self.dx))
        return self.dx

    def parameter_gradients(self) -> List[torch.Tensor]:
        if self.grads is None:
            raise ValueError("StateSpaceLayer: no backward() so far")
        return list(self.grads.values())
