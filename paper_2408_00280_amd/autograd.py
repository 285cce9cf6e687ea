"""The fused LIF layer as a torch autograd function and module.

This is the programming model of the paper's Listing 1 (a ``FusedLIF`` autograd function
wrapping the fused forward and backward kernels, and a ``LIFLayer`` module to drop into
``torch.nn.Sequential`` next to ANN operators), with two differences: the state the
backward needs (the input current and the membrane checkpoints) is saved explicitly, and
the backward returns no gradient for the hyper-parameters.

Inputs are time-major, ``x[T, ...]``, float32 or bfloat16; the output is the spike train
``y[T, ...]`` as 0/1 values of the same dtype.  The arithmetic runs in the HIP kernels;
torch allocates and orders the work on its current stream.

Beside the LIF layers stand the sequence operators that join them in one block, on the same
[T, B, F] data: causal_conv / CausalConv, selective_scan / SelectiveScan and block_norm /
BlockNorm.
"""
from __future__ import annotations

import functools
import math

import torch

from . import layer

_IO = {torch.float32: "f32", torch.bfloat16: "bf16"}


class FusedLIF(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x: torch.Tensor, cfg: layer.LifConfig):
        if x.dtype not in _IO or cfg.io != _IO[x.dtype] or cfg.spk != "io":
            raise TypeError("FusedLIF takes float32/bfloat16 input and a cfg with io matching it and spk='io'")
        xc = x.contiguous()
        T = xc.shape[0]
        x2 = xc.view(T, -1)
        spikes, saved, _ = layer.forward(cfg, x2)
        ctx.save_for_backward(x2, saved)
        ctx.cfg = cfg
        ctx.shape = x.shape
        return spikes.view(x.shape)

    @staticmethod
    def backward(ctx, grad_y: torch.Tensor):
        x2, saved = ctx.saved_tensors
        g = grad_y.to(x2.dtype).contiguous().view(x2.shape)
        grad_x = layer.backward(ctx.cfg, x2, saved, g)
        return grad_x.view(ctx.shape), None


class LIFLayer(torch.nn.Module):
    """Leaky integrate-and-fire neurons over the leading (time) axis of the input.

    decay is k_tau of Eq. (1) (k_tau = 1 - 1/tau), v_th the threshold of Eq. (2), v_reset
    V_rest (initial membrane and hard-reset value), alpha the sigmoid-surrogate sharpness,
    reset "hard" (Eq. (1)) or "soft" (subtract the threshold)."""

    def __init__(self, decay: float, v_th: float, v_reset: float = 0.0, alpha: float = 4.0, reset: str = "hard"):
        super().__init__()
        self.decay, self.v_th, self.v_reset, self.alpha, self.reset = decay, v_th, v_reset, alpha, reset

    def cfg(self, dtype: torch.dtype) -> layer.LifConfig:
        return layer.LifConfig(self.decay, self.v_th, self.v_reset, self.alpha, self.reset, _IO[dtype], "io")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return FusedLIF.apply(x, self.cfg(x.dtype))

    def extra_repr(self) -> str:
        return (f"decay={self.decay}, v_th={self.v_th}, v_reset={self.v_reset}, alpha={self.alpha}, "
                f"reset={self.reset}")


class FusedGainLIF(torch.autograd.Function):
    """A LIF layer fed by the previous layer's spikes through a fixed per-feature gain:
    input current gain[f] * spikes_in[t, ..., f], formed inside the fused kernels (the gain
    rounded to the I/O dtype first).  The backward returns dL/d spikes_in = gain[f] * dL/dx
    with the same rounded gain; the gain gets no gradient."""

    @staticmethod
    def forward(ctx, spikes_in: torch.Tensor, gain: torch.Tensor, cfg: layer.LifConfig):
        if spikes_in.dtype not in _IO or cfg.io != _IO[spikes_in.dtype] or cfg.spk != "io":
            raise TypeError("FusedGainLIF takes float32/bfloat16 spikes and a cfg with io matching them and spk='io'")
        F = gain.numel()
        if spikes_in.shape[-1] != F or gain.dtype != torch.float32:
            raise ValueError("gain must be float32 with one entry per feature (the last axis of spikes_in)")
        s = spikes_in.contiguous()
        T = s.shape[0]
        B = s.numel() // (T * F) if T else 0
        s2 = s.view(T, B * F)
        g = gain.contiguous()
        spikes, saved, _ = layer.forward_gain(cfg, s2, g, B, F)
        ctx.save_for_backward(s2, g, saved)
        ctx.cfg, ctx.shape, ctx.BF = cfg, spikes_in.shape, (B, F)
        return spikes.view(spikes_in.shape)

    @staticmethod
    def backward(ctx, grad_y: torch.Tensor):
        s2, g, saved = ctx.saved_tensors
        B, F = ctx.BF
        gy = grad_y.to(s2.dtype).contiguous().view(s2.shape)
        grad_in = layer.backward_gain(ctx.cfg, s2, g, saved, gy, B, F)
        return grad_in.view(ctx.shape), None, None


class GainLIF(torch.nn.Module):
    """LIF neurons fed by spikes through a fixed per-feature gain (the feature axis is the
    last one): the fused form of ``x = gain * spikes`` followed by a :class:`LIFLayer`, with
    the same spikes and membranes and without storing x."""

    def __init__(self, gain: torch.Tensor, decay: float, v_th: float, v_reset: float = 0.0, alpha: float = 4.0,
                 reset: str = "hard"):
        super().__init__()
        self.register_buffer("gain", gain.detach().to(torch.float32).contiguous())
        self.decay, self.v_th, self.v_reset, self.alpha, self.reset = decay, v_th, v_reset, alpha, reset

    def cfg(self, dtype: torch.dtype) -> layer.LifConfig:
        return layer.LifConfig(self.decay, self.v_th, self.v_reset, self.alpha, self.reset, _IO[dtype], "io")

    def forward(self, spikes_in: torch.Tensor) -> torch.Tensor:
        return FusedGainLIF.apply(spikes_in, self.gain, self.cfg(spikes_in.dtype))

    def extra_repr(self) -> str:
        return (f"features={self.gain.numel()}, decay={self.decay}, v_th={self.v_th}, v_reset={self.v_reset}, "
                f"alpha={self.alpha}, reset={self.reset}")


class FusedLIFStack(torch.autograd.Function):
    """len(gains) + 1 LIF layers joined by fixed per-feature gains, fused across depth and
    time: one kernel per direction for the whole stack.  Returns the last layer's spikes;
    the backward returns dL/dx of the first layer (the gains get no gradient)."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, gains: torch.Tensor, cfg: layer.LifConfig):
        if x.dtype not in _IO or cfg.io != _IO[x.dtype] or cfg.spk != "io":
            raise TypeError("FusedLIFStack takes float32/bfloat16 input and a cfg with io matching it and spk='io'")
        F = gains.shape[1]
        if x.shape[-1] != F:
            raise ValueError("gains must have one column per feature (the last axis of x)")
        xc = x.contiguous()
        T = xc.shape[0]
        B = xc.numel() // (T * F) if T else 0
        x2 = xc.view(T, B * F)
        g = gains.to(torch.float32).contiguous()
        spikes, _, saved, _ = layer.stack_forward(cfg, x2, g, B, F)
        ctx.save_for_backward(x2, g, saved)
        ctx.cfg, ctx.shape, ctx.BF = cfg, x.shape, (B, F)
        return spikes.view(x.shape)

    @staticmethod
    def backward(ctx, grad_y: torch.Tensor):
        x2, g, saved = ctx.saved_tensors
        B, F = ctx.BF
        gy = grad_y.to(x2.dtype).contiguous().view(x2.shape)
        grad_x = layer.stack_backward(ctx.cfg, x2, g, saved, gy, B, F)
        return grad_x.view(ctx.shape), None, None


class LIFStack(torch.nn.Module):
    """2 or 3 LIF layers joined by fixed per-feature gains (gains: [L-1, F], the feature axis
    last), run as one fused kernel per direction: the same spikes as LIFLayer followed by
    GainLIF layers, without their intermediate tensors."""

    def __init__(self, gains: torch.Tensor, decay: float, v_th: float, v_reset: float = 0.0, alpha: float = 4.0,
                 reset: str = "hard"):
        super().__init__()
        self.register_buffer("gains", gains.detach().to(torch.float32).contiguous())
        self.decay, self.v_th, self.v_reset, self.alpha, self.reset = decay, v_th, v_reset, alpha, reset

    def cfg(self, dtype: torch.dtype) -> layer.LifConfig:
        return layer.LifConfig(self.decay, self.v_th, self.v_reset, self.alpha, self.reset, _IO[dtype], "io")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return FusedLIFStack.apply(x, self.gains, self.cfg(x.dtype))

    def extra_repr(self) -> str:
        return (f"layers={self.gains.shape[0] + 1}, features={self.gains.shape[1]}, decay={self.decay}, "
                f"v_th={self.v_th}, v_reset={self.v_reset}, alpha={self.alpha}, reset={self.reset}")


@functools.cache
def _ops():
    """The sequence operators, at their first use: the LIF layers do without their module."""
    from . import sequence
    return sequence


def causal_conv(x, weight, bias=None, *, act="silu", state=None, lengths=None, return_state=False):
    """Short causal convolution of x[T, B, F] along time (see sequence.conv_forward), with
    gradients for x, weight, bias and state.  Returns y, or (y, the last W-1 inputs)."""
    ops = _ops()
    out = ops._sequence.causal_conv(x, weight, bias, ops.act_code(act), state, lengths, return_state)
    return out if return_state else out[0]


class CausalConv(torch.nn.Module):
    """Short causal convolution along the leading (time) axis, one filter per feature, with
    bias and activation (None or "silu")."""

    def __init__(self, features: int, width: int = 4, bias: bool = True, act: str | None = "silu"):
        super().__init__()
        bound = 1 / math.sqrt(width)
        self.weight = torch.nn.Parameter(torch.empty(features, width).uniform_(-bound, bound))
        self.bias = torch.nn.Parameter(torch.empty(features).uniform_(-bound, bound)) if bias else None
        self.act = act

    def _args(self):
        return self.weight.float(), None if self.bias is None else self.bias.float()

    def forward(self, x, *, state=None, lengths=None, return_state=False):
        return causal_conv(x, *self._args(), act=self.act, state=state, lengths=lengths, return_state=return_state)

    @torch.no_grad()
    def step(self, x, state):
        """One step x[B, F] on state[W-1, B, F], which is updated in place: y[B, F]."""
        return _ops().conv_forward(x[None], *self._args(), act=self.act, state=state, state_out=state)[0]

    def extra_repr(self) -> str:
        return f"features={self.weight.shape[0]}, width={self.weight.shape[1]}, act={self.act}"


def selective_scan(x, dt, A, Bm, Cm, D=None, dt_bias=None, *, softplus=True, h_in=None, lengths=None,
                   return_state=False):
    """Selective state space scan of x[T, B, F] (see sequence.scan_forward), with gradients for
    every input.  Returns y, or (y, the state [B, F, S] after the last step)."""
    out = _ops()._sequence.selective_scan(x, dt, A, Bm, Cm, D, dt_bias, bool(softplus), h_in, lengths, return_state)
    return out if return_state else out[0]


class SelectiveScan(torch.nn.Module):
    """Selective state space scan along the leading (time) axis: rates A = -exp(A_log) [F, S],
    skip weights D and step biases dt_bias [F]; x, dt [T, B, F] and B, C [T, B, G, S] are
    inputs (projections of the block's input)."""

    def __init__(self, features: int, states: int = 16, dt_min: float = 1e-3, dt_max: float = 0.1):
        super().__init__()
        rates = torch.arange(1, states + 1, dtype=torch.float32).expand(features, states)
        self.A_log = torch.nn.Parameter(torch.log(rates))
        self.D = torch.nn.Parameter(torch.ones(features))
        dt = torch.exp(torch.empty(features).uniform_(math.log(dt_min), math.log(dt_max)))
        self.dt_bias = torch.nn.Parameter(torch.log(torch.expm1(dt)))     # softplus(dt_bias) = dt

    def _A(self):
        return -torch.exp(self.A_log.float())

    def forward(self, x, dt, Bm, Cm, *, h_in=None, lengths=None, return_state=False):
        return selective_scan(x, dt, self._A(), Bm, Cm, self.D.float(), self.dt_bias.float(), h_in=h_in,
                              lengths=lengths, return_state=return_state)

    @torch.no_grad()
    def step(self, x, dt, Bm, Cm, h):
        """One step x, dt [B, F], Bm, Cm [B, G, S] on the state h[B, F, S], which is updated in
        place: y[B, F]."""
        y, _ = _ops().scan_forward(x[None], dt[None], self._A(), Bm[None], Cm[None], self.D.float(),
                                   self.dt_bias.float(), h_in=h, h_out=h)
        return y[0]

    def extra_repr(self) -> str:
        return f"features={self.A_log.shape[0]}, states={self.A_log.shape[1]}"


def block_norm(y, r=None, z=None, w_post=None, scale=None, w_pre=None, *, eps=1e-5, lengths=None):
    """A block's gate, norm and scaled residual with the next block's norm (see
    sequence.norm_forward), with gradients for every input: (r_new, u or None)."""
    out = _ops()._sequence.block_norm(y, r, z, w_post, scale, w_pre, lengths, eps)
    return out[0], out[1] if w_pre is not None else None


class BlockNorm(torch.nn.Module):
    """The end of a block and the start of the next: r_new = r + scale * norm(y * silu(z)) and
    u = norm(r_new), with learned weights for both norms and the scale (each can be left out)."""

    def __init__(self, features: int, *, post: bool = True, scale: float | None = 1.0, pre: bool = True,
                 eps: float = 1e-5):
        super().__init__()
        self.w_post = torch.nn.Parameter(torch.ones(features)) if post else None
        self.scale = torch.nn.Parameter(torch.full((features,), float(scale))) if scale is not None else None
        self.w_pre = torch.nn.Parameter(torch.ones(features)) if pre else None
        self.features, self.eps = features, eps

    def forward(self, y, r=None, z=None, *, lengths=None):
        w = (None if p is None else p.float() for p in (self.w_post, self.scale, self.w_pre))
        return block_norm(y, r, z, *w, eps=self.eps, lengths=lengths)

    def extra_repr(self) -> str:
        parts = [n for n in ("w_post", "scale", "w_pre") if getattr(self, n) is not None]
        return f"features={self.features}, {', '.join(parts)}, eps={self.eps}"
