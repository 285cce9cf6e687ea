"""Torch-tensor conveniences over the sequence operators of include/snn_seq.h: a short causal
convolution, a selective state space scan, and a block's gate, norm and scaled residual with
the next block's norm.

Data is [T, B, F] in float32 or bfloat16, as the LIF layers of this package take it, in any
strides whose last axis is contiguous: time-major, batch-major (a transposed [B, T, F]) and
slices of wider rows are read in place, anything else is copied first.  Parameters and their
gradients are float32.  ``lengths`` (int32 [B]) gives each sequence its own number of steps:
what lies behind is not read, and is 0 in outputs and gradients.

Checks, outputs and workspaces are made in csrc_seq/seq_torch.cpp, which calls the C ABI; wrong
arguments raise ValueError, refused ones native.SnnError.  Torch provides device memory and
streams only.  Work is enqueued on torch's current stream of the tensors' device, or on ``stream``
(a torch.cuda.Stream of that device or a raw handle): then the order of the two streams is the
caller's.  Memory of tensors that are dropped meanwhile is kept until a torch.cuda.Stream is done
with it; behind a raw handle, whose life torch does not know, the caller keeps them.
"""
from __future__ import annotations

import functools

import torch

from . import native

try:
    from . import _sequence
except ImportError as e:
    raise ImportError("the sequence operators are not built; run __graft_entry__.build()") from e

IO_OF = {torch.float32: native.SNN_IO_F32, torch.bfloat16: native.SNN_IO_BF16}
ACTS = {None: native.SNN_ACT_NONE, "silu": native.SNN_ACT_SILU}


def act_code(act) -> int:
    if act not in ACTS:
        raise ValueError("act must be None or 'silu'")
    return ACTS[act]


def _tensors(values):
    return [v for v in values if isinstance(v, torch.Tensor) and v.is_cuda]


def _on_stream(fn):
    """fn on `stream`, which belongs to its first tensor's device."""
    first = fn.__code__.co_varnames[0]

    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        x = args[0] if args else kw[first]
        if not x.is_cuda:
            raise ValueError("tensors must be on the GPU")
        known = isinstance(stream, torch.cuda.Stream)
        if known and stream.device != x.device:
            raise ValueError(f"stream is one of {stream.device}, the tensors are on {x.device}")
        with torch.cuda.device(x.device):
            if not known:
                stream = torch.cuda.ExternalStream(int(stream)) if stream else torch.cuda.default_stream()
            current = torch.cuda.current_stream()
            with torch.cuda.stream(stream):
                out = fn(*args, **kw)
            if known and stream != current:
                # neither side's memory goes to another tensor while the other side may be using it
                for t in _tensors([*args, *kw.values()]):
                    t.record_stream(stream)
                for t in _tensors(out if isinstance(out, tuple) else [out]):
                    t.record_stream(current)
            return out
    return call


@_on_stream
def conv_forward(x, weight, bias=None, *, act="silu", state=None, state_out=None, lengths=None):
    """Causal convolution of x[T, B, F] along time with weight[F, W] (W up to 8, the last tap
    on the current step), bias[F] and activation: y.  state ([W-1, B, F]): the inputs before
    step 0; state_out: written with the last W-1 inputs, may be `state` (in place)."""
    return _sequence.conv_forward(x, weight, bias, act_code(act), state, state_out, lengths)


@_on_stream
def conv_backward(x, weight, bias, grad_y, *, act="silu", state=None, lengths=None, grad_state_out=None):
    """Gradients (x, weight, bias or None, state or None) of conv_forward with the same
    arguments; grad_state_out: the gradient of its state_out."""
    return _sequence.conv_backward(x, weight, bias, grad_y, act_code(act), state, lengths, grad_state_out)


@_on_stream
def scan_forward(x, dt, A, Bm, Cm, D=None, dt_bias=None, *, softplus=True, h_in=None, h_out=None, lengths=None,
                 train=False):
    """Selective scan of x[T, B, F] with steps softplus(dt + dt_bias) (dt [T, B, F], dt_bias
    [F]), rates A [F, S], Bm and Cm [T, B, G, S] (shared by the F/G features of a group) and
    skip weights D [F].  h_in, h_out ([B, F, S] float32): the state before step 0 and after
    the last, h_out is written and may be h_in (in place).  Returns (y, saved), saved for
    scan_backward with train=True and None otherwise."""
    return _sequence.scan_forward(x, dt, A, Bm, Cm, D, dt_bias, bool(softplus), h_in, h_out, lengths, bool(train))


@_on_stream
def scan_backward(x, dt, A, Bm, Cm, D, dt_bias, saved, grad_y, *, softplus=True, h_in=None, lengths=None,
                  grad_h_out=None):
    """Gradients (x, dt, A, Bm, Cm, D or None, dt_bias or None, h_in or None) of scan_forward
    with the same arguments and what it saved; grad_h_out: the gradient of its h_out."""
    return _sequence.scan_backward(x, dt, A, Bm, Cm, D, dt_bias, saved, grad_y, bool(softplus), h_in, lengths, grad_h_out)


@_on_stream
def norm_forward(y, r=None, z=None, w_post=None, scale=None, w_pre=None, *, eps=1e-5, lengths=None, train=False):
    """The end of a block and the start of the next over the last axis of y[T, B, F]:
    r_new = r + scale * norm(y * silu(z)) and u = norm(r_new), root-mean-square norms with the
    weights w_post and w_pre.  Without z, w_post, scale, r or w_pre that part is left out.
    Returns (r_new, u or None, rstd), rstd for norm_backward with train=True, else None."""
    return _sequence.norm_forward(y, r, z, w_post, scale, w_pre, eps, lengths, bool(train))


@_on_stream
def norm_backward(y, r, z, w_post, scale, w_pre, rstd, grad_r_new, grad_u=None, *, eps=1e-5, lengths=None):
    """Gradients (y, r, z, w_post, scale, w_pre; None where the input is None) of norm_forward
    with the same arguments and its rstd.  grad_r_new or grad_u may be None (no gradient)."""
    return _sequence.norm_backward(y, r, z, w_post, scale, w_pre, rstd, grad_r_new, grad_u, eps, lengths)
