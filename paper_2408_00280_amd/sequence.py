"""Torch-tensor conveniences over the sequence operators of include/snn_seq.h: a short causal
convolution, a selective state space scan, and a block's gate, norm and scaled residual with
the next block's norm.

Data is [T, B, F] in float32 or bfloat16, as the LIF layers of this package take it, in any
strides whose last axis is contiguous: time-major, batch-major (a transposed [B, T, F]) and
slices of wider rows are read in place, anything else is copied first.  Parameters and their
gradients are float32.  ``lengths`` (int32 [B]) gives each sequence its own number of steps:
what lies behind is not read, and is 0 in outputs and gradients.

Torch provides device memory and streams only.  Work is enqueued on torch's current stream
of the tensors' device, or on ``stream`` (a torch.cuda.Stream or a raw handle).
"""
from __future__ import annotations

import functools

import torch

from . import native

IO_OF = {torch.float32: native.SNN_IO_F32, torch.bfloat16: native.SNN_IO_BF16}
ACTS = {None: native.SNN_ACT_NONE, "silu": native.SNN_ACT_SILU}


# Configurations with the bytes of saved data and workspaces, which depend on nothing but
# configuration and shape: a call finds them in a dictionary instead of asking for them.

@functools.lru_cache(maxsize=256)
def _conv_plan(io, W, act, T, B, F):
    cfg = native.snn_conv_cfg(io, W, act)
    return cfg, native.snn_conv_workspace_bytes(cfg, T, B, F)


@functools.lru_cache(maxsize=256)
def _scan_plan(io, S, G, softplus, T, B, F):
    cfg = native.snn_scan_cfg(io, S, G, softplus)
    return cfg, native.snn_scan_saved_bytes(cfg, T, B, F), *native.snn_scan_workspace_bytes(cfg, T, B, F)


@functools.lru_cache(maxsize=256)
def _norm_plan(io, eps, T, B, F):
    cfg = native.snn_norm_cfg(io, eps)
    return cfg, native.snn_norm_workspace_bytes(cfg, T, B, F)


def _on_stream(fn):
    """fn with its first tensor's device as the current one, on `stream`."""
    first = fn.__code__.co_varnames[0]

    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        x = args[0] if args else kw[first]
        if not x.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if stream is None and x.get_device() == torch._C._cuda_getDevice():
            return fn(*args, **kw)
        with torch.cuda.device(x.device):
            if stream is None:
                return fn(*args, **kw)
            if not isinstance(stream, torch.cuda.Stream):
                stream = torch.cuda.ExternalStream(int(stream)) if stream else torch.cuda.default_stream()
            with torch.cuda.stream(stream):
                return fn(*args, **kw)
    return call


def _shape(x):
    if x.dim() != 3 or x.dtype not in IO_OF:
        raise ValueError("data must be a float32 or bfloat16 tensor [T, B, F]")
    return x.shape


def _rows(a):
    """`a` with the axes behind the second contiguous."""
    if a.is_contiguous():
        return a
    n = 1
    for size, step in zip(reversed(a.shape[2:]), reversed(a.stride()[2:])):
        if size != 1 and step != n:
            return a.contiguous()
        n *= size
    return a


def _data(name, a, x, shape):
    """`a` as [T, B, X] data that goes with x."""
    if a.dtype != x.dtype or a.shape != shape or a.get_device() != x.get_device():
        raise ValueError(f"{name} must be a {x.dtype} tensor of shape {tuple(shape)} on {x.device}")
    return _rows(a)


def _dense(name, a, x, shape, dtype=torch.float32):
    """The address of a parameter, a state or lengths; None without one."""
    if a is None:
        return None
    if a.dtype != dtype or a.shape != shape or not a.is_contiguous() or a.get_device() != x.get_device():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {x.device}")
    return a.data_ptr() or None


def _bytes(n, x):
    return x.new_empty(n, dtype=torch.uint8) if n else None


def _params(p, empty):
    """A parameter's gradient: the kernels write it whole, unless there is nothing to do."""
    return None if p is None else (torch.zeros_like if empty else torch.empty_like)(p)


def _hand_over(out, given):
    """No steps: the state out is the state in."""
    if out is not None and out is not given:
        out.zero_() if given is None else out.copy_(given)


# ---------------------------------------------------------------------------------------

def _conv_args(x, weight, bias, act, state, lengths):
    T, B, F = _shape(x)
    if weight.dim() != 2 or act not in ACTS:
        raise ValueError("weight must be [F, W], act None or 'silu'")
    W = weight.shape[1]
    x = _rows(x)
    args = (x, _dense("weight", weight, x, (F, W)), _dense("bias", bias, x, (F,)),
            _dense("state", state, x, (W - 1, B, F), x.dtype), _dense("lengths", lengths, x, (B,), torch.int32))
    return args, (T, B, F, W), _conv_plan(IO_OF[x.dtype], W, ACTS[act], T, B, F)


@_on_stream
def conv_forward(x, weight, bias=None, *, act="silu", state=None, state_out=None, lengths=None):
    """Causal convolution of x[T, B, F] along time with weight[F, W] (W up to 8, the last tap
    on the current step), bias[F] and activation: y.  state ([W-1, B, F]): the inputs before
    step 0; state_out: written with the last W-1 inputs, may be `state` (in place)."""
    args, (T, B, F, W), (cfg, _) = _conv_args(x, weight, bias, act, state, lengths)
    x = args[0]
    out = _dense("state_out", state_out, x, (W - 1, B, F), x.dtype)
    y = torch.empty_like(x)
    if T and B and F:
        native.snn_conv_forward(cfg, T, B, F, *args, y, out)
    else:
        _hand_over(state_out, state)
    return y


@_on_stream
def conv_backward(x, weight, bias, grad_y, *, act="silu", state=None, lengths=None, grad_state_out=None):
    """Gradients (x, weight, bias or None, state or None) of conv_forward with the same
    arguments; grad_state_out: the gradient of its state_out."""
    args, (T, B, F, W), (cfg, ws) = _conv_args(x, weight, bias, act, state, lengths)
    x = args[0]
    gy = _data("grad_y", grad_y, x, (T, B, F))
    g_out = _dense("grad_state_out", grad_state_out, x, (W - 1, B, F), x.dtype)
    empty = not (T and B and F)
    gx, gw, gb = torch.empty_like(x), _params(weight, empty), _params(bias, empty)
    gs = None if state is None else torch.empty_like(state)
    if empty:
        _hand_over(gs, grad_state_out)
    else:
        native.snn_conv_backward(cfg, T, B, F, *args, gy, g_out, gx, gw, gb, gs, _bytes(ws, x))
    return gx, gw, gb, gs


# ---------------------------------------------------------------------------------------

def _scan_args(x, dt, A, Bm, Cm, D, dt_bias, softplus, h_in, lengths):
    T, B, F = _shape(x)
    if Bm.dim() != 4 or A.dim() != 2:
        raise ValueError("A must be [F, S], Bm and Cm [T, B, G, S]")
    G, S = Bm.shape[2:]
    x, dt = _rows(x), _data("dt", dt, x, (T, B, F))
    Bm, Cm = _data("Bm", Bm, x, (T, B, G, S)), _data("Cm", Cm, x, (T, B, G, S))
    args = (x, dt, _dense("A", A, x, (F, S)), Bm, Cm, _dense("D", D, x, (F,)), _dense("dt_bias", dt_bias, x, (F,)),
            _dense("h_in", h_in, x, (B, F, S)), _dense("lengths", lengths, x, (B,), torch.int32))
    return args, (T, B, F, S), _scan_plan(IO_OF[x.dtype], S, G, int(bool(softplus)), T, B, F)


@_on_stream
def scan_forward(x, dt, A, Bm, Cm, D=None, dt_bias=None, *, softplus=True, h_in=None, h_out=None, lengths=None,
                 train=False):
    """Selective scan of x[T, B, F] with steps softplus(dt + dt_bias) (dt [T, B, F], dt_bias
    [F]), rates A [F, S], Bm and Cm [T, B, G, S] (shared by the F/G features of a group) and
    skip weights D [F].  h_in, h_out ([B, F, S] float32): the state before step 0 and after
    the last, h_out is written and may be h_in (in place).  Returns (y, saved), saved for
    scan_backward with train=True and None otherwise."""
    args, (T, B, F, S), (cfg, kept, ws, _) = _scan_args(x, dt, A, Bm, Cm, D, dt_bias, softplus, h_in, lengths)
    x = args[0]
    out = _dense("h_out", h_out, x, (B, F, S))
    if train and out is not None and out == args[7]:
        raise ValueError("the backward reads h_in: h_out must be another tensor")
    y = torch.empty_like(x)
    saved = x.new_empty(kept, dtype=torch.uint8) if train else None
    if T and B and F:
        native.snn_scan_forward(cfg, T, B, F, *args, y, out, saved if train and kept else None, _bytes(ws, x))
    else:
        _hand_over(h_out, h_in)
    return y, saved


@_on_stream
def scan_backward(x, dt, A, Bm, Cm, D, dt_bias, saved, grad_y, *, softplus=True, h_in=None, lengths=None,
                  grad_h_out=None):
    """Gradients (x, dt, A, Bm, Cm, D or None, dt_bias or None, h_in or None) of scan_forward
    with the same arguments and what it saved; grad_h_out: the gradient of its h_out."""
    args, (T, B, F, S), (cfg, kept, _, ws) = _scan_args(x, dt, A, Bm, Cm, D, dt_bias, softplus, h_in, lengths)
    x = args[0]
    if saved is None:
        raise ValueError("saved must be what scan_forward(train=True) returned for these arguments")
    saved = _dense("saved", saved, x, (kept,), torch.uint8)
    gy = _data("grad_y", grad_y, x, (T, B, F))
    g_out = _dense("grad_h_out", grad_h_out, x, (B, F, S))
    empty = not (T and B and F)
    gx, gdt, gB, gC = torch.empty_like(x), torch.empty_like(x), torch.empty_like(args[3]), torch.empty_like(args[4])
    gA, gD, gbias = _params(A, empty), _params(D, empty), _params(dt_bias, empty)
    gh = None if h_in is None else torch.empty_like(h_in)
    if empty:
        gB.zero_(), gC.zero_()
        _hand_over(gh, grad_h_out)
    else:
        native.snn_scan_backward(cfg, T, B, F, *args, saved, gy, g_out, gx, gdt, gA, gB, gC, gD, gbias, gh,
                                 _bytes(ws, x))
    return gx, gdt, gA, gB, gC, gD, gbias, gh


# ---------------------------------------------------------------------------------------

def _norm_args(y, r, z, w_post, scale, w_pre, eps, lengths):
    T, B, F = _shape(y)
    y = _rows(y)
    r = None if r is None else _data("r", r, y, (T, B, F))
    z = None if z is None else _data("z", z, y, (T, B, F))
    args = (y, z, r, _dense("w_post", w_post, y, (F,)), _dense("scale", scale, y, (F,)),
            _dense("w_pre", w_pre, y, (F,)), _dense("lengths", lengths, y, (B,), torch.int32))
    return args, (T, B, F), _norm_plan(IO_OF[y.dtype], eps, T, B, F)


@_on_stream
def norm_forward(y, r=None, z=None, w_post=None, scale=None, w_pre=None, *, eps=1e-5, lengths=None, train=False):
    """The end of a block and the start of the next over the last axis of y[T, B, F]:
    r_new = r + scale * norm(y * silu(z)) and u = norm(r_new), root-mean-square norms with the
    weights w_post and w_pre.  Without z, w_post, scale, r or w_pre that part is left out.
    Returns (r_new, u or None, rstd), rstd for norm_backward with train=True, else None."""
    args, (T, B, F), (cfg, _) = _norm_args(y, r, z, w_post, scale, w_pre, eps, lengths)
    r_new, u = torch.empty_like(args[0]), None if w_pre is None else torch.empty_like(args[0])
    rstd = torch.empty((2, T, B), dtype=torch.float32, device=y.device) if train else None
    if T and B and F:
        native.snn_norm_forward(cfg, T, B, F, *args, r_new, u, rstd)
    return r_new, u, rstd


@_on_stream
def norm_backward(y, r, z, w_post, scale, w_pre, rstd, grad_r_new, grad_u=None, *, eps=1e-5, lengths=None):
    """Gradients (y, r, z, w_post, scale, w_pre; None where the input is None) of norm_forward
    with the same arguments and its rstd.  grad_r_new or grad_u may be None (no gradient)."""
    args, (T, B, F), (cfg, ws) = _norm_args(y, r, z, w_post, scale, w_pre, eps, lengths)
    y = args[0]
    rstd = _dense("rstd", rstd, y, (2, T, B))
    g1 = None if grad_r_new is None else _data("grad_r_new", grad_r_new, y, (T, B, F))
    g2 = None if grad_u is None else _data("grad_u", grad_u, y, (T, B, F))
    empty = not (T and B and F)
    gy, gr, gz = (None if a is None else torch.empty_like(a) for a in (args[0], args[2], args[1]))
    gw = [_params(w, empty) for w in (w_post, scale, w_pre)]
    if not empty:
        native.snn_norm_backward(cfg, T, B, F, *args, rstd, g1, g2, gy, gz, gr, *gw, _bytes(ws, y))
    return gy, gr, gz, *gw
