"""Thin ctypes binding over the C ABI in include/snn_lif.h and include/snn_seq.h (libsnnlif.so).

Argument marshalling only: every step of the work runs in the HIP kernels under
``csrc/``.  Functions keep the C names; tensor arguments may be torch
tensors (their ``data_ptr()`` is passed) or raw device addresses (int), and
``stream`` may be a ``torch.cuda.Stream``, a raw hipStream_t (int) or None for
torch's current stream.  A non-OK status raises :class:`SnnError`.

If the shared library is missing this module raises at import time: there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch  # loads the HIP runtime the library binds to (same soname)

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsnnlif.so")

SNN_OK = 0
SNN_RESET_HARD, SNN_RESET_SOFT = 0, 1
SNN_IO_F32, SNN_IO_BF16 = 0, 1
SNN_SPK_U8, SNN_SPK_BITS, SNN_SPK_IO = 0, 1, 2

STATUS_NAMES = {0: "SNN_OK", -1: "SNN_E_NULL", -2: "SNN_E_SHAPE", -3: "SNN_E_PARAM",
                -4: "SNN_E_ALIGN", -5: "SNN_E_UNSUPPORTED", -6: "SNN_E_LAUNCH"}

# Every symbol the header declares; a test checks the library exports all of them.
EXPORTS = ("snn_spike_row_bytes", "snn_lif_saved_bytes", "snn_lif_forward", "snn_lif_backward",
           "snn_lif_forward_seg", "snn_lif_backward_seg",
           "snn_gain_spikes_forward", "snn_gain_grad_backward", "snn_lif_forward_gain",
           "snn_lif_backward_gain", "snn_lif_stack_saved_bytes", "snn_lif_stack_forward",
           "snn_lif_stack_backward", "snn_lif_serial_forward_step",
           "snn_lif_serial_backward_step", "snn_status_str")

SNN_ACT_NONE, SNN_ACT_SILU = 0, 1

# The same for include/snn_seq.h.
SEQ_EXPORTS = ("snn_conv_forward", "snn_conv_workspace_bytes", "snn_conv_backward", "snn_scan_saved_bytes",
               "snn_scan_workspace_bytes", "snn_scan_forward", "snn_scan_backward", "snn_norm_forward",
               "snn_norm_workspace_bytes", "snn_norm_backward")


class SnnError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn}: {STATUS_NAMES.get(status, status)} ({text})")
        self.status = status


class snn_lif_cfg(ctypes.Structure):
    _fields_ = [("decay", ctypes.c_float), ("v_th", ctypes.c_float), ("v_reset", ctypes.c_float),
                ("alpha", ctypes.c_float), ("reset", ctypes.c_int32), ("io", ctypes.c_int32),
                ("spk", ctypes.c_int32)]


class snn_seq(ctypes.Structure):
    """A [T][B][X] tensor: address, elements between steps, elements between sequences."""
    _fields_ = [("data", ctypes.c_void_p), ("t", ctypes.c_int64), ("b", ctypes.c_int64)]


class snn_conv_cfg(ctypes.Structure):
    _fields_ = [("io", ctypes.c_int32), ("width", ctypes.c_int32), ("act", ctypes.c_int32)]


class snn_scan_cfg(ctypes.Structure):
    _fields_ = [("io", ctypes.c_int32), ("states", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("softplus", ctypes.c_int32)]


class snn_norm_cfg(ctypes.Structure):
    _fields_ = [("io", ctypes.c_int32), ("eps", ctypes.c_float)]


def make_cfg(decay: float, v_th: float, v_reset: float = 0.0, alpha: float = 4.0, reset="hard",
             io="f32", spk="u8") -> snn_lif_cfg:
    """Build a cfg from Python values ("hard"/"soft", "f32"/"bf16", "u8"/"bits"/"io" or the ints)."""
    r = {"hard": SNN_RESET_HARD, "soft": SNN_RESET_SOFT}.get(reset, reset)
    d = {"f32": SNN_IO_F32, "bf16": SNN_IO_BF16}.get(io, io)
    s = {"u8": SNN_SPK_U8, "bits": SNN_SPK_BITS, "io": SNN_SPK_IO}.get(spk, spk)
    return snn_lif_cfg(decay, v_th, v_reset, alpha, r, d, s)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(the LIF path has no non-HIP fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    C, i64, vp, st = ctypes.POINTER(snn_lif_cfg), ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    szp = ctypes.POINTER(ctypes.c_size_t)
    sig = {
        "snn_spike_row_bytes": [C, i64, szp],
        "snn_lif_saved_bytes": [C, i64, i64, szp],
        "snn_lif_forward": [C, i64, i64, vp, vp, vp, vp, vp],
        "snn_lif_backward": [C, i64, i64, vp, vp, vp, vp, vp],
        "snn_lif_forward_seg": [C, i64, i64, vp, vp, vp, vp, vp, vp, vp],
        "snn_lif_backward_seg": [C, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp],
        "snn_gain_spikes_forward": [C, i64, i64, i64, vp, vp, vp, vp],
        "snn_gain_grad_backward": [C, i64, i64, i64, vp, vp, vp, vp],
        "snn_lif_forward_gain": [C, i64, i64, i64, vp, vp, vp, vp, vp, vp],
        "snn_lif_backward_gain": [C, i64, i64, i64, vp, vp, vp, vp, vp, vp],
        "snn_lif_stack_saved_bytes": [C, ctypes.c_int32, i64, i64, szp],
        "snn_lif_stack_forward": [C, ctypes.c_int32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp],
        "snn_lif_stack_backward": [C, ctypes.c_int32, i64, i64, i64, vp, vp, vp, vp, vp, vp],
        "snn_lif_serial_forward_step": [C, i64, vp, vp, vp, vp, vp],
        "snn_lif_serial_backward_step": [C, i64, vp, vp, vp, vp, vp, vp],
    }
    q, cc, sc, nc = (ctypes.POINTER(t) for t in (snn_seq, snn_conv_cfg, snn_scan_cfg, snn_norm_cfg))
    shape = [i64, i64, i64]
    scan_in = [sc, *shape, q, q, vp, q, q, vp, vp, vp, vp]
    norm_in = [nc, *shape, q, q, q, vp, vp, vp, vp]
    sig.update({
        "snn_conv_forward": [cc, *shape, q, vp, vp, vp, vp, q, vp, vp],
        "snn_conv_workspace_bytes": [cc, *shape, szp],
        "snn_conv_backward": [cc, *shape, q, vp, vp, vp, vp, q, vp, q, vp, vp, vp, vp, vp],
        "snn_scan_saved_bytes": [sc, *shape, szp],
        "snn_scan_workspace_bytes": [sc, *shape, szp, szp],
        "snn_scan_forward": [*scan_in, q, vp, vp, vp, vp],
        "snn_scan_backward": [*scan_in, vp, q, vp, q, q, vp, q, q, vp, vp, vp, vp, vp],
        "snn_norm_forward": [*norm_in, q, q, vp, vp],
        "snn_norm_workspace_bytes": [nc, *shape, szp],
        "snn_norm_backward": [*norm_in, vp, q, q, q, q, q, vp, vp, vp, vp, vp],
    })
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = st
    lib.snn_status_str.argtypes = [st]
    lib.snn_status_str.restype = ctypes.c_char_p
    return lib


lib = _load()


def _ptr(a):
    if a is None:
        return None
    if isinstance(a, torch.Tensor):
        if not a.is_contiguous() and a.numel():
            raise ValueError("tensor arguments must be contiguous")
        return a.data_ptr() or None
    return int(a)


def _stream(s):
    if s is None:
        # the handle torch.cuda.current_stream() wraps, without making the wrapper: 0.5 instead
        # of 14 us per call in a training loop, whose backward runs on a thread of its own
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, torch.cuda.Stream):
        return s.cuda_stream
    return int(s)


def _check(fn: str, status: int):
    if status != SNN_OK:
        raise SnnError(fn, status, lib.snn_status_str(status).decode())


def snn_status_str(status: int) -> str:
    return lib.snn_status_str(status).decode()


def snn_spike_row_bytes(cfg: snn_lif_cfg, N: int) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_spike_row_bytes", lib.snn_spike_row_bytes(ctypes.byref(cfg), N, ctypes.byref(out)))
    return out.value


def snn_lif_saved_bytes(cfg: snn_lif_cfg, T: int, N: int) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_lif_saved_bytes", lib.snn_lif_saved_bytes(ctypes.byref(cfg), T, N, ctypes.byref(out)))
    return out.value


def snn_lif_forward(cfg, T, N, x, spikes, saved, v_out=None, stream=None):
    _check("snn_lif_forward", lib.snn_lif_forward(ctypes.byref(cfg), T, N, _ptr(x), _ptr(spikes),
                                                  _ptr(saved), _ptr(v_out), _stream(stream)))


def snn_lif_backward(cfg, T, N, x, saved, grad_s, grad_x, stream=None):
    _check("snn_lif_backward", lib.snn_lif_backward(ctypes.byref(cfg), T, N, _ptr(x), _ptr(saved),
                                                    _ptr(grad_s), _ptr(grad_x), _stream(stream)))


def snn_lif_forward_seg(cfg, T, N, x, v_in, spikes, saved, v_last=None, v_out=None, stream=None):
    _check("snn_lif_forward_seg", lib.snn_lif_forward_seg(
        ctypes.byref(cfg), T, N, _ptr(x), _ptr(v_in), _ptr(spikes), _ptr(saved), _ptr(v_last), _ptr(v_out),
        _stream(stream)))


def snn_lif_backward_seg(cfg, T, N, x, v_in, saved, grad_s, g_in, grad_x, g_out=None, stream=None):
    _check("snn_lif_backward_seg", lib.snn_lif_backward_seg(
        ctypes.byref(cfg), T, N, _ptr(x), _ptr(v_in), _ptr(saved), _ptr(grad_s), _ptr(g_in), _ptr(grad_x),
        _ptr(g_out), _stream(stream)))


def snn_gain_spikes_forward(cfg, T, B, F, spikes, gain, x_next, stream=None):
    _check("snn_gain_spikes_forward", lib.snn_gain_spikes_forward(
        ctypes.byref(cfg), T, B, F, _ptr(spikes), _ptr(gain), _ptr(x_next), _stream(stream)))


def snn_gain_grad_backward(cfg, T, B, F, grad_x_next, gain, grad_s, stream=None):
    _check("snn_gain_grad_backward", lib.snn_gain_grad_backward(
        ctypes.byref(cfg), T, B, F, _ptr(grad_x_next), _ptr(gain), _ptr(grad_s), _stream(stream)))


def snn_lif_forward_gain(cfg, T, B, F, spikes_in, gain, spikes, saved, v_out=None, stream=None):
    _check("snn_lif_forward_gain", lib.snn_lif_forward_gain(
        ctypes.byref(cfg), T, B, F, _ptr(spikes_in), _ptr(gain), _ptr(spikes), _ptr(saved), _ptr(v_out),
        _stream(stream)))


def snn_lif_backward_gain(cfg, T, B, F, spikes_in, gain, saved, grad_s, grad_s_in, stream=None):
    _check("snn_lif_backward_gain", lib.snn_lif_backward_gain(
        ctypes.byref(cfg), T, B, F, _ptr(spikes_in), _ptr(gain), _ptr(saved), _ptr(grad_s), _ptr(grad_s_in),
        _stream(stream)))


def snn_lif_stack_saved_bytes(cfg: snn_lif_cfg, L: int, T: int, N: int) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_lif_stack_saved_bytes", lib.snn_lif_stack_saved_bytes(ctypes.byref(cfg), L, T, N, ctypes.byref(out)))
    return out.value


def snn_lif_stack_forward(cfg, L, T, B, F, x, gains, spikes, hidden_spikes, saved, v_out=None, stream=None):
    _check("snn_lif_stack_forward", lib.snn_lif_stack_forward(
        ctypes.byref(cfg), L, T, B, F, _ptr(x), _ptr(gains), _ptr(spikes), _ptr(hidden_spikes), _ptr(saved),
        _ptr(v_out), _stream(stream)))


def snn_lif_stack_backward(cfg, L, T, B, F, x, gains, saved, grad_s, grad_x, stream=None):
    _check("snn_lif_stack_backward", lib.snn_lif_stack_backward(
        ctypes.byref(cfg), L, T, B, F, _ptr(x), _ptr(gains), _ptr(saved), _ptr(grad_s), _ptr(grad_x),
        _stream(stream)))


def snn_lif_serial_forward_step(cfg, N, x_t, v_prev, v_t, spikes_t, stream=None):
    _check("snn_lif_serial_forward_step", lib.snn_lif_serial_forward_step(
        ctypes.byref(cfg), N, _ptr(x_t), _ptr(v_prev), _ptr(v_t), _ptr(spikes_t), _stream(stream)))


def snn_lif_serial_backward_step(cfg, N, v_t, grad_s_t, g_next, grad_x_t, g_out=None, stream=None):
    _check("snn_lif_serial_backward_step", lib.snn_lif_serial_backward_step(
        ctypes.byref(cfg), N, _ptr(v_t), _ptr(grad_s_t), _ptr(g_next), _ptr(grad_x_t), _ptr(g_out),
        _stream(stream)))


# include/snn_seq.h.  A [T][B][X] tensor goes in as a torch tensor (its last axis contiguous;
# further axes behind the second count as part of X) or as an snn_seq.

def seq(a):
    if a is None or isinstance(a, snn_seq):
        return a
    st = a.stride()
    return snn_seq(a.data_ptr() or None, st[0], st[1])


def snn_conv_forward(cfg, T, B, F, x, weight, bias, state_in, lengths, y, state_out, stream=None):
    _check("snn_conv_forward", lib.snn_conv_forward(cfg, T, B, F, seq(x), _ptr(weight), _ptr(bias), _ptr(state_in),
                                                    _ptr(lengths), seq(y), _ptr(state_out), _stream(stream)))


def snn_conv_workspace_bytes(cfg, T, B, F) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_conv_workspace_bytes", lib.snn_conv_workspace_bytes(cfg, T, B, F, ctypes.byref(out)))
    return out.value


def snn_conv_backward(cfg, T, B, F, x, weight, bias, state_in, lengths, grad_y, grad_state_out, grad_x, grad_weight,
                      grad_bias, grad_state_in, workspace, stream=None):
    _check("snn_conv_backward", lib.snn_conv_backward(
        cfg, T, B, F, seq(x), _ptr(weight), _ptr(bias), _ptr(state_in), _ptr(lengths), seq(grad_y),
        _ptr(grad_state_out), seq(grad_x), _ptr(grad_weight), _ptr(grad_bias), _ptr(grad_state_in), _ptr(workspace),
        _stream(stream)))


def snn_scan_saved_bytes(cfg, T, B, F) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_scan_saved_bytes", lib.snn_scan_saved_bytes(cfg, T, B, F, ctypes.byref(out)))
    return out.value


def snn_scan_workspace_bytes(cfg, T, B, F):
    """(forward's, backward's)."""
    fwd, bwd = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check("snn_scan_workspace_bytes",
           lib.snn_scan_workspace_bytes(cfg, T, B, F, ctypes.byref(fwd), ctypes.byref(bwd)))
    return fwd.value, bwd.value


def snn_scan_forward(cfg, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths, y, h_out, saved, workspace, stream=None):
    _check("snn_scan_forward", lib.snn_scan_forward(
        cfg, T, B, F, seq(x), seq(dt), _ptr(A), seq(Bm), seq(Cm), _ptr(D), _ptr(dt_bias), _ptr(h_in), _ptr(lengths),
        seq(y), _ptr(h_out), _ptr(saved), _ptr(workspace), _stream(stream)))


def snn_scan_backward(cfg, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths, saved, grad_y, grad_h_out, grad_x,
                      grad_dt, grad_A, grad_Bm, grad_Cm, grad_D, grad_dt_bias, grad_h_in, workspace, stream=None):
    _check("snn_scan_backward", lib.snn_scan_backward(
        cfg, T, B, F, seq(x), seq(dt), _ptr(A), seq(Bm), seq(Cm), _ptr(D), _ptr(dt_bias), _ptr(h_in), _ptr(lengths),
        _ptr(saved), seq(grad_y), _ptr(grad_h_out), seq(grad_x), seq(grad_dt), _ptr(grad_A), seq(grad_Bm),
        seq(grad_Cm), _ptr(grad_D), _ptr(grad_dt_bias), _ptr(grad_h_in), _ptr(workspace), _stream(stream)))


def snn_norm_forward(cfg, T, B, F, y, z, r, w_post, scale, w_pre, lengths, r_new, u, rstd, stream=None):
    _check("snn_norm_forward", lib.snn_norm_forward(
        cfg, T, B, F, seq(y), seq(z), seq(r), _ptr(w_post), _ptr(scale), _ptr(w_pre), _ptr(lengths), seq(r_new),
        seq(u), _ptr(rstd), _stream(stream)))


def snn_norm_workspace_bytes(cfg, T, B, F) -> int:
    out = ctypes.c_size_t(0)
    _check("snn_norm_workspace_bytes", lib.snn_norm_workspace_bytes(cfg, T, B, F, ctypes.byref(out)))
    return out.value


def snn_norm_backward(cfg, T, B, F, y, z, r, w_post, scale, w_pre, lengths, rstd, grad_r_new, grad_u, grad_y, grad_z,
                      grad_r, grad_w_post, grad_scale, grad_w_pre, workspace, stream=None):
    _check("snn_norm_backward", lib.snn_norm_backward(
        cfg, T, B, F, seq(y), seq(z), seq(r), _ptr(w_post), _ptr(scale), _ptr(w_pre), _ptr(lengths), _ptr(rstd),
        seq(grad_r_new), seq(grad_u), seq(grad_y), seq(grad_z), seq(grad_r), _ptr(grad_w_post), _ptr(grad_scale),
        _ptr(grad_w_pre), _ptr(workspace), _stream(stream)))
