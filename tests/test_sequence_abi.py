"""The C ABI of the sequence operators: exports, sizes, and what it refuses.  CPU only: every
call is rejected, or is empty, before any HIP call, so that the addresses are never read."""
import ctypes
import os
import re

import pytest

from paper_2408_00280_amd import native as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "snn_seq.h")
P = 0x10000
SHAPE = (6, 3, 20)


def s(data=P, t=60, b=20):
    return N.snn_seq(data, t, b)


CONV, SCAN, NORM = N.snn_conv_cfg(1, 4, 1), N.snn_scan_cfg(1, 8, 2, 1), N.snn_norm_cfg(1, 1e-5)

# Arguments of each call by name, valid but for their addresses.
CALLS = {
    "snn_conv_forward": dict(cfg=CONV, x=s(), weight=P, bias=P, state_in=P, lengths=P, y=s(), state_out=P),
    "snn_conv_backward": dict(cfg=CONV, x=s(), weight=P, bias=P, state_in=P, lengths=P, grad_y=s(), grad_state_out=P,
                              grad_x=s(), grad_weight=P, grad_bias=P, grad_state_in=P, workspace=P),
    "snn_scan_forward": dict(cfg=SCAN, x=s(), dt=s(), A=P, Bm=s(), Cm=s(), D=P, dt_bias=P, h_in=P, lengths=P, y=s(),
                             h_out=P, saved=P, workspace=P),
    "snn_scan_backward": dict(cfg=SCAN, x=s(), dt=s(), A=P, Bm=s(), Cm=s(), D=P, dt_bias=P, h_in=P, lengths=P, saved=P,
                              grad_y=s(), grad_h_out=P, grad_x=s(), grad_dt=s(), grad_A=P, grad_Bm=s(), grad_Cm=s(),
                              grad_D=P, grad_dt_bias=P, grad_h_in=P, workspace=P),
    "snn_norm_forward": dict(cfg=NORM, y=s(), z=s(), r=s(), w_post=P, scale=P, w_pre=P, lengths=P, r_new=s(), u=s(),
                             rstd=P),
    "snn_norm_backward": dict(cfg=NORM, y=s(), z=s(), r=s(), w_post=P, scale=P, w_pre=P, lengths=P, rstd=P,
                              grad_r_new=s(), grad_u=s(), grad_y=s(), grad_z=s(), grad_r=s(), grad_w_post=P,
                              grad_scale=P, grad_w_pre=P, workspace=P),
}
OPTIONAL = {"bias", "state_in", "state_out", "lengths", "grad_state_out", "grad_bias", "grad_state_in", "D", "dt_bias",
            "h_in", "h_out", "grad_h_out", "grad_D", "grad_dt_bias", "grad_h_in", "z", "r", "w_post", "scale",
            "grad_r_new", "grad_u", "w_pre"}


def call(name, shape=SHAPE, **change):
    a = {**CALLS[name], **change}
    cfg = a.pop("cfg")
    return getattr(N.lib, name)(cfg, *shape, *a.values(), None)


def refused(name, status, **change):
    assert call(name, **change) == status, (name, change)


def test_exports():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(snn_\w+)\s*\(", text)))
    assert declared == sorted(N.SEQ_EXPORTS)
    out = os.popen(f"nm -D --defined-only {N.LIB_PATH}").read()
    for name in declared:
        assert re.search(rf"\bT {name}\b", out), name


@pytest.mark.parametrize("compiler,flags,ext", [("gcc", ["-std=c99"], "c"), ("g++", ["-std=c++11"], "cc")])
def test_header_is_plain_c_and_cxx(tmp_path, compiler, flags, ext):
    import shutil
    import subprocess
    if shutil.which(compiler) is None:
        pytest.skip(f"{compiler} not available")
    src = tmp_path / f"use.{ext}"
    src.write_text('#include "snn_seq.h"\nint probe(const snn_norm_cfg *c, size_t *b) '
                   "{ return snn_norm_workspace_bytes(c, 4, 2, 64, b); }\n")
    r = subprocess.run([compiler, *flags, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-I",
                        os.path.join(ROOT, "include"), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("name", list(CALLS))
def test_null_arguments(name):
    assert call(name, cfg=None) == -1
    for k in CALLS[name]:
        if k not in OPTIONAL and k != "cfg":
            if name == "snn_scan_forward" and k in ("saved", "workspace") or name == "snn_norm_forward" and k == "rstd":
                continue         # not needed, or not for few steps
            if k == "saved":     # needed as soon as there are two blocks of steps
                assert call(name, (40, 3, 20), **{k: None}) == -1
                continue
            refused(name, -1, **{k: None})
            if isinstance(CALLS[name][k], N.snn_seq):
                refused(name, -1, **{k: s(None)})


@pytest.mark.parametrize("name", list(CALLS))
def test_misaligned_arguments(name):
    for k, v in CALLS[name].items():
        if isinstance(v, N.snn_seq):
            refused(name, -4, **{k: s(P + 1)})
        elif v == P:
            refused(name, -4, **{k: P + (8 if k == "workspace" else 1)})


@pytest.mark.parametrize("name", list(CALLS))
def test_shapes_and_steps(name):
    for shape in ((-1, 3, 20), (6, -1, 20), (6, 3, -1), (2 ** 31, 3, 20), (6, 2 ** 24 + 2, 20), (6, 3, 2 ** 24 + 2),
                  (2 ** 20, 2 ** 12, 20), (2 ** 20, 2 ** 10, 2 ** 20)):
        assert call(name, shape) == -2, shape
    for k, v in CALLS[name].items():
        if not isinstance(v, N.snn_seq):
            continue
        refused(name, -2, **{k: s(t=-1)})
        refused(name, -2, **{k: s(b=-20)})
        refused(name, -2, **{k: s(t=2 ** 44)})
        output = (k in ("u", "r_new") or k == "y" and "norm" not in name
                  or k.startswith("grad_") and k not in ("grad_y", "grad_r_new", "grad_u")
                  or k == "grad_y" and "norm" in name)
        if output:       # rows on top of each other
            for t, b in ((0, 20), (60, 0), (20, 20), (59, 20), (30, 30), (1, 6)):
                if k in ("grad_Bm", "grad_Cm") and (t, b) == (59, 20):
                    continue        # rows of 16 values lie apart
                refused(name, -2, **{k: s(t=t, b=b)})


@pytest.mark.parametrize("name", list(CALLS))
def test_configurations(name):
    if "conv" in name:
        bad = [(2, 4, 1), (-1, 4, 1), (1, 0, 1), (1, 9, 1), (1, 4, 2), (1, 4, -1)]
        cfgs = [N.snn_conv_cfg(*v) for v in bad]
    elif "scan" in name:
        bad = [(2, 8, 2, 1), (1, 0, 2, 1), (1, 65, 2, 1), (1, 8, 0, 1), (1, 8, -2, 1), (1, 8, 2, 2)]
        cfgs = [N.snn_scan_cfg(*v) for v in bad]
        assert call(name, cfg=N.snn_scan_cfg(1, 8, 3, 1)) == -2      # 3 does not divide 20
    else:
        inf, nan = float("inf"), float("nan")
        cfgs = [N.snn_norm_cfg(*v) for v in ((2, 1e-5), (1, 0.0), (1, -1.0), (1, inf), (1, nan))]
    for cfg in cfgs:
        assert call(name, cfg=cfg) == -3


@pytest.mark.parametrize("name", list(CALLS))
def test_empty_problems(name):
    nothing = {k: None for k in CALLS[name] if k != "cfg"}
    for shape in ((0, 3, 20), (6, 0, 20), (6, 3, 0)):
        assert call(name, shape, **nothing) == 0


def test_sizes():
    n = ctypes.c_size_t(7)
    two = ctypes.c_size_t(7)
    for f, cfg in ((N.lib.snn_conv_workspace_bytes, CONV), (N.lib.snn_scan_saved_bytes, SCAN),
                   (N.lib.snn_norm_workspace_bytes, NORM)):
        assert f(None, *SHAPE, n) == -1 and f(cfg, *SHAPE, None) == -1 and f(cfg, -1, 3, 20, n) == -2
        assert f(cfg, 0, 3, 20, n) == 0 and n.value == 0
    assert N.lib.snn_scan_workspace_bytes(SCAN, *SHAPE, n, None) == -1
    assert N.lib.snn_scan_workspace_bytes(SCAN, *SHAPE, None, n) == -1
    assert N.lib.snn_scan_workspace_bytes(SCAN, 0, 3, 20, n, two) == 0 and n.value == two.value == 0
    # one state per feature and sequence is kept at each block's start but the first's
    assert N.snn_scan_saved_bytes(SCAN, 1, 3, 20) == 0
    per = 3 * 20 * 8 * 4
    sizes = [N.snn_scan_saved_bytes(SCAN, T, 3, 20) for T in range(1, 200)]
    assert sizes == sorted(sizes) and all(v % per == 0 for v in sizes)
