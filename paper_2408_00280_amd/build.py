"""Compile the HIP library libsnnlif.so for gfx950 (in-tree, next to this file).

The kernel variants are split over several translation units (one per forward I/O dtype and
spike format, one per backward I/O dtype, the same for the gain-fed layer and for the
stack fused across depth, the gain kernels, the serial baseline, the sequence operators, the
C ABI) that compile in parallel and link into one shared library.  Beside it stands the
extension module _sequence.so, host code that gives the sequence operators torch's tensors.
"""
from __future__ import annotations

import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
CSRC_SEQ = os.path.join(HERE, "csrc_seq")   # the sequence operators (include/snn_seq.h)
OUT = os.path.join(HERE, "libsnnlif.so")
SEQ_OUT = os.path.join(HERE, "_sequence.so")
OBJ_DIR = os.path.join(HERE, "_build")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # the membrane update must be one IEEE multiply and one IEEE add, never a fused FMA
    "-ffp-contract=off",
    # no packed-fp32 VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]

# (object name, source, defines)
UNITS = (
    [(f"fwd_io{io}_spk{spk}", "lif_forward.hip", [f"-DSNNLIF_IO={io}", f"-DSNNLIF_SPK={spk}"])
     for io in (0, 1) for spk in (0, 1, 2)]
    + [(f"fwdgain_io{io}_spk{spk}", "lif_forward.hip", [f"-DSNNLIF_IO={io}", f"-DSNNLIF_SPK={spk}", "-DSNNLIF_GAIN=1"])
       for io in (0, 1) for spk in (0, 1, 2)]
    + [(f"bwd_io{io}", "lif_backward.hip", [f"-DSNNLIF_IO={io}"]) for io in (0, 1)]
    + [(f"bwdgain_io{io}_spk{spk}", "lif_backward.hip", [f"-DSNNLIF_IO={io}", f"-DSNNLIF_SPK={spk}", "-DSNNLIF_GAIN=1"])
       for io in (0, 1) for spk in (0, 1, 2)]
    + [(f"stackf_io{io}_spk{spk}", "lif_stack.hip", [f"-DSNNLIF_IO={io}", f"-DSNNLIF_SPK={spk}"])
       for io in (0, 1) for spk in (0, 1, 2)]
    + [(f"stackb_io{io}", "lif_stack.hip", [f"-DSNNLIF_IO={io}", "-DSNNLIF_STACK_BWD=1"]) for io in (0, 1)]
    + [("glue", "lif_glue.hip", []), ("serial", "lif_serial.hip", []), ("api", "snn_lif_api.hip", [])]
    + [(name, os.path.join(CSRC_SEQ, f"{name}.hip"), [])
       for name in ("seq_conv", "seq_scan_forward", "seq_scan_backward", "seq_scan_split", "seq_norm", "snn_seq_api")]
)


def _compile(unit, extra):
    name, src, defs = unit
    obj = os.path.join(OBJ_DIR, name + ".o")
    cmd = ["hipcc", *HIPCC_FLAGS, *extra, *defs, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", CSRC_SEQ,
           "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "'-packed-fp32-ops' is not a recognized feature for this target (ignoring feature)"
    msgs = "\n".join(ln for ln in (r.stdout + r.stderr).splitlines() if noise not in ln)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {name}:\n{msgs}")
    return obj


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed:\n{r.stdout}{r.stderr}")


def _compile_torch():
    from torch.utils import cpp_extension

    obj = os.path.join(OBJ_DIR, "seq_torch.o")
    system = [*cpp_extension.include_paths("cuda"), sysconfig.get_paths()["include"]]
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-I",
          os.path.join(ROOT, "include"), *(f for p in system for f in ("-isystem", p)),
          "-c", os.path.join(CSRC_SEQ, "seq_torch.cpp"), "-o", obj])
    return obj


def _link_torch(obj):
    from torch.utils import cpp_extension

    dirs = [f for p in cpp_extension.library_paths("cuda") for f in ("-L", p)]
    _run(["g++", "-shared", obj, "-o", SEQ_OUT + ".tmp", "-L", HERE, "-l:" + os.path.basename(OUT), "-Wl,-rpath,$ORIGIN",
          *dirs, "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python"])
    os.replace(SEQ_OUT + ".tmp", SEQ_OUT)


def build(out: str = OUT, extra=(), jobs: int | None = None) -> str:
    """Always recompiles every translation unit, then links.  The extension module goes with the
    library in its own place."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    jobs = jobs or min(len(UNITS), os.cpu_count() or 4)
    with ThreadPoolExecutor(max_workers=jobs) as pool:
        torch_obj = pool.submit(_compile_torch) if out == OUT else None
        objs = list(pool.map(lambda u: _compile(u, list(extra)), UNITS))
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", out + ".tmp"], check=True)
    os.replace(out + ".tmp", out)
    if torch_obj is not None:
        _link_torch(torch_obj.result())
    return out


if __name__ == "__main__":
    print(build())
