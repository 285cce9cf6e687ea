"""The LIF layers' binding without the sequence operators' extension module: it needs libsnnlif.so
only.  On the CPU, in a process of its own."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
sys.modules["paper_2408_00280_amd._sequence"] = None      # as if it were not built, or did not load
import torch
from paper_2408_00280_amd import autograd, layer, native
lif = autograd.LIFLayer(0.5, 1.0)
stack = autograd.LIFStack(torch.ones(2, 4), decay=0.5, v_th=1.0)
assert native.snn_lif_saved_bytes(layer.LifConfig(0.5, 1.0).c(), 100, 64) > 0
x = torch.zeros(2, 1, 4)
scan = autograd.SelectiveScan(4, 2)
for call in (lambda: autograd.causal_conv(x, x[0].t()), lambda: autograd.block_norm(x), lambda: autograd.CausalConv(4)(x),
             lambda: scan(x, x, x[..., None, :2], x[..., None, :2]), lambda: scan.step(x[0], x[0], x[0], x[0], x)):
    try:
        call()
    except ImportError as e:
        assert "not built" in str(e), e
    else:
        raise AssertionError("ran without its module")
print("done")
"""


def test_lif_layers_without_the_sequence_module():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stdout + r.stderr
