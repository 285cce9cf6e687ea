"""Calls of the sequence operators that their documentation allows and that go wrong first: states
updated in place over many workgroups."""
import pytest
import torch

from tests.test_gpu_sequence import lengths_of, scan_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2408_00280_amd import sequence
    return sequence


@pytest.mark.parametrize("ragged", [None, "ragged"])
@pytest.mark.parametrize("T,B,F,S,io", [(442, 3, 2928, 47, "bf16"), (2048, 2, 4096, 16, "bf16"), (700, 3, 4100, 4, "f32"),
                                        (4096, 2, 70, 16, "f32"), (100, 3, 70, 16, "f32")])
def test_scan_states_in_place(ops, T, B, F, S, io, ragged):
    """A state updated in place gives the outputs and the state of separate ones, bit for bit: over
    segments of the time axis that no CU holds all of, over more segments than a workgroup walks
    itself, and over one."""
    x, step, A, Bm, Cm, D, bias, h, *_ = scan_inputs(io, T, B, F, S, 1, "D bias h")
    ln = lengths_of(ragged, T, B)
    out = torch.empty_like(h)
    y, _ = ops.scan_forward(x, step, A, Bm, Cm, D, bias, h_in=h, h_out=out, lengths=ln)
    for _ in range(3):
        state = h.clone()
        got, _ = ops.scan_forward(x, step, A, Bm, Cm, D, bias, h_in=state, h_out=state, lengths=ln)
        assert torch.equal(got, y) and torch.equal(state, out)
