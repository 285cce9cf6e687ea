"""Calls of the sequence operators that their documentation allows and that go wrong first: states
updated in place over many workgroups, launches of more threads than a grid takes,
tangents and traces, rows that overlap."""
import pytest
import torch

from tests.test_gpu_sequence import lengths_of, normal, scan_inputs

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


def of_sequences(rows, at):
    return [v[:, at].contiguous() for v in rows]


@pytest.mark.parametrize("T,B,F,S,G", [(2, 16384, 4096, 1, 4096), (64, 65536, 8, 64, 8)])
def test_launches_of_more_than_a_grids_threads(ops, T, B, F, S, G):
    """More workgroups, and more sums of partial results, than 2^32 threads of one grid axis: some
    sequences by themselves give the same bits."""
    x, step, gy = (normal(i, T, B, F, dtype=torch.bfloat16) for i in (1, 2, 3))
    Bm, Cm = (normal(i, T, B, G, S, dtype=torch.bfloat16) for i in (4, 5))
    A, D, bias = -torch.exp(normal(6, F, S, sd=0.7)), normal(7, F), normal(8, F, mean=-1.0)
    at = torch.tensor([0, 1, B // 2 - 1, B // 2, B - 2, B - 1], device="cuda")
    part = of_sequences((x, step, Bm, Cm, gy), at)

    def run(x, step, Bm, Cm, gy):
        y, saved = ops.scan_forward(x, step, A, Bm, Cm, D, bias, train=True)
        g = ops.scan_backward(x, step, A, Bm, Cm, D, bias, saved, gy)
        return [y, g[0], g[1], g[3], g[4]], [g[2], g[5], g[6]]
    rows, params = run(x, step, Bm, Cm, gy)
    for v, w in zip(of_sequences(rows, at), run(*part)[0]):
        assert torch.equal(v, w)
    assert all(torch.isfinite(v).all() for v in params)


def test_tokens_of_more_than_a_grids_threads(ops):
    """One step of 2^30 features of 64 states, 16 lanes each for 4 sequences."""
    B, F, S = 16384, 65536, 64
    x = normal(1, 1, B, F, dtype=torch.bfloat16)
    Bm, Cm = (normal(i, 1, B, 1, S, dtype=torch.bfloat16) for i in (2, 3))
    A = -torch.exp(normal(4, F, S, sd=0.7))
    y, _ = ops.scan_forward(x, x, A, Bm, Cm)
    at = torch.tensor([0, 1, B // 2 - 1, B // 2, B - 2, B - 1], device="cuda")
    part = of_sequences((x, Bm, Cm), at)
    assert torch.equal(y[:, at], ops.scan_forward(part[0], part[0], A, *part[1:])[0])


def test_tangents_are_refused(ops):
    """Forward-mode derivatives have no rule here: a tangent on any input raises an error instead of
    coming out as none, with gradients wanted and without."""
    import torch.autograd.forward_ad as fw

    from paper_2408_00280_amd import autograd
    x, step, A, Bm, Cm, D, *_ = scan_inputs("f32", 5, 2, 66, 4, 1, "D")
    w = normal(9, 66, 4)
    calls = {"conv x": (autograd.causal_conv, [x, w], 0), "conv weight": (autograd.causal_conv, [x, w], 1),
             "scan x": (autograd.selective_scan, [x, step, A, Bm, Cm], 0),
             "scan C": (autograd.selective_scan, [x, step, A, Bm, Cm], 4),
             "scan D": (autograd.selective_scan, [x, step, A, Bm, Cm, D], 5),
             "norm y": (autograd.block_norm, [x, step], 0), "norm r": (autograd.block_norm, [x, step], 1)}
    for name, (fn, args, at) in calls.items():
        with fw.dual_level():
            dual = [fw.make_dual(v, torch.ones_like(v)) if i == at else v for i, v in enumerate(args)]
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(RuntimeError, match="jvp"):
                    fn(*dual)
                    raise AssertionError(f"{name}: the tangent was dropped")
        fn(*args)


def test_traces_are_refused(ops):
    """A tracer would keep the outputs' allocation and none of the work."""
    from paper_2408_00280_amd import autograd
    x, step, A, Bm, Cm, *_ = scan_inputs("f32", 5, 2, 66, 4, 1, "")
    w = normal(9, 66, 4)
    for fn in (lambda v: autograd.causal_conv(v, w), lambda v: autograd.selective_scan(v, step, A, Bm, Cm),
               lambda v: autograd.block_norm(v)[0], lambda v: ops.conv_forward(v, w), lambda v: ops.norm_forward(v)[0],
               lambda v: ops.scan_forward(v, step, A, Bm, Cm)[0]):
        for grad in (False, True):
            with pytest.raises(RuntimeError, match="trace"):
                torch.jit.trace(fn, x.clone().requires_grad_(grad), check_trace=False)
                raise AssertionError("was traced")


@pytest.mark.parametrize("steps", [(1, 40), (40, 1), (2, 40)])
def test_windows_that_overlap(ops, steps):
    """Rows that share elements with the next, a step of 1 apart: the same as their copies."""
    T, B, F, S, W = 6, 3, 8, 4, 4
    room = normal(1, 1000)
    x = room.as_strided((T, B, F), (*steps, 1))
    bc = room[200:].as_strided((T, B, 2, S), (*steps, S, 1))
    A, w, one, gy = -positive_rates(F, S), normal(3, F, W), normal(4, F), normal(5, T, B, F)

    def run(x, bc):
        y, saved = ops.scan_forward(x, x, A, bc, bc, train=True)
        r, u, rstd = ops.norm_forward(x, x, x, one, one, one, train=True)
        return [y, *ops.scan_backward(x, x, A, bc, bc, None, None, saved, gy)[:5], ops.conv_forward(x, w),
                *ops.conv_backward(x, w, None, gy)[:2], r, u, *ops.norm_backward(x, x, x, one, one, one, rstd, gy, x)]
    for a, b in zip(run(x, bc), run(x.contiguous(), bc.contiguous())):
        assert torch.equal(a, b)


def positive_rates(F, S):
    return normal(2, F, S).abs() + 0.1


def test_tensors_dropped_while_another_stream_uses_them(ops):
    """Inputs dropped behind a call on another stream, and outputs dropped behind their use on this
    one, keep their memory until the other side has come to it."""
    T, B, F = 64, 8, 4100
    w, stream = normal(2, F, 4), torch.cuda.Stream()
    x = normal(1, T, B, F)
    want = ops.conv_forward(x, w)
    ref = want.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)                       # some 10 ms
    y = ops.conv_forward(x, w, stream=stream)
    at = x.data_ptr()
    del x
    others = [torch.zeros(T, B, F, device="cuda") for _ in range(3)]
    assert all(v.data_ptr() != at for v in others)
    torch.cuda.synchronize()
    assert torch.equal(y, ref)
    torch.cuda._sleep(20_000_000)
    kept, at = y + 1, y.data_ptr()
    del y
    with torch.cuda.stream(stream):
        others = [torch.zeros(T, B, F, device="cuda") for _ in range(3)]
    assert all(v.data_ptr() != at for v in others)
    torch.cuda.synchronize()
    assert torch.equal(kept, ref + 1)
