"""Values at which the scan's sums and products go wrong first: states that grow, infinite inputs
beside lanes that have none, and what follows the last step of a sequence."""
import pytest
import torch

from tests import sequence_ref as R
from tests.test_gpu_sequence import NAMES, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2408_00280_amd import sequence
    return sequence


def positive(seed, *shape):
    return normal(seed, *shape).abs() + 0.1


@pytest.mark.parametrize("T,B,F,S", [(100, 2, 70, 16), (300, 2, 70, 16), (300, 3, 65, 3), (4096, 1, 20, 4)])
def test_states_that_grow(ops, T, B, F, S):
    """Rates above 0 whose growth over a segment of the time axis passes the type: states that are 0
    until the last steps, and gradients that are 0 but for the first, are finite all the same (in one
    segment, in some, and in more than a workgroup walks itself).  A step's growth e^x, x < 7.2, is
    off by 3 roundings of x and 2 of its own, under 24 and with the state's 3 near the 26 per step
    that R.scan_roundings counts over all T steps, of which at most 8 count here."""
    g = torch.Generator(device="cuda").manual_seed(1)
    A = 5 + 1.5 * torch.rand((F, S), device="cuda", generator=g)
    step = 0.9 + 0.2 * torch.rand((T, B, F), device="cuda", generator=g)
    x, gy, Bm, Cm = normal(2, T, B, F), normal(3, T, B, F), normal(4, T, B, 1, S), normal(5, T, B, 1, S)
    x[:T - 8] = 0.0
    gy[8:] = 0.0
    ref, mag = (R.scan(x, step, A, Bm, Cm, softplus=False, gy=gy, mag=m) for m in (False, True))
    h = torch.empty((B, F, S), device="cuda")
    y, saved = ops.scan_forward(x, step, A, Bm, Cm, softplus=False, h_out=h, train=True)
    got = ops.scan_backward(x, step, A, Bm, Cm, None, None, saved, gy, softplus=False)
    n = R.scan_roundings(T, B, F, S)
    for name, v in zip(("y", "h_out", *NAMES), (y, h, *got)):
        if v is not None:
            R.check(name, v, ref[name], mag[name], n)


@pytest.mark.parametrize("S", [3, 16, 33])
@pytest.mark.parametrize("T,n", [(9, 5), (150, 133), (150, 3)])
@pytest.mark.parametrize("where", ["x", "gh_out"])
def test_what_is_infinite_at_a_sequences_end(ops, where, T, n, S):
    """An infinite input of the last step, or an infinite gradient of the state behind it: the steps
    that only fill up a block or the batch add nothing to dL/dA.  Held to each sequence alone."""
    B, F = 2, 67
    x, dt, Bm, Cm, gy = (positive(i, *s) for i, s in enumerate(((T, B, F), (T, B, F), (T, B, 1, S), (T, B, 1, S), (T, B, F))))
    A, gh, h, ends = -positive(6, F, S), positive(7, B, F, S), positive(8, B, F, S), [n, T]
    for b in range(B):
        if where == "x":
            x[ends[b] - 1, b, F - 1] = float("inf")
        else:
            gh[b, F - 1, S - 1] = float("inf")
    ln = torch.tensor(ends, dtype=torch.int32, device="cuda")
    _, saved = ops.scan_forward(x, dt, A, Bm, Cm, h_in=h, lengths=ln, train=True)
    got = dict(zip(NAMES, ops.scan_backward(x, dt, A, Bm, Cm, None, None, saved, gy, h_in=h, lengths=ln, grad_h_out=gh)))
    alone = [R.scan(*(v[:m, b:b + 1] for v in (x, dt)), A, *(v[:m, b:b + 1] for v in (Bm, Cm)), h_in=h[b:b + 1],
                    gy=gy[:m, b:b + 1], gh_out=gh[b:b + 1]) for b, m in enumerate(ends)]
    pairs = [("gA", got["gA"], alone[0]["gA"] + alone[1]["gA"])]
    pairs += [(k, got[k][:m, b:b + 1], alone[b][k]) for k in ("gx", "gB", "gC") for b, m in enumerate(ends)]
    for name, v, ref in pairs:
        assert torch.equal(torch.isinf(v.cpu()), torch.isinf(ref)), name
        assert torch.equal(torch.isnan(v.cpu()), torch.isnan(ref)), name


@pytest.mark.parametrize("S", [3, 16])
@pytest.mark.parametrize("T", [1, 9, 150])
@pytest.mark.parametrize("which", ["Bm", "Cm"])
def test_infinite_b_and_c(ops, which, T, S):
    """An infinite B or C gives infinite results where the definition does: lanes behind the last
    feature, which see the same B and C, add nothing to the sums over features."""
    B, F, at = 2, 67, T // 2
    x, dt, Bm, Cm, gy = (positive(i, *s) for i, s in enumerate(((T, B, F), (T, B, F), (T, B, 1, S), (T, B, 1, S), (T, B, F))))
    A = -positive(6, F, S)
    {"Bm": Bm, "Cm": Cm}[which][at, 0, 0, S - 1] = float("inf")
    h = torch.empty((B, F, S), device="cuda")
    y, saved = ops.scan_forward(x, dt, A, Bm, Cm, h_out=h, train=True)
    got = dict(zip(NAMES, ops.scan_backward(x, dt, A, Bm, Cm, None, None, saved, gy)))
    ref = R.scan(x, dt, A, Bm, Cm, gy=gy)
    for name, v in {"y": y, "h_out": h, **{k: got[k] for k in ("gx", "gdt", "gA", "gB", "gC")}}.items():
        assert torch.equal(torch.isinf(v.cpu()), torch.isinf(ref[name])), name
        assert torch.equal(torch.isnan(v.cpu()), torch.isnan(ref[name])), name


@pytest.mark.parametrize("io,F", [("f32", 9), ("bf16", 64)])
@pytest.mark.parametrize("at", [0, 7, 8, 9, 10, 11, 39])
def test_infinite_inputs_of_a_convolution(ops, at, io, F):
    """An infinite input gives its own filter infinite gradients, wherever it lies to the chunks that
    share out the steps, and no others."""
    T, B, W = 40, 2, 4
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[io]
    x, gy = positive(1, T, B, F).to(dt), positive(2, T, B, F).to(dt)
    w, bias = normal(3, F, W), normal(4, F)
    x[at, 1, F - 2] = float("inf")
    gx, gw, gb, _ = ops.conv_backward(x, w, bias, gy, act=None)
    ref = R.conv(x, w, bias, act=None, gy=gy)
    for name, v in (("gx", gx), ("gw", gw), ("gb", gb)):
        assert torch.equal(torch.isinf(v.cpu()), torch.isinf(ref[name])), name
        assert torch.equal(torch.isnan(v.cpu()), torch.isnan(ref[name])), name
