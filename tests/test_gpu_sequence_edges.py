"""The sequence operators where calls go wrong first: random configurations, offsets past 32
bits, outputs that are slices of wider rows (nothing beside them is written), values that are
not finite in one sequence or feature, and a whole block captured into a graph."""
import gc
import random

import pytest
import torch

from tests import sequence_ref as R
from tests.test_gpu_sequence import (DTYPES, NAMES, block, laid_out, lengths_of, normal, plain, poison, run_block,
                                     scan_inputs)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2408_00280_amd import sequence
    return sequence


def some(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


@pytest.mark.parametrize("seed", range(24))
def test_random_scans(ops, seed):
    rng = random.Random(seed)
    G = rng.choice([1, 1, 2, 3])
    T, B, F, S = some(rng, 1, 400), some(rng, 1, 6), G * some(rng, 1, 70), rng.choice([1, 2, 4, 6, 8, 15, 16, 16, 31, 40, 64])
    io, options = rng.choice(["f32", "bf16"]), " ".join(o for o in ("D", "bias", "h") if rng.random() < 0.6)
    ragged, layout = rng.choice([None, "ragged"]) if B > 1 else None, rng.choice([None, "batch", "slice"])
    x, step, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs(io, T, B, F, S, G, options, seed=1000 * seed)
    ln = lengths_of(ragged, T, B)
    px, pstep, pB, pC, pgy = plain(ln, x, step, Bm, Cm, gy)
    ref, mag = (R.scan(px, pstep, A, pB, pC, D, bias, h_in=h, lengths=None if ln is None else ln.cpu(), gy=pgy, gh_out=gh,
                       mag=m) for m in (False, True))
    poison(ln, x, step, Bm, Cm, gy)
    x, step, Bm, Cm, gy = (laid_out(v, layout) for v in (x, step, Bm, Cm, gy))
    out = torch.empty((B, F, S), device="cuda")
    args = (x, step, A, Bm, Cm, D, bias)
    y, saved = ops.scan_forward(*args, h_in=h, h_out=out, lengths=ln, train=True)
    got = ops.scan_backward(*args, saved, gy, h_in=h, lengths=ln, grad_h_out=gh)
    n = R.scan_roundings(T, B, F, S)
    R.check("y", y, ref["y"], mag["y"], n)
    R.check("h_out", out, ref["h_out"], mag["h_out"], n)
    for name, g in zip(NAMES, got):
        if g is not None:
            R.check(name, g, ref[name], mag[name], n)


@pytest.mark.parametrize("seed", range(16))
def test_random_convolutions(ops, seed):
    rng = random.Random(100 + seed)
    T, B, F, W = some(rng, 1, 300), some(rng, 1, 6), some(rng, 1, 300), rng.randint(1, 8)
    dt, act, layout = DTYPES[rng.choice(["f32", "bf16"])], rng.choice([None, "silu"]), rng.choice([None, "batch", "slice"])
    x, gy, w, bias = normal(1, T, B, F, dtype=dt), normal(2, T, B, F, dtype=dt), normal(3, F, W), normal(4, F)
    state, gstate = normal(5, W - 1, B, F, dtype=dt), normal(6, W - 1, B, F, dtype=dt)
    ln = lengths_of(rng.choice([None, "ragged"]) if B > 1 else None, T, B)
    args = dict(act=act, state=state, lengths=None if ln is None else ln.cpu())
    ref, mag = (R.conv(*plain(ln, x), w, bias, gy=plain(ln, gy)[0], gstate_out=gstate, mag=m, **args) for m in (False, True))
    poison(ln, x, gy)
    x, gy = laid_out(x, layout), laid_out(gy, layout)
    out = torch.empty_like(state)
    y = ops.conv_forward(x, w, bias, act=act, state=state, state_out=out, lengths=ln)
    gx, gw, gb, gs = ops.conv_backward(x, w, bias, gy, act=act, state=state, lengths=ln, grad_state_out=gstate)
    n = 2 * (3 * W + 32)
    assert torch.equal(out.cpu().to(torch.float64), ref["state_out"])
    for name, g, k in (("y", y, n), ("gx", gx, n), ("gw", gw, n + T * B), ("gb", gb, n + T * B), ("gstate", gs, n)):
        R.check(name, g, ref[name], mag[name], k)


@pytest.mark.parametrize("seed", range(12))
def test_random_norms(ops, seed):
    rng = random.Random(200 + seed)
    T, B, F = some(rng, 1, 200), some(rng, 1, 8), some(rng, 1, 9000)
    T = max(1, min(T, 400000 // (B * F)))
    dt, layout = DTYPES[rng.choice(["f32", "bf16"])], rng.choice([None, "batch", "slice"])
    on = [rng.random() < 0.75 for _ in range(5)]
    y = normal(1, T, B, F, dtype=dt)
    r, z = (normal(i, T, B, F, dtype=dt) if o else None for i, o in zip((2, 3), on))
    w = [normal(i, F, mean=1.0, sd=0.3) if o else None for i, o in zip((4, 5, 6), on[2:])]
    g_r = normal(7, T, B, F, dtype=dt)
    g_u = normal(8, T, B, F, dtype=dt) if w[2] is not None else None
    ln = lengths_of(rng.choice([None, "ragged"]) if B > 1 else None, T, B)
    rows = (y, r, z, g_r, g_u)
    py, pr, pz, pgr, pgu = plain(ln, *rows)
    ref, mag = (R.norm(py, pr, pz, *w, lengths=None if ln is None else ln.cpu(), g_r=pgr, g_u=pgu, mag=m) for m in (False, True))
    poison(ln, *rows)
    y, r, z, g_r, g_u = (None if v is None else laid_out(v, layout) for v in rows)
    r_new, u, rstd = ops.norm_forward(y, r, z, *w, lengths=ln, train=True)
    got = dict(zip(("gy", "gr", "gz", "gw_post", "gscale", "gw_pre"),
                   ops.norm_backward(y, r, z, *w, rstd, g_r, g_u, lengths=ln)))
    n = R.norm_roundings(T, B, F)
    for name, g in {"r_new": r_new, "u": u, **got}.items():
        if g is not None:
            R.check(name, g, ref[name], mag[name], n)


def test_offsets_past_32_bits(ops):
    """Three steps 2^30 elements apart: the last lies past 2^31 elements and 2^32 bytes."""
    T, B, F, S, W = 3, 2, 70, 16, 4
    step = 1 << 30
    room = torch.empty(2 * step + 4096, dtype=torch.bfloat16, device="cuda")

    def far(v, at):
        out = room[at:].as_strided(v.shape, (step, v[0, 0].numel(), *torch.empty(v.shape[2:]).stride()))
        return out.copy_(v)
    x, dt, A, Bm, Cm, D, bias, _, gy, _ = scan_inputs("bf16", T, B, F, S, 1, "D bias")
    w = normal(20, F, W)
    near = (x, dt, Bm, Cm, gy)
    spread = [far(v, 256 * i) for i, v in enumerate(near)]

    def run(x, dt, Bm, Cm, gy):
        y, saved = ops.scan_forward(x, dt, A, Bm, Cm, D, bias, train=True)
        g = ops.scan_backward(x, dt, A, Bm, Cm, D, bias, saved, gy)
        c = [ops.conv_forward(x, w, bias), *ops.conv_backward(x, w, bias, gy)[:3]]
        r, u, rstd = ops.norm_forward(x, dt, gy, D, D, D, train=True)
        return [y, *g[:7], *c, r, u, *ops.norm_backward(x, dt, gy, D, D, D, rstd, gy, x)]
    for a, b in zip(run(*near), run(*spread)):
        assert torch.equal(a, b)
    # and outputs
    from paper_2408_00280_amd import native
    y = ops.conv_forward(x, w, bias)
    out = far(torch.zeros_like(x), 256 * 6)
    native.snn_conv_forward(native.snn_conv_cfg(1, W, 1), T, B, F, x, w, bias, None, None, out, None)
    assert torch.equal(out, y)


def test_outputs_beside_which_nothing_is_written(ops):
    """Every output as a slice at an odd offset of rows that are marked all over."""
    from paper_2408_00280_amd import native as N
    T, B, F, S, G, W = 37, 3, 69, 6, 3, 4
    x, dt, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs("bf16", T, B, F, S, G, "D bias h")
    w = normal(20, F, W)
    mark = 12345.0
    made = []

    def out(width, dtype=torch.bfloat16):
        wide = torch.full((T, B, width + 9), mark, dtype=dtype, device="cuda")
        made.append((wide, width))
        return wide[..., 3:3 + width]

    def params(n):
        wide = torch.full((n + 8,), mark, device="cuda")
        made.append((wide, n))
        return wide[3:3 + n]
    cfg = N.snn_scan_cfg(1, S, G, 1)
    ws = torch.empty(max(N.snn_scan_workspace_bytes(cfg, T, B, F)) + 512, dtype=torch.uint8, device="cuda")
    y, saved = ops.scan_forward(x, dt, A, Bm, Cm, D, bias, h_in=h, train=True)
    want = ops.scan_backward(x, dt, A, Bm, Cm, D, bias, saved, gy, h_in=h, grad_h_out=gh)
    yo, ho = out(F), params(B * F * S)
    N.snn_scan_forward(cfg, T, B, F, x, dt, A, Bm, Cm, D, bias, h, None, yo, ho, None, ws)
    g = [out(F), out(F), params(F * S), out(G * S), out(G * S), params(F), params(F), params(B * F * S)]
    N.snn_scan_backward(cfg, T, B, F, x, dt, A, Bm, Cm, D, bias, h, None, saved, gy, gh, *g, ws)
    assert torch.equal(yo, y)
    for a, b in zip(g, want):
        assert torch.equal(a.reshape(-1), b.reshape(-1))

    cfg = N.snn_conv_cfg(1, W, 1)
    ws = torch.empty(N.snn_conv_workspace_bytes(cfg, T, B, F), dtype=torch.uint8, device="cuda")
    want = [ops.conv_forward(x, w, bias), *ops.conv_backward(x, w, bias, gy)[:3]]
    g = [out(F), out(F), params(F * W), params(F)]
    N.snn_conv_forward(cfg, T, B, F, x, w, bias, None, None, g[0], None)
    N.snn_conv_backward(cfg, T, B, F, x, w, bias, None, None, gy, None, *g[1:], None, ws)
    for a, b in zip(g, want):
        assert torch.equal(a.reshape(-1), b.reshape(-1))

    cfg = N.snn_norm_cfg(1, 1e-5)
    ws = torch.empty(N.snn_norm_workspace_bytes(cfg, T, B, F), dtype=torch.uint8, device="cuda")
    r, u, rstd = ops.norm_forward(x, dt, gy, D, bias, D, train=True)
    want = [r, u, *ops.norm_backward(x, dt, gy, D, bias, D, rstd, gy, x)]
    g = [out(F), out(F)]
    N.snn_norm_forward(cfg, T, B, F, x, gy, dt, D, bias, D, None, *g, None)
    back = [out(F), out(F), out(F), params(F), params(F), params(F)]       # y, z, r and the weights
    N.snn_norm_backward(cfg, T, B, F, x, gy, dt, D, bias, D, None, rstd, gy, x, *back, ws)
    for a, b in zip(g + [back[0], back[2], back[1], *back[3:]], want):
        assert torch.equal(a.reshape(-1), b.reshape(-1))
    for wide, width in made:
        assert (wide[..., :3] == mark).all() and (wide[..., 3 + width:] == mark).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_where_it_belongs(ops, value):
    """One input value that is not finite reaches its own feature and sequence only (its own
    sequence through B and C), in forward and backward."""
    T, B, F, S, W = 40, 3, 70, 16, 4
    x, dt, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs("f32", T, B, F, S, 1, "D bias h")
    w = normal(20, F, W)

    def clean(t, b, f, ok):
        """Finite everywhere but at (from step t, sequence b, feature f)."""
        bad = ~torch.isfinite(ok)
        bad[t:, b, f] = False
        assert not bad.any()
    x[9, 1, 5] = value
    y = ops.conv_forward(x, w, bias)
    clean(9, 1, 5, y)
    assert torch.isfinite(y[9 + W:]).all()
    gx, gw, gb, _ = ops.conv_backward(x, w, bias, gy)
    assert torch.isfinite(gx[:9 - W]).all() and torch.isfinite(gx[:, [0, 2]]).all()
    assert torch.isfinite(gw[[0, 4, 6, 69]]).all()
    y, saved = ops.scan_forward(x, dt, A, Bm, Cm, D, bias, h_in=h, train=True)
    clean(9, 1, 5, y)
    g = ops.scan_backward(x, dt, A, Bm, Cm, D, bias, saved, gy, h_in=h, grad_h_out=gh)
    keep = [f for f in range(F) if f != 5]
    assert all(torch.isfinite(v[..., keep]).all() for v in g[:2]) and torch.isfinite(g[2][keep]).all()
    assert torch.isfinite(g[3][:, [0, 2]]).all() and torch.isfinite(g[4][:, [0, 2]]).all()
    x[9, 1, 5] = 0.0
    Bm[9, 1] = value
    y, _ = ops.scan_forward(x, dt, A, Bm, Cm, D, bias, h_in=h)
    assert torch.isfinite(y[:9]).all() and torch.isfinite(y[:, [0, 2]]).all()
    x[9, 1, 5] = value
    r, u, _ = ops.norm_forward(x, dt, gy, D, D, D)
    bad = ~torch.isfinite(r) | ~torch.isfinite(u)
    bad[9, 1] = False
    assert not bad.any()


@pytest.mark.parametrize("S", [1, 3, 7, 16])
@pytest.mark.parametrize("T", [1, 9, 150])
def test_infinities_are_not_made_nan(ops, S, T):
    """An infinite input gives infinite outputs where the definition does: states behind the
    last one and lanes behind the last feature add nothing to it."""
    B, F = 2, 67
    g = lambda seed, *shape: normal(seed, *shape).abs() + 0.1  # noqa: E731
    x, dt, Bm, Cm, gy = g(1, T, B, F), g(2, T, B, F), g(3, T, B, 1, S), g(4, T, B, 1, S), g(5, T, B, F)
    A = -g(6, F, S)
    x[0, 0, F - 1] = float("inf")
    h = torch.empty((B, F, S), device="cuda")
    y, saved = ops.scan_forward(x, dt, A, Bm, Cm, h_out=h, train=True)
    gx, _, _, gB, gC, *_ = ops.scan_backward(x, dt, A, Bm, Cm, None, None, saved, gy)
    ref = R.scan(x, dt, A, Bm, Cm, gy=gy)
    for name, v in (("y", y), ("h_out", h), ("gx", gx), ("gB", gB), ("gC", gC)):
        assert torch.equal(torch.isinf(v.cpu()), torch.isinf(ref[name])), name
        assert torch.equal(torch.isnan(v.cpu()), torch.isnan(ref[name])), name


@pytest.mark.parametrize("S", [3, 16])
@pytest.mark.parametrize("T", [1, 9, 150])
def test_rates_whose_exponent_is_past_the_type(ops, T, S):
    """A = -3e38 is finite and A log2(e) is not: such states forget all in a step, and keep
    what they hold behind the end of their sequence."""
    B, F = 3, 67
    x, step, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs("f32", T, B, F, S, 1, "D bias h")
    A[::2, S - 1] = -3e38
    ln = torch.tensor([T, T // 2, 0], dtype=torch.int32, device="cuda")
    ref, mag = (R.scan(x, step, A, Bm, Cm, D, bias, h_in=h, lengths=ln.cpu(), gy=gy, gh_out=gh, mag=m) for m in (False, True))
    out = torch.empty((B, F, S), device="cuda")
    y, saved = ops.scan_forward(x, step, A, Bm, Cm, D, bias, h_in=h, h_out=out, lengths=ln, train=True)
    got = ops.scan_backward(x, step, A, Bm, Cm, D, bias, saved, gy, h_in=h, lengths=ln, grad_h_out=gh)
    n = R.scan_roundings(T, B, F, S)
    for name, v in zip(("y", "h_out", *NAMES), (y, out, *got)):
        R.check(name, v, ref[name], mag[name], n)
    with pytest.raises(ValueError):
        ops.scan_backward(x, step, A, Bm, Cm, D, bias, None, gy, h_in=h, lengths=ln, grad_h_out=gh)


def test_gradients_are_differentiated_once(ops):
    """A second backward through a gradient raises an error: it is no constant."""
    from paper_2408_00280_amd import autograd
    x, step, A, Bm, Cm, *_ = scan_inputs("f32", 5, 2, 66, 4, 1, "")
    w = normal(9, 66, 4)
    for run in (lambda v: autograd.causal_conv(v, w), lambda v: autograd.selective_scan(v, step, A, Bm, Cm),
                lambda v: autograd.block_norm(v, w_pre=w[:, 0].contiguous())[1]):
        v = x.clone().requires_grad_(True)
        g, = torch.autograd.grad(run(v).square().sum(), v, create_graph=True)
        assert g.requires_grad
        with pytest.raises(RuntimeError):
            g.sum().backward()
        plain_g, = torch.autograd.grad(run(v).square().sum(), v)
        assert not plain_g.requires_grad and torch.equal(plain_g, g.detach())


def test_a_state_written_behind_a_graph_is_noticed(ops):
    """A state that a graph keeps for its backward and a later call updates in place."""
    from paper_2408_00280_amd import autograd
    x, step, A, Bm, Cm, _, _, h, *_ = scan_inputs("f32", 5, 2, 66, 4, 1, "h")
    w, state = normal(9, 66, 4), normal(10, 3, 2, 66)
    x.requires_grad_(True)
    y = autograd.selective_scan(x, step, A, Bm, Cm, h_in=h)
    ops.scan_forward(x.detach(), step, A, Bm, Cm, h_in=h, h_out=h)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()
    y = autograd.causal_conv(x, w, state=state)
    ops.conv_forward(x.detach(), w, state=state, state_out=state)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


def test_what_autograd_refuses(ops):
    """Wrong arguments raise the same errors as without gradients."""
    from paper_2408_00280_amd import autograd
    from paper_2408_00280_amd.native import SnnError
    x, step, A, Bm, Cm, *_ = scan_inputs("f32", 5, 2, 66, 4, 1, "")
    v = x.clone().requires_grad_(True)
    for call in (lambda: autograd.causal_conv(v, A[:, 0]), lambda: autograd.causal_conv(v, A, act="relu"),
                 lambda: autograd.causal_conv(v.cpu(), A), lambda: autograd.selective_scan(v, step[:3], A, Bm, Cm),
                 lambda: autograd.selective_scan(v, step, A.bfloat16(), Bm, Cm), lambda: autograd.block_norm(v, x[:3]),
                 lambda: autograd.selective_scan(v, step, A, Bm, Cm, h_in=A), lambda: autograd.causal_conv(v, None),
                 lambda: autograd.selective_scan(v, step, None, Bm, Cm), lambda: autograd.selective_scan(v, None, A, Bm, Cm),
                 lambda: autograd.selective_scan(v, step, A, None, Cm), lambda: autograd.block_norm(None),
                 lambda: ops.conv_forward(x, None), lambda: ops.scan_forward(x, step, A, None, Cm),
                 lambda: ops.norm_backward(None, None, None, None, None, None, None, x)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: autograd.causal_conv(v, normal(8, 66, 9)), lambda: autograd.block_norm(v, eps=0.0)):
        with pytest.raises(SnnError):
            call()


def test_block_captured_through_autograd(ops):
    """A block's forward and gradients captured into a graph with no eager graph of its leaves
    alive; every replay, with new inputs and other work in between, gives the eager values."""
    T, B, F, S, G, W = 24, 2, 72, 16, 2, 4
    mods = block(ops, 0, T, B, F, S, G, W, torch.float32)
    leaves = [normal(i, T, B, F).requires_grad_(True) for i in (1, 2, 3)]
    leaves += [normal(i, T, B, G, S).requires_grad_(True) for i in (4, 5)]
    params = [p for m in mods for p in m.parameters()]
    g1, g2 = normal(6, T, B, F), normal(7, T, B, F)

    def run():
        r, u = run_block(mods, *leaves)
        return [r, u, *torch.autograd.grad((r, u), leaves + params, (g1, g2))]

    def eager():
        return [v.detach().clone() for v in run()]
    eager()
    gc.collect()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [v.detach() for v in run()]
    for rep in range(3):
        with torch.no_grad():
            leaves[0].copy_(normal(100 + rep, T, B, F))
        ref = eager()
        for v in outs:
            v.fill_(float("nan"))
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, ref):
            assert torch.equal(a, b)
        del junk
