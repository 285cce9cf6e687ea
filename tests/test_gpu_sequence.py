"""The sequence operators on the GPU against their 64-bit definitions (tests/sequence_ref.py):
odd sizes, one step and many, padded batches with whatever in the padding, strides, states
handed on and updated in place, both I/O types."""
import pytest
import torch

from tests import sequence_ref as R

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2408_00280_amd import sequence
    return sequence


def normal(seed, *shape, dtype=torch.float32, mean=0.0, sd=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, sd, generator=g)


def laid_out(v, layout):
    """The same values [T, B, X...] in another layout."""
    T, B = v.shape[:2]
    if layout == "batch":                                   # [B, T, X] transposed
        return v.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "slice":                                   # odd offset in rows of odd length
        X = v[0, 0].numel() if T and B else 1
        wide = torch.full((T, B, 2 * X + 3), float("nan"), dtype=v.dtype, device=v.device)
        wide[..., 1:X + 1] = v.reshape(T, B, X)
        return wide[..., 1:X + 1].unflatten(2, v.shape[2:])
    return v


def lengths_of(kind, T, B):
    if kind is None:
        return None
    n = [(T * (i + 1)) // B - (i % 2) for i in range(B)]
    n[0], n[-1] = 0, T
    if B > 2:
        n[1] = T + 5                                        # taken as T
        n[2] = -3                                           # taken as 0
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def poison(lengths, *ts):
    """NaN and infinities behind each sequence's end."""
    if lengths is None:
        return
    for t in ts:
        if t is not None:
            T, B = t.shape[:2]
            for b, n in enumerate(R.steps(T, B, lengths)):
                t[n:, b] = float("nan")
                t[n + 1:, b] = float("inf")


def plain(lengths, *ts):
    """The same with zeros there, for the 64-bit side."""
    out = []
    for t in ts:
        if t is None or lengths is None:
            out.append(t)
        else:
            T, B = t.shape[:2]
            m = R.inside(T, B, lengths).to(t.device)
            out.append(torch.where(m.view(T, B, *([1] * (t.dim() - 2))), t, torch.zeros_like(t)))
    return out


# ---------------------------------------------------------------------------------------

CONV = [
    # T, B, F, W, act, bias, state, lengths, layout
    (1, 1, 1, 4, "silu", True, True, None, None),
    (1, 3, 1030, 4, "silu", True, True, None, "slice"),
    (2, 3, 9, 4, "silu", True, True, "ragged", None),
    (3, 2, 64, 8, None, False, True, None, "batch"),
    (17, 4, 5, 1, "silu", True, False, "ragged", None),
    (40, 4, 129, 2, None, True, False, "ragged", "slice"),
    (70, 5, 264, 4, "silu", True, True, "ragged", None),
    (70, 3, 263, 3, "silu", False, True, "ragged", "batch"),
    (33, 2, 8, 7, "silu", True, False, None, None),
    (600, 1, 40, 4, "silu", True, True, None, None),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,F,W,act,has_bias,has_state,ragged,layout", CONV)
def test_conv(ops, io, T, B, F, W, act, has_bias, has_state, ragged, layout):
    dt = DTYPES[io]
    x, gy = normal(1, T, B, F, dtype=dt), normal(2, T, B, F, dtype=dt)
    w = normal(3, F, W)
    bias = normal(4, F) if has_bias else None
    state = normal(5, W - 1, B, F, dtype=dt) if has_state else None
    gstate = normal(6, W - 1, B, F, dtype=dt) if has_state else None
    ln = lengths_of(ragged, T, B)
    args = dict(act=act, state=state, lengths=None if ln is None else ln.cpu())
    ref, mag = (R.conv(*plain(ln, x), w, bias, gy=plain(ln, gy)[0], gstate_out=gstate, mag=m, **args) for m in (False, True))
    poison(ln, x, gy)
    x, gy = laid_out(x, layout), laid_out(gy, layout)
    out = torch.full((W - 1, B, F), float("nan"), dtype=dt, device="cuda")
    y = ops.conv_forward(x, w, bias, act=act, state=state, state_out=out, lengths=ln)
    gx, gw, gb, gs = ops.conv_backward(x, w, bias, gy, act=act, state=state, lengths=ln, grad_state_out=gstate)
    n = 3 * W + 32
    R.check("y", y, ref["y"], mag["y"], n)
    assert torch.equal(out.cpu().to(torch.float64), ref["state_out"])
    R.check("gx", gx, ref["gx"], mag["gx"], 2 * n)
    R.check("gw", gw, ref["gw"], mag["gw"], 2 * n + T * B)
    if has_bias:
        R.check("gb", gb, ref["gb"], mag["gb"], 2 * n + T * B)
    if has_state:
        R.check("gstate", gs, ref["gstate"], mag["gstate"], 2 * n)
        inplace = state.clone()
        y2 = ops.conv_forward(x, w, bias, act=act, state=inplace, state_out=inplace, lengths=ln)
        assert torch.equal(y2, y) and torch.equal(inplace, out)


def test_conv_tokens_equal_prompt(ops):
    """Tokens one at a time on a state updated in place give the prompt's outputs bit for bit,
    and so do two pieces of the prompt."""
    T, B, F, W = 12, 3, 70, 4
    x, w, bias = normal(1, T, B, F), normal(2, F, W), normal(3, F)
    y = ops.conv_forward(x, w, bias)
    state = torch.zeros((W - 1, B, F), device="cuda")
    for t in range(T):
        assert torch.equal(ops.conv_forward(x[t:t + 1], w, bias, state=state, state_out=state)[0], y[t])
    assert torch.equal(state, x[T - W + 1:])
    state = torch.zeros((W - 1, B, F), device="cuda")
    parts = [ops.conv_forward(p, w, bias, state=state, state_out=state) for p in (x[:2], x[2:])]
    assert torch.equal(torch.cat(parts), y)


# ---------------------------------------------------------------------------------------

SCAN = [
    # T, B, F, S, G, softplus, options (D, bias, h), lengths, layout
    (1, 1, 1, 1, 1, True, "", None, None),
    (1, 3, 65, 16, 1, True, "D bias h", None, None),
    (2, 2, 130, 4, 2, True, "D bias", None, "slice"),
    (15, 3, 64, 16, 1, True, "D bias h", None, "batch"),
    (16, 2, 63, 3, 1, False, "D h", None, None),
    (17, 3, 96, 5, 3, True, "bias h", "ragged", None),
    (33, 4, 70, 16, 1, True, "D bias h", "ragged", "slice"),
    (50, 5, 129, 7, 3, True, "D bias", "ragged", "batch"),
    (40, 1, 66, 17, 2, True, "D bias h", None, None),
    (24, 2, 40, 33, 1, True, "D bias h", "ragged", None),
    (20, 1, 72, 64, 2, True, "D bias h", None, "slice"),
    (130, 1, 64, 16, 1, True, "D bias h", None, None),
    (300, 1, 20, 8, 2, True, "D bias", None, None),
    (270, 4, 70, 16, 1, True, "D bias h", "ragged", "batch"),     # several segments of the time axis
    (333, 3, 65, 33, 1, True, "bias h", "ragged", None),
    (150, 2, 130, 2, 2, False, "h", "ragged", "slice"),
    (1, 33, 2100, 62, 3, True, "D bias h", "ragged", "slice"),    # several sequences per lane
]


def scan_inputs(io, T, B, F, S, G, options, seed=0):
    dt = DTYPES[io]
    x, step, gy = (normal(seed + i, T, B, F, dtype=dt) for i in (1, 2, 3))
    Bm, Cm = (normal(seed + i, T, B, G, S, dtype=dt) for i in (4, 5))
    A = -torch.exp(normal(seed + 6, F, S, sd=0.7))
    D = normal(seed + 7, F) if "D" in options else None
    bias = normal(seed + 8, F, mean=-1.0) if "bias" in options else None
    h, gh = (normal(seed + i, B, F, S) if "h" in options.split() else None for i in (9, 10))
    return x, step, A, Bm, Cm, D, bias, h, gy, gh


NAMES = ("gx", "gdt", "gA", "gB", "gC", "gD", "gdt_bias", "gh_in")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,F,S,G,softplus,options,ragged,layout", SCAN)
def test_scan(ops, io, T, B, F, S, G, softplus, options, ragged, layout):
    x, step, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs(io, T, B, F, S, G, options)
    if not softplus:
        step = step.abs() * 0.3
    ln = lengths_of(ragged, T, B)
    px, pstep, pB, pC, pgy = plain(ln, x, step, Bm, Cm, gy)
    ref, mag = (R.scan(px, pstep, A, pB, pC, D, bias, softplus=softplus, h_in=h, lengths=None if ln is None else ln.cpu(),
                       gy=pgy, gh_out=gh, mag=m) for m in (False, True))
    poison(ln, x, step, Bm, Cm, gy)
    x, step, Bm, Cm, gy = (laid_out(v, layout) for v in (x, step, Bm, Cm, gy))
    out = torch.full((B, F, S), float("nan"), device="cuda")
    args = (x, step, A, Bm, Cm, D, bias)
    y, saved = ops.scan_forward(*args, softplus=softplus, h_in=h, h_out=out, lengths=ln, train=True)
    got = ops.scan_backward(*args, saved, gy, softplus=softplus, h_in=h, lengths=ln, grad_h_out=gh)
    n = R.scan_roundings(T, B, F, S)
    R.check("y", y, ref["y"], mag["y"], n)
    R.check("h_out", out, ref["h_out"], mag["h_out"], n)
    given = (True,) * 5 + (D is not None, bias is not None, h is not None)
    for name, g, there in zip(NAMES, got, given):
        if there:
            R.check(name, g, ref[name], mag[name], n)
        else:
            assert g is None
    y2, none = ops.scan_forward(*args, softplus=softplus, h_in=h, lengths=ln)
    assert none is None and torch.equal(y2, y)
    if h is not None:
        inplace = h.clone()
        y3, _ = ops.scan_forward(*args, softplus=softplus, h_in=inplace, h_out=inplace, lengths=ln)
        assert torch.equal(y3, y) and torch.equal(inplace, out)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_scan_tokens_follow_a_prompt(ops, io):
    """A prompt's state, then single tokens on it in place: the whole sequence's outputs."""
    T, P, B, F, S, G = 40, 33, 3, 70, 16, 2
    x, step, A, Bm, Cm, D, bias, *_ = scan_inputs(io, T, B, F, S, G, "D bias")
    ref, mag = (R.scan(x, step, A, Bm, Cm, D, bias, mag=m) for m in (False, True))
    h = torch.empty((B, F, S), device="cuda")
    ys = [ops.scan_forward(x[:P], step[:P], A, Bm[:P], Cm[:P], D, bias, h_out=h)[0]]
    for t in range(P, T):
        i = slice(t, t + 1)
        ys.append(ops.scan_forward(x[i], step[i], A, Bm[i], Cm[i], D, bias, h_in=h, h_out=h)[0])
    n = R.scan_roundings(T, B, F, S)
    R.check("y", torch.cat(ys), ref["y"], mag["y"], n)
    R.check("h", h, ref["h_out"], mag["h_out"], n)


@pytest.mark.parametrize("value", [-30.0, -9.0, 0.0, 9.0, 30.0, 200.0])
def test_scan_steps_at_the_ends_of_the_softplus(ops, value):
    """Steps from 1e-13 to 200: ln(1 + e^v) keeps its relative precision where e^v is far
    below 1, and large steps forget the state."""
    T, B, F, S = 5, 1, 64, 4
    x, _, A, Bm, Cm, D, _, h, gy, gh = scan_inputs("f32", T, B, F, S, 1, "h")
    step = torch.full((T, B, F), value, device="cuda")
    Cm = Cm.abs()
    ref, mag = (R.scan(x, step, A, Bm, Cm, h_in=0 * h, gy=gy, gh_out=gh, mag=m) for m in (False, True))
    y, saved = ops.scan_forward(x, step, A, Bm, Cm, h_in=0 * h, train=True)
    got = ops.scan_backward(x, step, A, Bm, Cm, None, None, saved, gy, h_in=0 * h, grad_h_out=gh)
    n = R.scan_roundings(T, B, F, S)
    # a step of 30 or 200 takes decays under 2^-126, which become 0: with d <= 200, |A| < 20 and
    # normal values under 6, the state is at most T d x B < 5 * 200 * 36 = 4e4, dL/dh at most
    # T C dL/dy < 200, and what a decay is multiplied with at most T d A dL/dh h < 2e11
    R.check("y", y, ref["y"], mag["y"], n, 2e11)
    for name, g in zip(NAMES, got):
        if g is not None:
            R.check(name, g, ref[name], mag[name], n, 2e11)


# ---------------------------------------------------------------------------------------

NORM = [
    # T, B, F, parts, lengths, layout, gradients that are given
    (1, 1, 1, "r z w_post scale w_pre", None, None, "r u"),
    (3, 2, 7, "r z w_post scale w_pre", "ragged", None, "r u"),
    (5, 3, 64, "r w_pre", None, "batch", "u"),
    (4, 2, 257, "z w_post", None, "slice", "r"),
    (2, 3, 1000, "r z scale", "ragged", None, "r"),
    (3, 4, 1536, "r z w_post scale w_pre", "ragged", "slice", "r u"),
    (2, 2, 4097, "w_post w_pre", None, None, "r u"),
    (40, 60, 33, "r z w_post scale w_pre", None, None, "r u"),
    (1, 2, 20000, "r z w_post scale w_pre", None, None, "r u"),
    (2, 1, 70001, "r z w_post scale w_pre", None, None, "r u"),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,F,parts,ragged,layout,given", NORM)
def test_norm(ops, io, T, B, F, parts, ragged, layout, given):
    dt = DTYPES[io]
    rows = {k: normal(i, T, B, F, dtype=dt) for i, k in enumerate(("y", "r", "z")) if k == "y" or k in parts.split()}
    weights = {k: normal(10 + i, F, mean=1.0, sd=0.3) for i, k in enumerate(("w_post", "scale", "w_pre")) if k in parts.split()}
    grads = {k: normal(20 + i, T, B, F, dtype=dt) for i, k in enumerate(("r", "u")) if k in given.split()}
    ln = lengths_of(ragged, T, B)
    cpu = None if ln is None else ln.cpu()
    pr, pg = dict(zip(rows, plain(ln, *rows.values()))), dict(zip(grads, plain(ln, *grads.values())))
    ref, mag = (R.norm(**pr, **weights, lengths=cpu, g_r=pg.get("r"), g_u=pg.get("u"), mag=m) for m in (False, True))
    poison(ln, *rows.values(), *grads.values())
    rows = {k: laid_out(v, layout) for k, v in rows.items()}
    grads = {k: laid_out(v, layout) for k, v in grads.items()}
    args = (rows["y"], rows.get("r"), rows.get("z"), *(weights.get(k) for k in ("w_post", "scale", "w_pre")))
    r_new, u, rstd = ops.norm_forward(*args, lengths=ln, train=True)
    got = ops.norm_backward(*args, rstd, grads.get("r"), grads.get("u"), lengths=ln)
    n = R.norm_roundings(T, B, F)
    R.check("r_new", r_new, ref["r_new"], mag["r_new"], n)
    assert (u is None) == ("w_pre" not in weights)
    if u is not None:
        R.check("u", u, ref["u"], mag["u"], n)
    names = dict(zip(("gy", "gr", "gz", "gw_post", "gscale", "gw_pre"), got))
    wanted = {"gy"} | {"g" + k for k in parts.split()}
    for name, g in names.items():
        assert (g is not None) == (name in wanted), name
        if g is not None:
            if name == "gw_pre" and "u" not in grads:
                assert not g.any()
            else:
                R.check(name, g, ref[name], mag[name], n)
    again = ops.norm_forward(y=args[0], **dict(zip(("r", "z", "w_post", "scale", "w_pre"), args[1:])), lengths=ln)
    assert torch.equal(again[0], r_new) and again[2] is None


# ---------------------------------------------------------------------------------------

def block(A, seed, T, B, F, S, G, W, dtype):
    """A block as a model has it: norm -> conv -> scan -> LIF -> gate, norm, residual -> norm."""
    from paper_2408_00280_amd import autograd
    torch.manual_seed(seed)
    conv, scan = autograd.CausalConv(F, W).cuda(), autograd.SelectiveScan(F, S).cuda()
    lif, norm = autograd.LIFLayer(0.5, 0.4), autograd.BlockNorm(F, scale=0.5).cuda()
    return conv, scan, lif, norm


def run_block(mods, x, z, dt, Bm, Cm, lengths=None):
    conv, scan, lif, norm = mods
    c = conv(x, lengths=lengths)
    return norm(lif(scan(c, dt, Bm, Cm, lengths=lengths)), x, z, lengths=lengths)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_operators_together(ops, io):
    """A whole block, forward and backward through autograd, a padded batch: rows behind the
    sequences are 0 and take no gradient whatever they hold, and the batch gives each
    sequence's outputs as alone."""
    T, B, F, S, G, W = 21, 3, 72, 16, 2, 4
    dt = DTYPES[io]
    mods = block(ops, 0, T, B, F, S, G, W, dt)
    leaves = [normal(i, T, B, F, dtype=dt) for i in (1, 2, 3)] + [normal(i, T, B, G, S, dtype=dt) for i in (4, 5)]
    ln = torch.tensor([21, 0, 13], dtype=torch.int32, device="cuda")
    poison(ln, *leaves)
    for v in leaves:
        v.requires_grad_(True)
    r, u = run_block(mods, *leaves, lengths=ln)
    (r.float().square().sum() + u.float().sum()).backward()
    assert torch.isfinite(r).all() and torch.isfinite(u).all()
    for b, n in enumerate(ln.tolist()):
        assert not r[n:, b].any() and not u[n:, b].any()
        if n:
            alone = run_block(mods, *(v.detach()[:n, b:b + 1] for v in leaves))
            assert torch.equal(alone[0], r[:n, b:b + 1]) and torch.equal(alone[1], u[:n, b:b + 1])
        for v in leaves:
            assert torch.isfinite(v.grad[:, b]).all() and not v.grad[n:, b].any()
    for m in mods:
        for p in m.parameters():
            assert p.grad is not None and torch.isfinite(p.grad).all()


def test_modules_step_like_their_prompt(ops):
    T, B, F, S, G, W = 9, 2, 70, 16, 1, 4
    conv, scan, _, _ = block(ops, 0, T, B, F, S, G, W, torch.float32)
    x, dt, Bm, Cm = normal(1, T, B, F), normal(2, T, B, F), normal(3, T, B, G, S), normal(4, T, B, G, S)
    with torch.no_grad():
        c = conv(x)
        y = scan(c, dt, Bm, Cm)
        state, h = torch.zeros((W - 1, B, F), device="cuda"), torch.zeros((B, F, S), device="cuda")
        for t in range(T):
            ct = conv.step(x[t], state)
            yt = scan.step(ct, dt[t], Bm[t], Cm[t], h)
            assert torch.equal(ct, c[t])
            torch.testing.assert_close(yt, y[t], rtol=0, atol=float((26 * T + 128) * R.U32 * 4 * y.abs().max()))


def test_shared_inputs_get_the_sum_of_their_gradients(ops):
    """B and C broadcast over the batch (steps of 0) and one tensor used as x and dt."""
    from paper_2408_00280_amd import autograd
    T, B, F, S = 12, 3, 66, 8
    x, _, A, Bm, Cm, D, bias, _, gy, _ = scan_inputs("f32", T, B, F, S, 1, "D bias")
    one = Bm[:, :1].clone().requires_grad_(True)
    xs = x.clone().requires_grad_(True)
    y = autograd.selective_scan(xs, xs, A, one.expand(T, B, 1, S), Cm, D, bias)
    gx, gB = torch.autograd.grad(y, (xs, one), gy)
    full = one.detach().expand(T, B, 1, S).contiguous()
    ref, mag = (R.scan(x, x, A, full, Cm, D, bias, gy=gy, mag=m) for m in (False, True))
    n = R.scan_roundings(T, B, F, S)
    R.check("y", y, ref["y"], mag["y"], n)
    R.check("x", gx, ref["gx"] + ref["gdt"], mag["gx"] + mag["gdt"], n + 1)
    R.check("B", gB, ref["gB"].sum(1, keepdim=True), mag["gB"].sum(1, keepdim=True), n + B)


def test_state_gradients_through_autograd(ops):
    """Two pieces joined by their states: the whole sequence's gradients."""
    from paper_2408_00280_amd import autograd
    T, P, B, F, S, W = 20, 7, 2, 66, 8, 4
    x, dt, A, Bm, Cm, D, bias, _, gy, _ = scan_inputs("f32", T, B, F, S, 1, "D bias")
    w = normal(40, F, W)
    for v in (x, dt, Bm, Cm, A, w):
        v.requires_grad_(True)

    def run(pieces):
        ys, st, h = [], None, None
        for i in pieces:
            c, st = autograd.causal_conv(x[i], w, act="silu", state=st, return_state=True)
            y, h = autograd.selective_scan(c, dt[i], A, Bm[i], Cm[i], D, bias, h_in=h, return_state=True)
            ys.append(y)
        y = torch.cat(ys)
        return y, torch.autograd.grad(y, (x, dt, Bm, Cm, A, w), gy)
    whole, split = run([slice(0, T)]), run([slice(0, P), slice(P, T)])
    tol = R.scan_roundings(T, B, F, S) * R.U32
    for a, b in zip((whole[0], *whole[1]), (split[0], *split[1])):
        assert (a - b).abs().max() <= 8 * tol * a.abs().max()


@pytest.mark.parametrize("op", ["conv", "scan", "norm"])
def test_graph_replays_match_eager(ops, op):
    """Forward and backward captured, replayed with new inputs and other work in between; two
    graphs at once do not share scratch memory that either still needs."""
    T, B, F, S, G, W = 40, 2, 130, 16, 1, 4
    x, step, A, Bm, Cm, D, bias, h, gy, gh = scan_inputs("bf16", T, B, F, S, G, "D bias h")
    w, wp = normal(50, F, W), normal(51, F, mean=1.0)

    def run():
        if op == "conv":
            return [ops.conv_forward(x, w, bias), *ops.conv_backward(x, w, bias, gy)[:3]]
        if op == "scan":
            y, saved = ops.scan_forward(x, step, A, Bm, Cm, D, bias, h_in=h, train=True)
            return [y, *ops.scan_backward(x, step, A, Bm, Cm, D, bias, saved, gy, h_in=h, grad_h_out=gh)]
        r, u, rstd = ops.norm_forward(x, step, gy, wp, D, wp, train=True)
        return [r, u, *ops.norm_backward(x, step, gy, wp, D, wp, rstd, gy, x)]

    run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = run()
        graphs.append((g, outs))
    for rep in range(3):
        x.copy_(normal(100 + rep, T, B, F, dtype=x.dtype))
        ref = [v.clone() for v in run()]
        for _, outs in graphs:
            for v in outs:
                v.fill_(float("nan"))
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            for a, b in zip(outs, ref):
                assert torch.equal(a, b), f"replay {rep}"
        del junk


def test_two_streams_and_repeats(ops):
    """The same calls on two streams at once and again and again give the same bits."""
    T, B, F, S, G, W = 64, 2, 300, 16, 1, 4
    ins = [scan_inputs("f32", T, B, F, S, G, "D bias h", seed=s) for s in (0, 100)]
    w = normal(50, F, W)
    torch.cuda.synchronize()

    def run(v, stream=None):
        x, step, A, Bm, Cm, D, bias, h, gy, gh = v
        y, saved = ops.scan_forward(x, step, A, Bm, Cm, D, bias, h_in=h, train=True, stream=stream)
        g = ops.scan_backward(x, step, A, Bm, Cm, D, bias, saved, gy, h_in=h, grad_h_out=gh, stream=stream)
        c = ops.conv_forward(x, w, bias, stream=stream)
        return [y, c, *g, *ops.conv_backward(x, w, bias, gy, stream=stream)[:3]]
    ref = [run(v) for v in ins]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for rep in range(4):
        got = [run(v, s if rep % 2 else s.cuda_stream) for v, s in zip(ins, streams)]
        torch.cuda.synchronize()
        for a, b in zip(ref, got):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_empty_problems(ops):
    """No steps hand the state on; no sequences or features give empty outputs and zero
    gradients of the parameters."""
    for T, B, F in ((0, 2, 5), (3, 0, 5), (3, 2, 0)):
        x = torch.empty((T, B, F), device="cuda")
        bc = torch.empty((T, B, 1, 4), device="cuda")
        w, A, one = normal(1, F, 3), normal(2, F, 4), normal(3, F)
        state, h = normal(4, 2, B, F), normal(5, B, F, 4)
        out, hout = torch.empty_like(state), torch.empty_like(h)
        assert ops.conv_forward(x, w, one, state=state, state_out=out).shape == x.shape
        gx, gw, gb, gs = ops.conv_backward(x, w, one, x, state=state, grad_state_out=state)
        assert gx.shape == x.shape and not gw.any() and not gb.any()
        y, saved = ops.scan_forward(x, x, A, bc, bc, one, one, h_in=h, h_out=hout, train=True)
        g = ops.scan_backward(x, x, A, bc, bc, one, one, saved, x, h_in=h, grad_h_out=h)
        assert y.shape == x.shape and not any(v.any() for v in g[2:7])
        if T == 0:
            assert torch.equal(out, state) and torch.equal(hout, h) and torch.equal(gs, state) and torch.equal(g[7], h)
        r, u, rstd = ops.norm_forward(x, x, x, one, one, one, train=True)
        assert r.shape == u.shape == x.shape
        assert not any(v.any() for v in ops.norm_backward(x, x, x, one, one, one, rstd, x, x)[3:])


def test_refusals(ops):
    x, w, A = normal(1, 4, 2, 6), normal(2, 6, 3), normal(3, 6, 4)
    bc = normal(4, 4, 2, 1, 4)
    state, h = normal(5, 2, 2, 6), normal(6, 2, 6, 4)
    bad = [
        lambda: ops.conv_forward(x.cpu(), w),
        lambda: ops.conv_forward(x.half(), w),
        lambda: ops.conv_forward(x[0], w),
        lambda: ops.conv_forward(x, w[:5]),
        lambda: ops.conv_forward(x, w.double()),
        lambda: ops.conv_forward(x, w.t().contiguous().t()),
        lambda: ops.conv_forward(x, w, act="relu"),
        lambda: ops.conv_forward(x, w, state=state[:1]),
        lambda: ops.conv_forward(x, w, state=state.bfloat16()),
        lambda: ops.conv_forward(x, w, lengths=torch.ones(2, device="cuda", dtype=torch.int64)),
        lambda: ops.conv_forward(x, w, lengths=torch.ones(2, dtype=torch.int32)),
        lambda: ops.conv_backward(x, w, None, x[:3]),
        lambda: ops.scan_forward(x, x.bfloat16(), A, bc, bc),
        lambda: ops.scan_forward(x, x, A, bc[..., :3], bc),
        lambda: ops.scan_forward(x, x, A, bc, bc.cpu()),
        lambda: ops.scan_forward(x, x, A, bc, bc, h_in=h[:, :, :3]),
        lambda: ops.scan_forward(x, x, A, bc, bc, h_in=h, h_out=h, train=True),
        lambda: ops.scan_backward(x, x, A, bc, bc, None, None, torch.empty(3, dtype=torch.uint8, device="cuda"), x),
        lambda: ops.norm_forward(x, x[:2]),
        lambda: ops.norm_forward(x, w_post=w[0]),
        lambda: ops.norm_backward(x, None, None, None, None, None, h, x),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was taken")
    from paper_2408_00280_amd.native import SnnError
    wide = normal(7, 4, 2, 1, 65)
    for call in (lambda: ops.conv_forward(x, normal(8, 6, 9)), lambda: ops.norm_forward(x, eps=0.0),
                 lambda: ops.scan_forward(x, x, normal(9, 6, 65), wide, wide),
                 lambda: ops.scan_forward(x, x, A, bc.expand(4, 2, 4, 4).contiguous(), bc.expand(4, 2, 4, 4).contiguous())):
        with pytest.raises(SnnError):
            call()
