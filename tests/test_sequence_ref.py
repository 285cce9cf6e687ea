"""The 64-bit definitions of the sequence operators that the GPU tests compare with: their
written-out gradients against central differences of their forwards (a difference over 2h is
off by h^2 / 6 times the third derivative and by 2^-53 of the values over h: h = 1e-5 leaves
less than 1e-7 of values of order 1), and closed forms."""
import math

import pytest
import torch

from tests import sequence_ref as R

F64 = torch.float64


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rnd(g, *shape):
    return torch.randn(shape, generator=g, dtype=F64)


def differences(f, args, weights, names):
    """d(sum of outputs times weights)/d(arg) by central differences, for some entries."""
    def value():
        out = f(*args.values())
        return sum(float((out[k] * w).sum()) for k, w in weights.items())
    h = 1e-5
    for name in names:
        flat = args[name].view(-1)
        for i in {0, flat.numel() // 2, flat.numel() - 1}:
            old = float(flat[i])
            flat[i] = old + h
            up = value()
            flat[i] = old - h
            down = value()
            flat[i] = old
            yield name, i, (up - down) / (2 * h)


def compare(grads, got):
    for name, i, d in got:
        g = float(grads[name].reshape(-1)[i])
        assert abs(g - d) <= 1e-6 * max(1.0, abs(g)), (name, i, g, d)


LENGTHS = [None, [5, 0, 2]]


@pytest.mark.parametrize("act", ["silu", None])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("W", [1, 3, 4])
def test_conv_gradients(act, lengths, W):
    g = gen(W)
    T, B, F = 5, 3, 4
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    args = {"x": rnd(g, T, B, F), "w": rnd(g, F, W), "b": rnd(g, F), "s": rnd(g, W - 1, B, F)}
    gy, gs = rnd(g, T, B, F), rnd(g, W - 1, B, F)
    run = lambda x, w, b, s, **k: R.conv(x, w, b, state=s, act=act, lengths=ln, **k)  # noqa: E731
    out = run(*args.values(), gy=gy, gstate_out=gs)
    names = ["x", "w", "b"] + (["s"] if W > 1 else [])
    compare({"x": out["gx"], "w": out["gw"], "b": out["gb"], "s": out["gstate"]},
            differences(run, args, {"y": gy, "state_out": gs}, names))


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("G", [1, 2])
def test_scan_gradients(softplus, lengths, G):
    g = gen(G)
    T, B, F, S = 5, 3, 4, 3
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    args = {"x": rnd(g, T, B, F), "dt": rnd(g, T, B, F), "A": -rnd(g, F, S).abs(), "B": rnd(g, T, B, G, S),
            "C": rnd(g, T, B, G, S), "D": rnd(g, F), "bias": rnd(g, F), "h": rnd(g, B, F, S)}
    gy, gh = rnd(g, T, B, F), rnd(g, B, F, S)
    run = lambda x, dt, A, Bm, Cm, D, bias, h, **k: R.scan(  # noqa: E731
        x, dt, A, Bm, Cm, D, bias, h_in=h, softplus=softplus, lengths=ln, **k)
    out = run(*args.values(), gy=gy, gh_out=gh)
    grads = {"x": out["gx"], "dt": out["gdt"], "A": out["gA"], "B": out["gB"], "C": out["gC"], "D": out["gD"],
             "bias": out["gdt_bias"], "h": out["gh_in"]}
    compare(grads, differences(run, args, {"y": gy, "h_out": gh}, list(args)))


@pytest.mark.parametrize("parts", ["r z w_post scale w_pre", "r w_pre", "z w_post", "r z scale", "w_post w_pre"])
@pytest.mark.parametrize("lengths", [None, [2, 0]])
def test_norm_gradients(parts, lengths):
    g = gen(len(parts))
    T, B, F = 3, 2, 5
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    shapes = {"y": (T, B, F), "r": (T, B, F), "z": (T, B, F), "w_post": (F,), "scale": (F,), "w_pre": (F,)}
    args = {k: rnd(g, *s) for k, s in shapes.items() if k == "y" or k in parts.split()}
    g_r, g_u = rnd(g, T, B, F), rnd(g, T, B, F)

    def run(*values, **k):
        return R.norm(**dict(zip(args, values)), lengths=ln, **k)
    pre = "w_pre" in args
    out = run(*args.values(), g_r=g_r, g_u=g_u if pre else None)
    weights = {"r_new": g_r, **({"u": g_u} if pre else {})}
    names = {"y": "gy", "r": "gr", "z": "gz", "w_post": "gw_post", "scale": "gscale", "w_pre": "gw_pre"}
    compare({k: out[names[k]] for k in args}, differences(run, args, weights, list(args)))


def test_scan_closed_form():
    """Constant inputs: h_T = dxB (1 - a^T) / (1 - a), and a state alone decays as a^T."""
    T, d, a_rate = 7, 0.3, -0.5
    one = torch.ones(T, 1, 1, dtype=F64)
    out = R.scan(2 * one, d * one, torch.tensor([[a_rate]], dtype=F64), one[..., None], one[..., None], softplus=False)
    a = math.exp(d * a_rate)
    assert abs(float(out["y"][-1]) - 2 * d * (1 - a ** T) / (1 - a)) < 1e-14
    out = R.scan(0 * one, d * one, torch.tensor([[a_rate]], dtype=F64), one[..., None], one[..., None], softplus=False,
                 h_in=torch.full((1, 1, 1), 3.0, dtype=F64))
    assert abs(float(out["h_out"]) - 3 * a ** T) < 1e-14
