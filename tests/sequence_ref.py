"""The sequence operators from their definitions, in 64 bits on the CPU, with gradients by
the chain rule written out, and bounds of what rounding can do to them.

Every function takes mag=True as well: then each product and sum is taken of absolute values,
which gives the sum of the magnitudes of the terms that a result is formed of.  A result
formed with n roundings of 32 bits on the way is off by at most n * 2^-24 of that, to first
order, and storing it in the I/O type by half a step (2^-8 relative for bf16: finfo.eps / 2).
"""
import torch

F64 = torch.float64
U32 = 2.0 ** -24


def tolerance(ref, mag, roundings, dtype, factors=1.0):
    """Largest error per value of a result with `roundings` roundings, then stored as dtype.
    Values under 2^-126 on the way may become 0: that moves a result by 2^-126 times what they
    are multiplied with, at most `factors`."""
    tol = roundings * U32 * mag
    if dtype == torch.bfloat16:
        tol = tol + torch.finfo(dtype).eps / 2 * (ref.abs() + tol)
    return tol + 2.0 ** -126 * max(8.0, factors)


def check(name, got, ref, mag, roundings, factors=1.0):
    assert got is not None and got.shape == ref.shape, name
    g = got.detach().cpu().to(F64)
    tol = tolerance(ref, mag, roundings, got.dtype, factors)
    bad = ~((g - ref).abs() <= tol)
    if bad.any():
        i = int((((g - ref).abs() - tol) * bad).nan_to_num(float("inf")).argmax())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} values off; value {i}: {g.flatten()[i]} "
                             f"for {ref.flatten()[i]}, tolerance {tol.flatten()[i]:.3g}")


def _abs(mag, *ts):
    return [None if t is None else t.detach().cpu().to(F64).abs() if mag else t.detach().cpu().to(F64) for t in ts]


def inside(T, B, lengths):
    if lengths is None:
        return torch.ones(T, B, 1, dtype=torch.bool)
    return (torch.arange(T)[:, None] < lengths.cpu())[..., None]


def steps(T, B, lengths):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def conv(x, w, bias, *, act="silu", state=None, lengths=None, gy=None, gstate_out=None, mag=False):
    """y, state_out and, with gy: gx, gw, gb, gstate."""
    T, B, F = x.shape
    W = w.shape[1]
    xa, wa, ba, sa, ga, gsa = _abs(mag, x, w, bias, state, gy, gstate_out)
    xt, wt, bt, st = _abs(False, x, w, bias, state)
    m = inside(T, B, lengths)
    ln = steps(T, B, lengths)

    def padded(v, s):
        past = torch.zeros(W - 1, B, F, dtype=F64) if s is None else s
        return torch.cat([past, torch.where(m, v, torch.zeros((), dtype=F64))])

    def drive(p, ww, bb):
        u = torch.zeros(T, B, F, dtype=F64) + (0 if bb is None else bb)
        for j in range(W):
            u = u + ww[:, j] * p[j:j + T]
        return u

    xs, true = padded(xa, sa), padded(xt, st)
    u, u0 = drive(xs, wa, ba), drive(true, wt, bt)
    sig = torch.sigmoid(u0)
    y = u * sig if act else u
    if mag and act:
        y = u * sig * (1 + u)            # the error of u reaches the sigmoid too
    out = {"y": torch.where(m, y, torch.zeros((), dtype=F64)),
           "state_out": torch.stack([true[ln[b]:ln[b] + W - 1, b] for b in range(B)], 1)}
    if gy is None:
        return out
    slope = torch.ones_like(u)
    if act:
        slope = sig * (1 + u0 * (1 - sig)) if not mag else sig * (1 + u) * (1 + u)
    gu = torch.where(m, ga * slope, torch.zeros((), dtype=F64))
    gxs = torch.zeros(T + W - 1, B, F, dtype=F64)
    gw = torch.zeros(F, W, dtype=F64)
    for j in range(W):
        gxs[j:j + T] += wa[:, j] * gu
        gw[:, j] = (gu * xs[j:j + T]).sum((0, 1))
    if gsa is not None:
        for b in range(B):
            gxs[ln[b]:ln[b] + W - 1, b] += gsa[:, b]
    out.update(gx=torch.where(m, gxs[W - 1:], torch.zeros((), dtype=F64)), gw=gw, gb=gu.sum((0, 1)), gstate=gxs[:W - 1])
    return out


def scan(x, dt, A, Bm, Cm, D=None, dt_bias=None, *, softplus=True, h_in=None, lengths=None, gy=None, gh_out=None,
         mag=False):
    """y, h_out and, with gy, the gradients g* of every input."""
    T, B, F = x.shape
    G, S = Bm.shape[2:]
    m = inside(T, B, lengths)
    zero = torch.zeros((), dtype=F64)
    xa, Ba, Ca, Da, ha, gya, gha = _abs(mag, x, Bm, Cm, D, h_in, gy, gh_out)
    dtt, At, bt = _abs(False, dt, A, dt_bias)
    xa = torch.where(m, xa, zero)
    v = torch.where(m, dtt, zero) + (0 if bt is None else bt)
    d = torch.where(m, torch.logaddexp(v, zero) if softplus else v, zero)
    dm = d.abs() if mag else d
    per = F // G
    Bf, Cf = (torch.where(m[..., None], t.repeat_interleave(per, 2), zero) for t in (Ba, Ca))
    h = torch.zeros(B, F, S, dtype=F64) if ha is None else ha
    through_d = lambda v: 0.0 if Da is None else Da * v  # noqa: E731
    hs, decays = [h], []
    for t in range(T):
        decays.append(torch.exp(d[t][..., None] * At))
        hs.append(decays[t] * hs[-1] + (dm[t] * xa[t])[..., None] * Bf[t])
    y = torch.stack([(hs[t + 1] * Cf[t]).sum(-1) + through_d(xa[t]) for t in range(T)]) if T else xa
    out = {"y": torch.where(m, y, zero), "h_out": hs[-1]}
    if gy is None:
        return out
    gya = torch.where(m, gya, zero)
    rate = At.abs() if mag else At
    e = torch.zeros(B, F, S, dtype=F64) if gha is None else gha
    g = {"gx": torch.zeros(T, B, F, dtype=F64), "gdt": torch.zeros(T, B, F, dtype=F64), "gA": torch.zeros(F, S, dtype=F64)}
    gBf, gCf = torch.zeros(T, B, F, S, dtype=F64), torch.zeros(T, B, F, S, dtype=F64)
    for t in range(T - 1, -1, -1):
        dh = gya[t][..., None] * Cf[t] + e
        q = dh * decays[t] * hs[t]
        gCf[t] = gya[t][..., None] * hs[t + 1]
        gBf[t] = dh * (dm[t] * xa[t])[..., None]
        through = (dh * Bf[t]).sum(-1)
        g["gx"][t] = dm[t] * through + through_d(gya[t])
        gd = (q * rate).sum(-1) + xa[t] * through
        g["gdt"][t] = gd * (torch.sigmoid(v[t]) if softplus else 1.0)
        g["gA"] += (q * dm[t][..., None]).sum(0)
        e = decays[t] * dh
    g["gx"], g["gdt"] = torch.where(m, g["gx"], zero), torch.where(m, g["gdt"], zero)
    g.update(gB=gBf.view(T, B, G, per, S).sum(3), gC=gCf.view(T, B, G, per, S).sum(3), gD=(gya * xa).sum((0, 1)),
             gdt_bias=g["gdt"].sum((0, 1)), gh_in=e)
    return {**out, **g}


def scan_roundings(T, B, F, S):
    """A step's decay is off by 2 roundings and by those of its exponent (at most 8, of a
    magnitude x whose effect x e^-x stays under 1), a state by 3 more per step: 13 T for the
    state and as much for its gradient; then sums over states, features, sequences and steps."""
    return 26 * T + S + F + 2 * T * B + 64


def norm(y, r=None, z=None, w_post=None, scale=None, w_pre=None, *, eps=1e-5, lengths=None, g_r=None, g_u=None,
         mag=False):
    T, B, F = y.shape
    zero = torch.zeros((), dtype=F64)
    m = inside(T, B, lengths)
    ya, ra, za, wa, sa, pa, ga, gua = _abs(mag, y, r, z, w_post, scale, w_pre, g_r, g_u)
    yt, rt, zt, wt, st, pt = _abs(False, y, r, z, w_post, scale, w_pre)
    keep = lambda t: None if t is None else torch.where(m, t, zero)  # noqa: E731
    ya, ra, za, yt, rt, zt, ga, gua = (keep(t) for t in (ya, ra, za, yt, rt, zt, ga, gua))
    ones = torch.ones(F, dtype=F64)

    def run(yy, rr, zz, ww, ss, k1=None):
        g = yy if zz is None else yy * zz * torch.sigmoid(zt)
        if k1 is None:
            k1 = torch.rsqrt((g * g).mean(-1, keepdim=True) + eps) if w_post is not None else torch.ones(T, B, 1, dtype=F64)
        n = g * k1 * (ones if ww is None else ww)
        return g, k1, n, (0 if rr is None else rr) + (ones if ss is None else ss) * n

    g0, k1, n0, r0 = run(yt, rt, zt, wt, st)
    k2 = torch.rsqrt((r0 * r0).mean(-1, keepdim=True) + eps)
    g, _, n, rn = run(ya, ra, za, wa, sa, k1) if mag else (g0, k1, n0, r0)
    if mag and z is not None:
        g = g * (1 + za)
        n, rn = n * (1 + za), rn * (1 + za)
    out = {"r_new": keep(rn)}
    # a relative error of the mean square (2 roundings per term) moves k by half of that; where
    # r' cancels, its own error moves k2 by at most that error over the root mean square
    grow = (rn * rn).mean(-1, keepdim=True).sqrt() * k2 if mag else 0.0
    if w_pre is not None:
        out["u"] = keep(rn * k2 * pa * (1 + grow))
    if g_r is None and g_u is None:
        return out
    gr = torch.zeros(T, B, F, dtype=F64) if ga is None else ga.clone()
    if g_u is not None:
        rk, t = rn * k2, gua * pa
        c = (t * rk).mean(-1, keepdim=True)
        gr = gr + (k2 * (t + rk * c) * (1 + grow) ** 2 if mag else k2 * (t - rk * c))
        out["gw_pre"] = keep(gua * rk * (1 + grow)).sum((0, 1))
    gn = gr * (ones if sa is None else sa)
    out["gr"] = keep(gr)
    out["gscale"] = keep(gr * n).sum((0, 1))
    if w_post is not None:
        hat, t = g * k1, gn * wa
        c = (t * hat).mean(-1, keepdim=True)
        grow1 = (hat * hat).mean(-1, keepdim=True).sqrt() if mag else 0.0
        gg = k1 * (t + hat * c) * (1 + grow1) ** 2 if mag else k1 * (t - hat * c)
        out["gw_post"] = keep(gn * hat).sum((0, 1))
    else:
        gg = gn
    if z is None:
        out["gy"] = keep(gg)
    else:
        s = torch.sigmoid(zt)
        out["gy"] = keep(gg * za * s * ((1 + za) if mag else 1))
        out["gz"] = keep(gg * ya * (s * (1 + za) ** 2 if mag else s * (1 + zt * (1 - s))))
    return out


def norm_roundings(T, B, F):
    return 4 * F + 2 * T * B + 64
