"""Float64 references of the layer norm, the causal convolution and the selective
scan, each with a bound on the fp32 kernels' error beside its value: the roundings
of every operation, carried on as the formula carries them.  U is half a step of
fp32; a sum of m terms, each of which is off by k half-steps of its own magnitude, is
off by at most (m + k) U times the sum of the magnitudes."""
import numpy as np
import torch

U = 2.0 ** -24
TINY = 1e-35  # results that leave fp32's normal numbers


def half(dtype) -> float:
    return {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]


def f64(t):
    return t.detach().cpu().double().numpy()


def near(what, got, want, bound, dtype=None):
    """got (tensor) within bound and the half-step of its type of want."""
    got = f64(got)
    h = half(dtype) if dtype is not None else U
    lim = bound + h * (np.abs(want) + bound) + TINY
    err = np.abs(got - want)
    ok = np.isfinite(got) & (err <= lim)
    assert np.all(ok), (what, float(np.nanmax(err / lim)), int((~ok).sum()), ok.size)


# ------------------------------------------------------------- layer norm ---
# A row's sums: at most 32 terms in a thread and 10 levels of joining.
SUM = 42


def layer_norm(x, res, w, b, eps):
    """y, t and y's bound.  The mean's rounding is taken off again by the mean of
    the deviations, so that only the rounding of t (of x + res) and those of the
    deviations remain."""
    t = x if res is None else x + res
    cols = t.shape[1]
    w = np.ones(cols) if w is None else w
    b = np.zeros(cols) if b is None else b
    mean = lambda v: v.mean(1, keepdims=True)
    d = t - mean(t)
    inv = 1 / np.sqrt(mean(d * d) + eps)
    u = d * inv
    te = 0.0 if res is None else np.abs(t) + mean(np.abs(t))
    m2 = SUM * U * mean(np.abs(t))  # what the rounded mean adds to a deviation before it goes
    centre = U * inv * (te + (SUM + 4) * (mean(np.abs(d)) + m2) + np.abs(d) + m2)
    # the variance: its sum, what is left of the rounded mean, the rounding of t
    rel = U * (SUM + 8 + inv ** 2 * (SUM * m2 * m2 + mean(np.abs(d) * te)))
    y = u * w + b
    return y, t, np.abs(w) * (centre + np.abs(u) * rel) + 3 * U * (np.abs(u * w) + np.abs(b))


def layer_norm_grad(t, w, dy, ds, eps):
    """(dx, dw, db) and their bounds; a column's sum over rows adds 8 rows in fp32,
    rounds the workgroup's partial and the result."""
    cols = t.shape[1]
    w = np.ones(cols) if w is None else w
    mean = lambda v: v.mean(1, keepdims=True)
    d = t - mean(t)
    inv = 1 / np.sqrt(mean(d * d) + eps)
    u, g = d * inv, dy * w
    m2 = SUM * U * mean(np.abs(t))
    eu = U * ((SUM + 6) * inv * (mean(np.abs(d)) + m2) + inv * m2 + (SUM + 12) * np.abs(u)) + U * SUM * np.abs(u) * inv ** 2 * m2 * m2
    mg, mu = mean(g), mean(g * u)
    emu = U * (SUM + 4) * mean(np.abs(g * u)) + mean(np.abs(g) * eu) + U * (SUM + 8) * mean(np.abs(g)) * inv * (mean(np.abs(d)) + m2)
    e0 = 5 * U * (np.abs(g) + np.abs(mg) + np.abs(u * mu)) + U * (SUM + 2) * mean(np.abs(g)) + eu * np.abs(mu) + np.abs(u) * emu
    core = (g - mg - u * mu) * inv
    dx = core if ds is None else core + ds
    ex = inv * e0 * 1.01 + np.abs(core) * U * (SUM + 12) + (0 if ds is None else U * np.abs(dx))
    dw, db = (dy * u).sum(0), dy.sum(0)
    ew = (np.abs(dy) * eu + 11 * U * np.abs(dy * u)).sum(0) + 2 * U * np.abs(dw)
    eb = 10 * U * np.abs(dy).sum(0) + 2 * U * np.abs(db)
    return dx, dw, db, ex, ew, eb


# ------------------------------------------------------ causal convolution ---
def _sig(v):
    return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def silu_bound(v, ev, y):
    """Of v sigmoid(v): its slope is at most 1.1, and the exponential's argument and
    value, the sum, the reciprocal and two products round."""
    return 1.1 * ev + np.abs(y) * U * (8 + 2 * np.abs(v))


def sees(T, W, starts):
    """[T][W]: whether step t sees the input k before it."""
    ok = np.ones((T, W), bool)
    for t in range(T):
        for k in range(1, W):
            if starts is not None and starts[max(0, t - k + 1):t + 1].any():
                ok[t, k] = False
    return ok


def _taps(x, w, past, starts):
    T, W = x.shape[0], w.shape[1]
    before = np.zeros((W - 1,) + x.shape[1:]) if past is None else past
    xp, ok = np.concatenate([before, x]), sees(T, W, starts)
    return xp, ok


def conv(x, w, b, past, starts, silu):
    """y, its bound, and past_out."""
    xp, ok = _taps(x, w, past, starts)
    T, W = x.shape[0], w.shape[1]
    b = np.zeros(x.shape[2]) if b is None else b
    v, mag = np.zeros_like(x), np.zeros_like(x)
    for t in range(T):
        v[t], mag[t] = b, np.abs(b)
        for k in range(W):
            if ok[t, k]:
                p = w[:, W - 1 - k] * xp[t + W - 1 - k]
                v[t] += p
                mag[t] += np.abs(p)
    ev = (W + 1) * U * mag
    out = np.zeros((W - 1,) + x.shape[1:])
    for j in range(W - 1):
        i = T + j  # of xp
        lag = W - 2 - j
        if starts is None or not starts[max(0, T - lag):T].any():
            out[j] = xp[i]
    if not silu:
        return v, ev, out
    y = v * _sig(v)
    return y, silu_bound(v, ev, y), out


def conv_grad(x, w, b, past, starts, silu, dy, d_past_out):
    """(dx, dw, db, d_past) and their bounds; 8 steps at most are added in fp32 to a
    column's sums."""
    xp, ok = _taps(x, w, past, starts)
    T, W = x.shape[0], w.shape[1]
    v, ev, _ = conv(x, w, b, past, starts, False)
    d, ed = dy, np.zeros_like(dy)
    if silu:
        s = _sig(v)
        slope = s * (1 + v * (1 - s))
        d = dy * slope
        ed = np.abs(dy) * (0.5 * ev + U * (12 + 4 * np.abs(v)) * s * (1 + np.abs(v) * (1 - s))) + 2 * U * np.abs(d)
    dxp, ex, mag = np.zeros_like(xp), np.zeros_like(xp), np.zeros_like(xp)
    dw, ew = np.zeros(w.shape), np.zeros(w.shape)
    for t in range(T):
        for k in range(W):
            if not ok[t, k]:
                continue
            i, c = t + W - 1 - k, w[:, W - 1 - k]
            dxp[i] += c * d[t]
            mag[i] += np.abs(c * d[t])
            ex[i] += np.abs(c) * ed[t]
            dw[:, W - 1 - k] += (d[t] * xp[i]).sum(0)
            ew[:, W - 1 - k] += (np.abs(xp[i]) * ed[t] + 10 * U * np.abs(d[t] * xp[i])).sum(0)
    if d_past_out is not None:
        for j in range(W - 1):
            lag = W - 2 - j
            if starts is None or not starts[max(0, T - lag):T].any():
                dxp[T + j] += d_past_out[j]
                mag[T + j] += np.abs(d_past_out[j])
    ex += (W + 2) * U * mag
    db, eb = d.sum((0, 1)), (ed + 10 * U * np.abs(d)).sum((0, 1))
    return dxp[W - 1:], dw, db, dxp[:W - 1], ex[W - 1:], ew + 2 * U * np.abs(dw), eb + 2 * U * np.abs(db), ex[:W - 1]


# --------------------------------------------------------- selective scan ---
def _steps(c):
    """delta and its bound: the sum's rounding moves it by the softplus's slope; in
    log(1 + e) the exponential is off by its argument's and its own rounding, and the
    series, quotient and sum by 8."""
    v = c["dt"] + (0 if c["bias"] is None else c["bias"])
    if not c["softplus"]:
        return v, v, U * np.abs(v)
    e = np.exp(-np.abs(v))
    delta = np.maximum(v, 0) + np.log1p(e)
    finite = np.where(np.isfinite(v), np.abs(v), 0)
    return v, delta, U * (_sig(v) * finite + (2 * finite + 4) * e + 8 * delta)


def ssm(c, chunk=0):
    """c: x, dt, A, B, C, D, bias, z, h0 (None: none), starts (None: none), softplus.
    Returns a dict with y, h (every state) and their bounds ey, eh, and what the
    backward takes of it.  chunk: steps over which deltas are summed where the time
    axis is cut."""
    x, A, B, Cn = c["x"], c["A"], c["B"], c["C"]
    T, R, D = x.shape
    n = A.shape[1]
    v, delta, ed = _steps(c)
    h = np.zeros((R, D, n)) if c["h0"] is None else c["h0"]
    e = np.zeros_like(h)
    H, E, O, EO, Ad, EA = [], [], [], [], [], []
    for t in range(T):
        if c["starts"] is not None and c["starts"][t]:
            h, e = np.zeros_like(h), np.zeros_like(h)
        arg = delta[t][:, :, None] * A
        a = np.exp(arg)
        ea = a * (np.abs(A) * ed[t][:, :, None] + (4 + chunk) * U * np.abs(arg) + 2 * U)
        u = delta[t] * np.where(delta[t] == 0, 0, x[t])
        eu = np.where(delta[t] == 0, 0, np.abs(x[t])) * ed[t] + U * np.abs(u)
        b = u[:, :, None] * np.where(u[:, :, None] == 0, 0, B[t][:, None, :])
        eb = np.where(u[:, :, None] == 0, 0, np.abs(B[t][:, None, :])) * eu[:, :, None] + U * np.abs(b)
        prev = h
        h = a * h + b
        e = (a + ea) * e + ea * np.abs(prev) + eb + 2 * U * np.abs(h) + (U * np.abs(a * prev) if chunk else 0)
        o = (h * Cn[t][:, None, :]).sum(2)
        eo = (np.abs(Cn[t][:, None, :]) * (e + (n + 3) * U * np.abs(h))).sum(2)
        if c["D"] is not None:
            o = o + c["D"] * x[t]
            eo = eo + 2 * U * np.abs(c["D"] * x[t]) + U * np.abs(o)
        for lst, val in ((H, h), (E, e), (O, o), (EO, eo), (Ad, a), (EA, ea)):
            lst.append(val)
    out = dict(v=v, delta=delta, ed=ed, h=H, eh=E, o=O, eo=EO, a=Ad, ea=EA, last=h, elast=e)
    o, eo = (np.stack(O), np.stack(EO)) if T else (np.zeros_like(x), np.zeros_like(x))
    if c["z"] is None:
        return dict(out, y=o, ey=eo)
    g = c["z"] * _sig(c["z"])
    y = o * g
    return dict(out, y=y, ey=np.abs(g) * eo + np.abs(y) * U * (9 + 2 * np.abs(c["z"])))


def ssm_grad(c, f, dy, dh_last, tiles=1, chunk=0):
    """Gradients and their bounds {name: (value, bound)} from f = ssm(c); block sums
    over 8 steps, 16 lanes and `tiles` parts of a row's columns in fp32."""
    x, A, B, Cn = c["x"], c["A"], c["B"], c["C"]
    T, R, D = x.shape
    n = A.shape[1]
    fr = c["starts"] if c["starts"] is not None else np.zeros(T, np.uint8)
    o, eo, dz, ez = dy, np.zeros_like(dy), None, None
    if c["z"] is not None:
        z, s = c["z"], _sig(c["z"])
        o = dy * z * s
        eo = np.abs(o) * U * (9 + 2 * np.abs(z))
        pre, epre = np.stack(f["o"]), np.stack(f["eo"])
        slope = s * (1 + z * (1 - s))
        dz = dy * pre * slope
        ez = np.abs(dy) * (epre * np.abs(slope) + np.abs(pre) * U * (14 + 4 * np.abs(z)) * s * (1 + np.abs(z) * (1 - s)))
    carry = np.zeros((R, D, n)) if dh_last is None else dh_last
    ec = np.zeros_like(carry)
    z3, z2 = np.zeros((T, R, n)), np.zeros((T, R, D))
    dx, ex, dd, edd = z2.copy(), z2.copy(), z2.copy(), z2.copy()
    dB, eB, dC, eC = z3.copy(), z3.copy(), z3.copy(), z3.copy()
    dA, eA = np.zeros((D, n)), np.zeros((D, n))
    for t in range(T - 1, -1, -1):
        Ct, Bt = Cn[t][:, None, :], B[t][:, None, :]
        ot, et = o[t][:, :, None], eo[t][:, :, None]
        dl, el = f["delta"][t], f["ed"][t]
        held = dl == 0
        xt = np.where(held, 0, x[t])
        u = dl * xt
        eu = np.abs(xt) * el + U * np.abs(u)
        Bs = np.where(held[:, :, None], 0, Bt)
        G = Ct * ot + carry
        eG = np.abs(Ct) * et + U * np.abs(Ct * ot) + ec + U * np.abs(G)
        sB = (G * Bs).sum(2)
        esB = (np.abs(Bs) * eG + (n + 2) * U * np.abs(G * Bs)).sum(2)
        dC[t] = (ot * f["h"][t]).sum(1)
        eC[t] = (np.abs(f["h"][t]) * et + np.abs(ot) * f["eh"][t] + (14 + tiles) * U * np.abs(ot * f["h"][t])).sum(1)
        dB[t] = (G * u[:, :, None]).sum(1)
        eB[t] = (np.abs(u[:, :, None]) * eG + np.abs(G) * eu[:, :, None] + (14 + tiles) * U * np.abs(G * u[:, :, None])).sum(1)
        dx[t] = sB * dl
        ex[t] = dl * esB + np.abs(sB) * el + 3 * U * np.abs(dx[t])
        if c["D"] is not None:
            dx[t] += c["D"] * o[t]
            ex[t] += np.abs(c["D"]) * eo[t] + 2 * U * np.abs(c["D"] * o[t]) + U * np.abs(dx[t])
        a, ea = f["a"][t], f["ea"][t]
        back = G * a
        eback = (a + ea) * eG + np.abs(G) * ea + U * np.abs(back) * 2
        if fr[t]:
            back, eback, prev, ep = np.zeros_like(back), np.zeros_like(back), 0.0, 0.0
        else:
            prev = f["h"][t - 1] if t else (np.zeros_like(back) if c["h0"] is None else c["h0"])
            ep = f["eh"][t - 1] if t else 0.0
        w = back * prev
        ew = np.abs(prev) * eback + np.abs(back) * ep + U * np.abs(w)
        q = (w * A).sum(2) + sB * xt
        eq = (np.abs(A) * ew + (n + 6) * U * np.abs(w * A)).sum(2) + np.abs(xt) * esB + 3 * U * (np.abs(sB * xt) + np.abs((w * A).sum(2)))
        if c["softplus"]:
            s = _sig(f["v"][t])
            fin = np.where(np.isfinite(f["v"][t]), np.abs(f["v"][t]), 0)
            eq = s * eq + np.abs(q) * U * (0.25 * fin + s * (6 + 2 * fin))
            q = q * s
        dd[t], edd[t] = q, eq
        dA += (w * dl[:, :, None]).sum(0)
        eA += (dl[:, :, None] * ew + np.abs(w) * el[:, :, None] + 10 * U * np.abs(w * dl[:, :, None])).sum(0)
        carry, ec = back, eback
    r = dict(dx=(dx, ex), ddt=(dd, edd), dB=(dB, eB), dC=(dC, eC), dA=(dA, eA + 2 * U * np.abs(dA)), dh0=(carry, ec),
             d_bias=(dd.sum((0, 1)), (edd + 10 * U * np.abs(dd)).sum((0, 1)) + 2 * U * np.abs(dd.sum((0, 1)))))
    if c["D"] is not None:
        dD = (o * x).sum((0, 1))
        r["dD"] = (dD, (np.abs(x) * eo + 10 * U * np.abs(o * x)).sum((0, 1)) + 2 * U * np.abs(dD))
    if dz is not None:
        r["dz"] = (dz, ez)
    return r
