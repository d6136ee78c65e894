"""The row and time operators in float64 with numpy, from their definitions,
and bounds on the rounding errors a float32 implementation may make."""
import numpy as np
import torch

U32, U16, U8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4  # half a step, relative: fp32, bf16, e4m3
BLOCK = 128


def blocks(cols):
    return -(-cols // BLOCK)


def half(dtype):
    return {torch.float32: U32, torch.bfloat16: U16}[dtype]


def store8(x):
    """(values float64, scales float32) of rows x (float64) in e4m3."""
    x = np.asarray(x, np.float64)
    n, cols = x.shape
    out = np.zeros_like(x)
    scale = np.ones((n, blocks(cols)), np.float64)
    for b in range(blocks(cols)):
        blk = x[:, b * BLOCK:(b + 1) * BLOCK]
        a = np.max(np.where(np.isfinite(blk), np.abs(blk), 0.0), axis=1)
        m, e = np.frexp(a)  # a = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
        s = np.where(a > 0, np.exp2(np.maximum(e - 9 + (m > 0.875), -126.0)), 1.0)
        with np.errstate(invalid="ignore"):
            v = np.clip(blk / s[:, None], -448.0, 448.0)
            step = np.exp2(np.maximum(np.frexp(v)[1] - 1, -6) - 3.0)
            out[:, b * BLOCK:(b + 1) * BLOCK] = np.round(v / step) * step * s[:, None]
        scale[:, b] = s
    return out, scale


def values8(q, scale):
    """Values (float64) of codes q (uint8 tensor) and scales."""
    v = q.cpu().view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    return v * np.repeat(scale.cpu().numpy().astype(np.float64), BLOCK, axis=-1)[..., :v.shape[-1]]


def f64(t):
    return t.detach().cpu().float().numpy().astype(np.float64) if t.dtype != torch.float64 else t.cpu().numpy()


def rms_norm(x, res, w, eps):
    t = x + res if res is not None else x
    inv = 1 / np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)
    return t * inv * (w if w is not None else 1.0), t


def rms_norm_grad(t, w, dy, d_total, eps):
    """(dx, dw, bound on dx's fp32 error, sum of |dy u| that dw adds up)."""
    inv = 1 / np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)
    u = t * inv
    wdy = dy * w if w is not None else dy
    m = np.mean(u * wdy, axis=1, keepdims=True)
    dx = (wdy - u * m) * inv + (d_total if d_total is not None else 0.0)
    # fp32: a row sum of at most 8192 products adds at most 32 of them in one
    # thread and then joins at most 8 levels (40 half-steps, of the sum of the
    # magnitudes); inv takes half of that and 6 roundings of its own
    ma = np.mean(np.abs(u * wdy), axis=1, keepdims=True)
    slack = (np.abs(wdy) + np.abs(u) * ma) * inv * 90 * U32
    if d_total is not None:
        slack = slack + np.abs(dx) * U32 * 2
    return dx, np.sum(dy * u, axis=0), slack, np.sum(np.abs(dy * u), axis=0)


TINY = 2.0 ** -126


def gates(g):
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(g))
    small = e / (1 + e)
    small = np.where(small < TINY, 0.0, small)
    big = 1 / (1 + e)
    return np.where(g < 0, small, big), np.where(g < 0, big, small)


def term(w, v):
    with np.errstate(invalid="ignore"):
        return np.where(w == 0, 0.0, w * v)


def _gate_err(g):
    # exp of a product rounded once (|g| log2(e) half-steps in the exponent,
    # times ln 2), exp, add, reciprocal and product within a step each
    return (np.minimum(np.abs(g), 90.0) + 10) * U32


def scan(g, x, h0, starts):
    """(h, bound on h's fp32 error) for [T][rows][cols] float64 arrays.  The
    bound follows the recurrence's own roundings, twice: once for a step and
    once for steps joined in groups."""
    T = g.shape[0]
    f, z = gates(g)
    h = np.zeros_like(g)
    err = np.zeros_like(g)
    prev = h0 if h0 is not None else np.zeros(g.shape[1:])
    e = np.zeros(g.shape[1:])
    for t in range(T):
        ft = np.zeros_like(f[t]) if starts is not None and starts[t] else f[t]
        a, b = term(ft, prev), term(z[t], x[t])
        d = _gate_err(g[t])
        e = term(ft, e) + 2 * (d + 2 * U32) * (np.abs(np.where(ft == 0, 0, a)) + np.abs(np.where(z[t] == 0, 0, b)))
        prev = a + b
        h[t], err[t] = prev, e
    return h, err + 1e-37


def scan_grad(g, x, h, h0, starts, dh, dh_last):
    """dg, dx, dh0 and bounds on their fp32 errors (h as the forward stored it)."""
    T = g.shape[0]
    f, z = gates(g)
    dg, dx = np.zeros_like(g), np.zeros_like(g)
    edg, edx = np.zeros_like(g), np.zeros_like(g)
    D = dh_last if dh_last is not None else np.zeros(g.shape[1:])
    E = np.zeros(g.shape[1:])
    for t in range(T - 1, -1, -1):
        fresh = starts is not None and starts[t]
        if dh is not None:
            D = D + dh[t]
            E = E + 2 * U32 * np.abs(D)
        prev = np.zeros_like(D) if fresh else h[t - 1] if t else (h0 if h0 is not None else np.zeros_like(D))
        d = _gate_err(g[t])
        dx[t] = term(z[t], D)
        edx[t] = term(z[t], E) + np.abs(dx[t]) * (d + 2 * U32)
        fz = f[t] * z[t]
        dg[t] = term(fz, (prev - x[t]) * D)
        with np.errstate(invalid="ignore"):
            edg[t] = (term(fz, np.abs(prev - x[t]) * E) +
                      term(fz, (np.abs(prev) + np.abs(x[t])) * np.abs(D)) * 2 * U32 + np.abs(dg[t]) * (2 * d + 4 * U32))
        if fresh:
            D, E = np.zeros_like(D), np.zeros_like(E)
        else:
            D, E = term(f[t], D), term(f[t], E) + 2 * (d + 2 * U32) * np.abs(term(f[t], D))
    return dg, dx, D, edg + 1e-37, edx + 1e-37, E + 1e-37
