"""The root-mean-square norm with the residual's addition and its backward
(mgn_rms_norm, mgn_rms_norm_grad) against float64.

Tolerances (half-steps of 2^-24): a row's sum of squares adds at most 32
products in one thread and joins at most 8 levels, so its relative error is at
most 41, half of that after the square root, and eps, the mean, the root, the
reciprocal, two products and the residual's addition round once each: 32.  Then
the half-step of the type that is written."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref
from paper_2307_13592_amd.runner import LatentCache, RmsNorm

pytestmark = pytest.mark.gpu
EPS = 1e-6
SHAPES = [(1, 1), (3, 5), (2, 7), (1, 16), (3, 6), (900, 5), (333, 11), (64, 8), (40, 16), (9, 9), (33, 64), (501, 17), (77, 21), (64, 32), (33, 48), (1885, 77), (130, 128), (65, 129), (7, 200), (1001, 256), (5, 257), (6, 1000),
          (3, 1024), (4, 1025), (2, 8192), (3, 8191)]


def _inputs(n, cols, dtype, seed=0):
    r = np.random.default_rng([seed, n, cols])
    size = np.exp(3 * r.standard_normal((n, 1)))
    size[n // 2] = 0 if n > 2 else 1  # a row of zeros
    t = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    x = t(r.standard_normal((n, cols)) * size).to(dtype)
    res = t(r.standard_normal((n, cols)) * size).to(dtype)
    return x, res, t(1 + 0.2 * r.standard_normal(cols)), t(r.standard_normal((n, cols))).to(dtype)


def _near(got, want, bound):
    err = np.abs(ref.f64(got) - want)
    assert np.all(err <= bound), (float(np.max(err - bound)), float(np.max(err / (bound + 1e-300))))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", SHAPES)
def test_norm(n, cols, dtype):
    print(f"[rms] {n} x {cols} {dtype}", flush=True)
    x, res, w, _ = _inputs(n, cols, dtype)
    for with_res in (False, True):
        for weight in (w, None):
            rr = res if with_res else None
            y64, t64 = ref.rms_norm(ref.f64(x), ref.f64(rr) if with_res else None,
                                    ref.f64(weight) if weight is not None else None, EPS)
            for out in (torch.float32, torch.bfloat16):
                y = torch.empty(n, cols, dtype=out, device="cuda")
                total = torch.empty_like(x) if with_res else None
                mgn.mgn_rms_norm(x, weight, y, res=rr, total=total, eps=EPS)
                _near(y, y64, np.abs(y64) * (32 * ref.U32 + (ref.U16 if out == torch.bfloat16 else 0)) + 1e-37)
                if with_res:
                    _near(total, t64, np.abs(t64) * (ref.U32 + (ref.U16 if dtype == torch.bfloat16 else 0)) + 1e-37)
            # 8-bit rows: half a step of the value, or of the smallest step 2^-9 of its scale
            c = LatentCache(n + 2, cols)
            s64 = np.repeat(ref.store8(y64)[1], 128, axis=1)[:, :cols]
            mgn.mgn_rms_norm(x, weight, c.q[1:n + 1], res=rr, y_scale=c.scale[1:n + 1], eps=EPS)
            # (the fp32 y may fall on the other side of a power of two: one scale up)
            _near(torch.as_tensor(ref.values8(c.q[1:n + 1], c.scale[1:n + 1])), y64,
                  np.abs(y64) * (ref.U8 + 34 * ref.U32) + 2 * s64 * 2.0 ** -10)
            assert not c.q[0].any() and not c.q[n + 1].any() and float(c.scale[0, 0]) == 1.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", SHAPES + [(5003, 64), (40001, 128), (2500, 256), (2051, 1000)])
def test_grad(n, cols, dtype):
    print(f"[rms grad] {n} x {cols} {dtype}", flush=True)
    t, ds, w, dy = _inputs(n, cols, dtype, seed=1)
    for with_ds in (False, True):
        for weight in (w, None):
            dx = torch.empty_like(t)
            dw = torch.full((cols,), 2.0, device="cuda")
            mgn.mgn_rms_norm_grad(t, weight, dy, dx, dw, d_total=ds if with_ds else None, eps=EPS)
            dx64, dw64, slack, mag = ref.rms_norm_grad(ref.f64(t), ref.f64(weight) if weight is not None else None,
                                                       ref.f64(dy), ref.f64(ds) if with_ds else None, EPS)
            _near(dx, dx64, slack + np.abs(dx64) * (ref.half(dtype) + ref.U32) + 1e-37)
            # a column's sum: u within 32, one product, at most n / 1024 + 1 rows
            # in one thread (of 1024 workgroups a row each), at most 128 row groups
            # of a workgroup, then fp64
            bound = mag * (36 + n / 1024 + 1 + 128) * ref.U32 + np.abs(dw64) * ref.U32 + 1e-37
            _near(dw, dw64, bound)
            dw2 = dw.clone()
            mgn.mgn_rms_norm_grad(t, weight, dy, dx, dw2, d_total=ds if with_ds else None, accumulate=True, eps=EPS)
            _near(dw2, 2 * dw64, 2 * bound + np.abs(dw64) * 4 * ref.U32)
            again, dxa = torch.empty_like(dw), torch.empty_like(dx)
            mgn.mgn_rms_norm_grad(t, weight, dy, dxa, again, d_total=ds if with_ds else None, eps=EPS)
            assert torch.equal(again, dw) and torch.equal(dxa, dx)  # the same bits
    only = torch.empty_like(t)
    mgn.mgn_rms_norm_grad(t, None, dy, only, d_total=ds, eps=EPS)
    assert torch.equal(only, dx)


def test_grad_against_differences():
    """Central differences of the float64 forward."""
    n, cols, step = 3, 12, 1e-6
    x, res, w, c = (ref.f64(a) for a in _inputs(n, cols, torch.float32, seed=2))
    x[1] += 0.3  # (no row of zeros here: its curvature is 1 / eps)
    t = (x + res).astype(np.float32).astype(np.float64)
    loss = lambda t, w: float(np.sum(ref.rms_norm(t, None, w, EPS)[0] * c))
    num = np.zeros_like(t)
    for i in np.ndindex(t.shape):
        d = np.zeros_like(t)
        d[i] = step
        num[i] = (loss(t + d, w) - loss(t - d, w)) / (2 * step)
    numw = np.array([(loss(t, w + step * e) - loss(t, w - step * e)) / (2 * step) for e in np.eye(cols)])
    dev = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    dx, dw = torch.empty(n, cols, device="cuda"), torch.empty(cols, device="cuda")
    mgn.mgn_rms_norm_grad(dev(t), dev(w), dev(c), dx, dw, eps=EPS)
    assert np.allclose(ref.f64(dx), num, rtol=1e-5, atol=1e-5 * np.abs(num).max())
    assert np.allclose(ref.f64(dw), numw, rtol=1e-5, atol=1e-5 * np.abs(numw).max())


@pytest.mark.parametrize("cols", [64, 128, 77, 1500])
def test_rows_that_hold_nan_or_infinity_stay_alone(cols):
    x, res, w, dy = _inputs(9, cols, torch.float32, seed=3)
    y0, t0 = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_rms_norm(x, w, y0, res=res, total=t0, eps=EPS)
    x2 = x.clone()
    x2[2, cols - 1], x2[5, 0] = float("nan"), float("inf")
    y, t = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_rms_norm(x2, w, y, res=res, total=t, eps=EPS)
    keep = [0, 1, 3, 4, 6, 7, 8]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(t[keep], t0[keep])
    assert bool(y[2].isnan().all()) and bool(y[5, 0].isnan())
    assert bool(t[2, cols - 1].isnan()) and bool(t[2, :cols - 1].isfinite().all())
    c = LatentCache(9, cols)
    mgn.mgn_rms_norm(x2, w, c.q, res=res, y_scale=c.scale, eps=EPS)
    v = ref.values8(c.q, c.scale)
    assert np.isnan(v[2]).all() and np.isfinite(v[keep]).all()
    assert bool((c.scale[2] == 1).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [128, 77, 2000, 5, 1501])
def test_in_place_and_unaligned(cols, dtype):
    """Results on the arrays they may stand on (the same bits), and arrays
    aligned to their type only."""
    n = 37
    x, res, w, dy = _inputs(n, cols, dtype, seed=4)
    y, t = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_rms_norm(x, w, y, res=res, total=t, eps=EPS)
    a, b = x.clone(), res.clone()
    mgn.mgn_rms_norm(a, w, b, res=b, total=a, eps=EPS)
    assert torch.equal(a, t) and torch.equal(b, y)
    a, b = x.clone(), res.clone()
    mgn.mgn_rms_norm(a, w, a, res=b, total=b, eps=EPS)
    assert torch.equal(a, y) and torch.equal(b, t)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    mgn.mgn_rms_norm_grad(t, w, dy, dx, dw, d_total=res, eps=EPS)
    for k in range(3):
        arr = [t.clone(), dy.clone(), res.clone()]
        dw2 = torch.empty_like(dw)
        mgn.mgn_rms_norm_grad(arr[0], w, arr[1], arr[k], dw2, d_total=arr[2], eps=EPS)
        assert torch.equal(arr[k], dx) and torch.equal(dw2, dw)

    def at(v, o):
        return torch.full((v.numel() + 8,), 5.0, dtype=v.dtype, device="cuda")[o:o + v.numel()].view(v.shape).copy_(v)

    # arrays that only their type aligns are read by other threads, so their sums
    # add in another order: within the same bounds of the float64 values
    y64, t64 = ref.rms_norm(ref.f64(x), ref.f64(res), ref.f64(w), EPS)
    dx64, dw64, slack, mag = ref.rms_norm_grad(ref.f64(t), ref.f64(w), ref.f64(dy), ref.f64(res), EPS)
    h = ref.half(dtype)
    def kept(v, o):  # what lies around an array of at()
        all_ = v.new_empty(0).set_(v.untyped_storage(), 0, (v.numel() + 8,))
        return bool((all_[:o] == 5).all()) and bool((all_[o + v.numel():] == 5).all())

    for o in (1, 2, 3):
        y2, t2, wo = at(y * 0, o), at(t * 0, (o + 1) % 4), at(w, o)
        mgn.mgn_rms_norm(at(x, o), wo, y2, res=at(res, 0), total=t2, eps=EPS)
        _near(y2, y64, np.abs(y64) * (32 * ref.U32 + h) + 1e-37)
        assert torch.equal(t2, t) and kept(y2, o) and kept(t2, (o + 1) % 4)
        d2 = at(dx * 0, o)
        mgn.mgn_rms_norm_grad(at(t, o), wo, at(dy, 0), d2, dw2, d_total=at(res, 2), eps=EPS)
        _near(d2, dx64, slack + np.abs(dx64) * (h + ref.U32) + 1e-37)
        assert kept(d2, o)
        _near(dw2, dw64, mag * (36 + n / 1024 + 1 + 128) * ref.U32 + np.abs(dw64) * ref.U32 + 1e-37)


def test_no_rows():
    e = torch.empty(0, 128, device="cuda")
    w = torch.ones(128, device="cuda")
    mgn.mgn_rms_norm(e, w, e)
    dw = torch.full((128,), 3.0, device="cuda")
    mgn.mgn_rms_norm_grad(e, w, e, e, dw, accumulate=True)
    assert bool((dw == 3).all())
    mgn.mgn_rms_norm_grad(e, w, e, e, dw)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", [(3_000_001, 64), (700_001, 77), (40_001, 1100), (33_001, 4100), (33_001, 4099)])
def test_more_rows_than_a_grid(n, cols, dtype):
    """Rows beyond the launched workgroups' first turn, and more bytes than the
    caches hold; rows of one wave's lanes, of 256 and of 1024 threads."""
    print(f"[rms] {n} x {cols} {dtype}", flush=True)
    h = ref.half(dtype) + 2 * ref.U32
    x = torch.randn(n, cols, device="cuda").to(dtype)
    y = torch.empty_like(x)
    mgn.mgn_rms_norm(x, None, y, eps=EPS)
    inv = torch.rsqrt((x.double() ** 2).mean(1, keepdim=True) + EPS)
    u = x.double() * inv
    assert float(((y.double() - u).abs() - (32 * ref.U32 + h) * u.abs()).max()) <= 1e-37
    nz = RmsNorm(cols)
    dx = nz.grad(x, y)
    g = y.double()
    m = (u * g).mean(1, keepdim=True)
    want = (g - u * m) * inv
    slack = (g.abs() + u.abs() * (u * g).abs().mean(1, keepdim=True)) * inv * 92 * ref.U32
    assert float(((dx.double() - want).abs() - slack - h * want.abs()).max()) <= 1e-37
    dw = (g * u).sum(0)  # (all terms positive)
    assert bool(((nz.d_weight.double() - dw).abs() <= dw.abs() * (36 + n / 1024 + 1 + 128 + 1) * ref.U32).all())


def test_streams_and_captured_replays():
    x, res, w, dy = _inputs(5000, 128, torch.bfloat16, seed=6)
    nz = RmsNorm(128)
    nz.weight.copy_(w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y0, t0 = nz.apply(x, res)
    dx0 = nz.grad(t0, dy, res)
    dw0 = nz.d_weight.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y1, t1 = nz.apply(x, res, stream=side.cuda_stream)
        dx1 = nz.grad(t1, dy, res, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y0, y1) and torch.equal(dx0, dx1) and torch.equal(nz.d_weight, dw0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, t = nz.apply(x, res)
        dx = nz.grad(t, dy, res)
    for k in range(4):
        a, b, _, c = _inputs(5000, 128, torch.bfloat16, seed=10 + k)
        x.copy_(a), res.copy_(b), dy.copy_(c)
        g.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y, t, dx, nz.d_weight)]
        ye, te = nz.apply(x, res)
        want = (ye, te, nz.grad(te, dy, res), nz.d_weight)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
