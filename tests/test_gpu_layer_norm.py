"""The layer norm with the residual's addition and its backward (mgn_layer_norm,
mgn_layer_norm_grad) against float64, within the bounds of memory_ref."""
import numpy as np
import pytest
import torch

import memory_ref as ref
import paper_2307_13592_amd as mgn
import row_ref
from paper_2307_13592_amd.runner import LatentCache, LayerNorm

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(1, 1), (3, 5), (2, 7), (1, 16), (900, 5), (64, 8), (40, 16), (33, 64), (501, 17), (64, 32), (1885, 77),
          (130, 128), (65, 129), (7, 200), (1001, 256), (5, 257), (6, 1000), (3, 1024), (4, 1025), (2, 8192), (3, 8191)]


def _inputs(n, cols, dtype, seed=0, offset=2.0):
    r = np.random.default_rng([seed, n, cols])
    size = np.exp(2 * r.standard_normal((n, 1)))
    size[n // 2] = 0 if n > 2 else 1  # a row of zeros
    t = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    x = t((r.standard_normal((n, cols)) + offset * r.standard_normal((n, 1))) * size).to(dtype)
    return (x, t(r.standard_normal((n, cols)) * size).to(dtype), t(1 + 0.2 * r.standard_normal(cols)),
            t(0.3 * r.standard_normal(cols)), t(r.standard_normal((n, cols))).to(dtype))


def _o(a, on=True):
    return ref.f64(a) if on and a is not None else None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", SHAPES)
def test_norm(n, cols, dtype):
    print(f"[layer] {n} x {cols} {dtype}", flush=True)
    x, res, w, b, _ = _inputs(n, cols, dtype)
    for r in (None, res):
        for weight, bias in ((w, b), (None, None), (w, None)):
            y64, t64, e = ref.layer_norm(ref.f64(x), _o(r), _o(weight), _o(bias), EPS)
            for out in (torch.float32, torch.bfloat16):
                y = torch.empty(n, cols, dtype=out, device="cuda")
                total = torch.empty_like(x) if r is not None else None
                mgn.mgn_layer_norm(x, weight, bias, y, res=r, total=total, eps=EPS)
                ref.near("y", y, y64, e, out)
                if r is not None:
                    ref.near("total", total, t64, ref.U * np.abs(t64), dtype)
            # 8-bit rows: the scale's smallest step is 2^-9 of it, and may be one scale up
            c = LatentCache(n + 2, cols)
            s64 = np.repeat(row_ref.store8(y64)[1], 128, axis=1)[:, :cols]
            mgn.mgn_layer_norm(x, weight, bias, c.q[1:n + 1], res=r, y_scale=c.scale[1:n + 1], eps=EPS)
            got = row_ref.values8(c.q[1:n + 1], c.scale[1:n + 1])
            assert np.all(np.abs(got - y64) <= e + (np.abs(y64) + e) * 2.0 ** -4 + 2 * s64 * 2.0 ** -10)
            assert not c.q[0].any() and not c.q[n + 1].any() and float(c.scale[0, 0]) == 1.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", SHAPES + [(5003, 64), (40001, 128), (2051, 1000)])
def test_grad(n, cols, dtype):
    print(f"[layer grad] {n} x {cols} {dtype}", flush=True)
    t, ds, w, _, dy = _inputs(n, cols, dtype, seed=1)
    for d_total in (None, ds):
        for weight in (w, None):
            dx = torch.empty_like(t)
            dw, db = torch.full((cols,), 2.0, device="cuda"), torch.full((cols,), 3.0, device="cuda")
            mgn.mgn_layer_norm_grad(t, weight, dy, dx, dw, db, d_total=d_total, eps=EPS)
            dx64, dw64, db64, ex, ew, eb = ref.layer_norm_grad(ref.f64(t), _o(weight), ref.f64(dy), _o(d_total), EPS)
            ref.near("dx", dx, dx64, ex, dtype)
            ref.near("dw", dw, dw64, ew)
            ref.near("db", db, db64, eb)
            dw2, db2, dxa = dw.clone(), db.clone(), torch.empty_like(dx)
            mgn.mgn_layer_norm_grad(t, weight, dy, dxa, dw2, db2, d_total=d_total, accumulate=True, eps=EPS)
            ref.near("dw + dw", dw2, 2 * dw64, 2 * ew)
            ref.near("db + db", db2, 2 * db64, 2 * eb)
            again = torch.empty_like(dw)
            mgn.mgn_layer_norm_grad(t, weight, dy, dxa, again, None, d_total=d_total, eps=EPS)
            assert torch.equal(again, dw) and torch.equal(dxa, dx)  # the same bits, with db or without
            mgn.mgn_layer_norm_grad(t, weight, dy, dxa, None, again, d_total=d_total, eps=EPS)
            assert torch.equal(again, db) and torch.equal(dxa, dx)
    only = torch.empty_like(t)
    mgn.mgn_layer_norm_grad(t, None, dy, only, d_total=ds, eps=EPS)
    assert torch.equal(only, dx)


def test_grad_against_differences():
    """Central differences of the float64 forward."""
    n, cols, step = 3, 12, 1e-6
    x, _, w, b, c = (ref.f64(a) for a in _inputs(n, cols, torch.float32, seed=2))
    x[1] = np.linspace(-1, 2, cols).astype(np.float32)  # (no row of zeros here: its curvature is 1 / eps)
    loss = lambda x, w, b: float(np.sum(ref.layer_norm(x, None, w, b, EPS)[0] * c))
    diff = lambda f, a: np.array([(f(a + d) - f(a - d)) / (2 * step) for d in step * np.eye(a.size).reshape((-1,) + a.shape)])
    dev = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    dx, dw, db = torch.empty(n, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    mgn.mgn_layer_norm_grad(dev(x), dev(w), dev(c), dx, dw, db, eps=EPS)
    for got, f, a in ((dx, lambda v: loss(v, w, b), x), (dw, lambda v: loss(x, v, b), w), (db, lambda v: loss(x, w, v), b)):
        num = diff(f, a).reshape(a.shape)
        assert np.allclose(ref.f64(got), num, rtol=1e-5, atol=1e-5 * np.abs(num).max())


@pytest.mark.parametrize("cols", [64, 77, 1000, 3001])
def test_offsets_and_equal_values(cols):
    """An offset far above the deviations costs none of their digits; a row of equal
    values is its bias."""
    r = np.random.default_rng(cols)
    x = torch.as_tensor((4096.0 + r.integers(-64, 65, (5, cols)) / 64).astype(np.float32)).cuda()  # exact in fp32
    w, b = torch.ones(cols, device="cuda"), torch.as_tensor(r.standard_normal(cols).astype(np.float32)).cuda()
    x[2] = 1000.1
    y = torch.empty_like(x)
    mgn.mgn_layer_norm(x, w, b, y, eps=EPS)
    y64, _, e = ref.layer_norm(ref.f64(x), None, ref.f64(w), ref.f64(b), EPS)
    assert np.abs(ref.f64(y) - y64).max() <= 2e-5  # (the mean's own rounding would be 4096 * 2^-24 / deviation: 4e-4)
    assert np.abs(ref.f64(y[2]) - ref.f64(b)).max() <= 1e-6


@pytest.mark.parametrize("cols", [64, 128, 77, 1500])
def test_rows_that_are_not_finite_or_pass_the_range(cols):
    x, res, w, b, dy = _inputs(9, cols, torch.float32, seed=3)
    y0, t0 = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_layer_norm(x, w, b, y0, res=res, total=t0, eps=EPS)
    x2 = x.clone()
    x2[2, cols - 1], x2[5, 0] = float("nan"), float("inf")
    x2[7] = 3e38 * (torch.arange(cols, device="cuda") % 2 * 2 - 1)
    y, t = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_layer_norm(x2, w, b, y, res=res, total=t, eps=EPS)
    keep = [0, 1, 3, 4, 6, 8]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(t[keep], t0[keep])
    assert bool(y[2].isnan().all()) and bool(y[5].isnan().all())
    assert bool(t[2, :cols - 1].isfinite().all()) and torch.equal(y[7], b)
    for bad in (2, 5):
        t[bad] = 0.5
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    mgn.mgn_layer_norm_grad(t, w, dy, dx, dw, db, d_total=res, eps=EPS)
    assert torch.equal(dx[7], res[7]) and bool(dw.isfinite().all()) and bool(db.isfinite().all())
    t[2, 3] = float("nan")
    mgn.mgn_layer_norm_grad(t, w, dy, dx, None, None, d_total=res, eps=EPS)
    assert bool(dx[2].isnan().all()) and bool(dx[[0, 1, 3, 4, 5, 6, 7, 8]].isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [128, 77, 2000, 5, 1501])
def test_in_place_and_unaligned(cols, dtype):
    n = 37
    x, res, w, b, dy = _inputs(n, cols, dtype, seed=4)
    y, t = torch.empty_like(x), torch.empty_like(x)
    mgn.mgn_layer_norm(x, w, b, y, res=res, total=t, eps=EPS)
    p, q = x.clone(), res.clone()
    mgn.mgn_layer_norm(p, w, b, q, res=q, total=p, eps=EPS)
    assert torch.equal(p, t) and torch.equal(q, y)
    p, q = x.clone(), res.clone()
    mgn.mgn_layer_norm(p, w, b, p, res=q, total=q, eps=EPS)
    assert torch.equal(p, y) and torch.equal(q, t)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    mgn.mgn_layer_norm_grad(t, w, dy, dx, dw, db, d_total=res, eps=EPS)
    for k in range(3):
        arr = [t.clone(), dy.clone(), res.clone()]
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        mgn.mgn_layer_norm_grad(arr[0], w, arr[1], arr[k], dw2, db2, d_total=arr[2], eps=EPS)
        assert torch.equal(arr[k], dx) and torch.equal(dw2, dw) and torch.equal(db2, db)

    def at(v, o):
        return torch.full((v.numel() + 8,), 5.0, dtype=v.dtype, device="cuda")[o:o + v.numel()].view(v.shape).copy_(v)

    def kept(v, o):
        all_ = v.new_empty(0).set_(v.untyped_storage(), 0, (v.numel() + 8,))
        return bool((all_[:o] == 5).all()) and bool((all_[o + v.numel():] == 5).all())

    y64, _, e = ref.layer_norm(ref.f64(x), ref.f64(res), ref.f64(w), ref.f64(b), EPS)
    dx64, dw64, db64, ex, ew, eb = ref.layer_norm_grad(ref.f64(t), ref.f64(w), ref.f64(dy), ref.f64(res), EPS)
    for o in (1, 2, 3):
        y2, t2 = at(y * 0, o), at(t * 0, (o + 1) % 4)
        mgn.mgn_layer_norm(at(x, o), at(w, o), at(b, 0), y2, res=at(res, 0), total=t2, eps=EPS)
        ref.near("y", y2, y64, e, dtype)
        assert torch.equal(t2, t) and kept(y2, o) and kept(t2, (o + 1) % 4)
        d2 = at(dx * 0, o)
        mgn.mgn_layer_norm_grad(at(t, o), at(w, o), at(dy, 0), d2, dw2, db2, d_total=at(res, 2), eps=EPS)
        ref.near("dx", d2, dx64, ex, dtype)
        ref.near("dw", dw2, dw64, ew)
        assert kept(d2, o)


def test_no_rows():
    e, w = torch.empty(0, 128, device="cuda"), torch.ones(128, device="cuda")
    mgn.mgn_layer_norm(e, w, w, e)
    dw, db = torch.full((128,), 3.0, device="cuda"), torch.full((128,), 4.0, device="cuda")
    mgn.mgn_layer_norm_grad(e, w, e, e, dw, db, accumulate=True)
    assert bool((dw == 3).all()) and bool((db == 4).all())
    mgn.mgn_layer_norm_grad(e, w, e, e, dw, db)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", [(3_000_001, 64), (700_001, 77), (40_001, 1100), (33_001, 4099)])
def test_more_rows_than_a_grid(n, cols, dtype):
    """Rows beyond the workgroups' first turn, and more bytes than the caches hold."""
    print(f"[layer] {n} x {cols} {dtype}", flush=True)
    h, U = ref.half(dtype) + 2 * ref.U, ref.U
    x = torch.randn(n, cols, device="cuda").to(dtype)
    y = torch.empty_like(x)
    mgn.mgn_layer_norm(x, None, None, y, eps=EPS)
    t = x.double()
    d = t - t.mean(1, keepdim=True)
    inv = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    u = d * inv
    # 110: the sums' 42 of the centre and of the deviation each, and the roundings between
    assert float(((y.double() - u).abs() - h * u.abs() - 110 * U * (u.abs() + 1)).max()) <= 0
    nz = LayerNorm(cols)
    g = torch.randn(n, cols, device="cuda").to(dtype)
    dx = nz.grad(x, g)
    g = g.double()
    want = (g - g.mean(1, keepdim=True) - u * (g * u).mean(1, keepdim=True)) * inv
    slack = 250 * U * inv * (g.abs() + u.abs() * (u * g).abs().mean(1, keepdim=True) + g.abs().mean(1, keepdim=True) * (1 + u.abs()))
    assert float(((dx.double() - want).abs() - slack - h * want.abs()).max()) <= 0
    dw, db = (g * u).sum(0), g.sum(0)
    assert bool(((nz.d_weight.double() - dw).abs() <= 120 * U * ((g * u).abs().sum(0) + g.abs().sum(0))).all())
    assert bool(((nz.d_bias.double() - db).abs() <= 12 * U * g.abs().sum(0)).all())


def test_streams_and_captured_replays():
    x, res, w, b, dy = _inputs(5000, 128, torch.bfloat16, seed=6)
    nz = LayerNorm(128)
    nz.weight.copy_(w)
    nz.bias.copy_(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y0, t0 = nz.apply(x, res)
    dx0 = nz.grad(t0, dy, res)
    dw0, db0 = nz.d_weight.clone(), nz.d_bias.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y1, t1 = nz.apply(x, res, stream=side.cuda_stream)
        dx1 = nz.grad(t1, dy, res, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y0, y1) and torch.equal(dx0, dx1) and torch.equal(nz.d_weight, dw0) and torch.equal(nz.d_bias, db0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, t = nz.apply(x, res)
        dx = nz.grad(t, dy, res)
    for k in range(4):
        a, c, _, _, d = _inputs(5000, 128, torch.bfloat16, seed=10 + k)
        x.copy_(a), res.copy_(c), dy.copy_(d)
        g.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y, t, dx, nz.d_weight, nz.d_bias)]
        ye, te = nz.apply(x, res)
        want = (ye, te, nz.grad(te, dy, res), nz.d_weight, nz.d_bias)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
