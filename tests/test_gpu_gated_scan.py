"""The gated linear recurrence and its backward (mgn_gated_scan,
mgn_gated_scan_grad) against float64 step by step.  The bounds on the fp32
error follow the recurrence (row_ref.scan, row_ref.scan_grad): each step's
roundings of gate, product and sum, carried on with the gates."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref
from paper_2307_13592_amd.runner import GatedMemory, LatentCache

pytestmark = pytest.mark.gpu
KINDS = [("fp32", False), ("bf16", False), ("fp32", True), ("bf16", True)]
# single steps, odd widths, few columns over many steps (split time axes),
# many columns over few steps
SHAPES = [(1, 1, 1), (1, 1885, 128), (2, 3, 5), (7, 33, 64), (8, 1, 77), (9, 130, 129), (20, 1003, 64), (64, 17, 128),
          (65, 5, 200), (127, 2, 256), (600, 3, 128), (129, 1, 1), (1000, 1, 7), (4097, 1, 64), (2049, 2, 33),
          (3, 9001, 128), (5, 2, 1025), (33, 1, 8191), (16, 700, 256), (513, 65, 64)]


def _case(T, rows, cols, typ, x8, starts=None, state=True, seed=0):
    r = np.random.default_rng([seed, T, rows, cols])
    dt = torch.float32 if typ == "fp32" else torch.bfloat16
    t = lambda a: torch.as_tensor(a.astype(np.float32)).cuda()
    c = dict(g=t(2 * r.standard_normal((T, rows, cols)) + 1).to(dt), x_scale=None, starts=None, h0=None, dh_last=None)
    x = t(r.standard_normal((T, rows, cols)) * np.exp(r.standard_normal((T, rows, 1))))
    if x8:
        cache = LatentCache(max(T * rows, 1), cols)
        cache.store(x.view(T * rows, cols))
        c["x"], c["x_scale"] = cache.window(0, T, rows)
    else:
        c["x"] = x.to(dt)
    if starts is not None:
        c["starts"] = torch.as_tensor((r.random(T) < starts).astype(np.uint8)).cuda()
    if state:
        c["h0"] = t(3 * r.standard_normal((rows, cols)))
        c["dh_last"] = t(r.standard_normal((rows, cols)))
    c["dh"] = t(r.standard_normal((T, rows, cols)))
    return c


def _x64(c):
    return ref.values8(c["x"], c["x_scale"]) if c["x_scale"] is not None else ref.f64(c["x"])


def _opt64(t):
    return None if t is None else ref.f64(t)


def _forward(c, **kw):
    h = torch.empty(c["g"].shape, device="cuda")
    last = torch.empty(c["g"].shape[1:], device="cuda")
    mgn.mgn_gated_scan(c["g"], c["x"], h=h, h_last=last, h0=c["h0"], starts=c["starts"], x_scale=c["x_scale"], **kw)
    return h, last


def _backward(c, h, **kw):
    dg, dx = torch.empty_like(c["g"]), torch.empty_like(c["g"])
    dh0 = torch.empty(c["g"].shape[1:], device="cuda")
    mgn.mgn_gated_scan_grad(c["g"], c["x"], h, dg, dx, dh=c["dh"], dh_last=c["dh_last"], dh0=dh0, h0=c["h0"],
                            starts=c["starts"], x_scale=c["x_scale"], **kw)
    return dg, dx, dh0


def _near(what, got, want, bound):
    err = np.abs(ref.f64(got) - want)
    assert np.all(err <= bound), (what, float(np.max(err / bound)))


def _check(c):
    st = None if c["starts"] is None else c["starts"].cpu().numpy()
    g64, x64, h0 = ref.f64(c["g"]), _x64(c), _opt64(c["h0"])
    h64, eh = ref.scan(g64, x64, h0, st)
    h, last = _forward(c)
    _near("h", h, h64, eh)
    assert torch.equal(last, h[-1])
    only = torch.empty_like(last)
    mgn.mgn_gated_scan(c["g"], c["x"], h=None, h_last=only, h0=c["h0"], starts=c["starts"], x_scale=c["x_scale"])
    assert torch.equal(only, last)
    h2, _ = _forward(c)
    assert torch.equal(h, h2)  # the same bits
    dg, dx, dh0 = _backward(c, h)
    hb = ref.f64(h)
    dg64, dx64, d064, eg, ex, e0 = ref.scan_grad(g64, x64, hb, h0, st, _opt64(c["dh"]), _opt64(c["dh_last"]))
    u = ref.half(dg.dtype) + ref.U32
    _near("dg", dg, dg64, eg + np.abs(dg64) * u)
    _near("dx", dx, dx64, ex + np.abs(dx64) * u)
    _near("dh0", dh0, d064, e0)
    again = _backward(c, h)
    assert all(torch.equal(a, b) for a, b in zip((dg, dx, dh0), again))


@pytest.mark.parametrize("typ,x8", KINDS)
@pytest.mark.parametrize("T,rows,cols", SHAPES)
def test_scan_and_grad(T, rows, cols, typ, x8):
    print(f"[scan] T={T} {rows} x {cols} {typ} x8={x8}", flush=True)
    _check(_case(T, rows, cols, typ, x8))


@pytest.mark.parametrize("typ,x8", [("fp32", False), ("bf16", True)])
def test_chunks_of_several_tiles(typ, x8):
    _check(_case(2050, 50, 128, typ, x8, starts=0.01, seed=9))


@pytest.mark.parametrize("typ,x8", [("fp32", False), ("bf16", True)])
@pytest.mark.parametrize("T,rows,cols", [(1, 5, 64), (20, 103, 64), (33, 1, 77), (600, 2, 128), (2050, 1, 40)])
@pytest.mark.parametrize("starts", [0.02, 0.3, 1.1])
def test_trajectories_in_one_window(T, rows, cols, typ, x8, starts):
    """Steps that begin a trajectory take no state (1.1: every step does)."""
    print(f"[scan] starts {starts} T={T} {rows} x {cols} {typ} x8={x8}", flush=True)
    c = _case(T, rows, cols, typ, x8, starts=starts, seed=1)
    _check(c)
    c["h0"] = c["dh_last"] = None
    _check(c)


def test_trajectory_equals_its_own_scan():
    """A window of three trajectories gives each one's own states and
    gradients, and a state before a start has no gradient."""
    c = _case(30, 40, 64, "fp32", False, seed=2)
    c["starts"] = torch.zeros(30, dtype=torch.uint8, device="cuda")
    c["starts"][[0, 11, 12]] = 1
    h, last = _forward(c)
    dg, dx, dh0 = _backward(c, h)
    assert not dh0.any()
    for a, b in ((0, 11), (11, 12), (12, 30)):
        p = dict(c, g=c["g"][a:b].contiguous(), x=c["x"][a:b].contiguous(), dh=c["dh"][a:b].contiguous(), starts=None,
                 h0=None, dh_last=c["dh_last"] if b == 30 else None)
        hp, _ = _forward(p)
        assert torch.allclose(hp, h[a:b], rtol=1e-5, atol=1e-5)
        gp = _backward(p, hp)
        assert torch.allclose(gp[0], dg[a:b], rtol=1e-4, atol=1e-5)
        assert torch.allclose(gp[1], dx[a:b], rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("T,rows,cols", [(9, 30, 64), (300, 2, 77), (2100, 1, 64)])
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_held_and_replaced_states(T, rows, cols, typ):
    """g = +inf or the type's largest value holds a state through steps whose
    x is NaN or infinite; -inf or the lowest value replaces a state that is
    NaN.  What is left out has no gradient."""
    print(f"[scan] held and replaced T={T} {rows} x {cols} {typ}", flush=True)
    c = _case(T, rows, cols, typ, False, seed=3)
    big = torch.finfo(c["g"].dtype).max
    r = np.random.default_rng(T)
    hold = torch.as_tensor(r.random((T, rows, cols)) < 0.3).cuda()
    c["g"][hold] = float("inf")
    c["g"][hold & torch.as_tensor(r.random((T, rows, cols)) < 0.5).cuda()] = big
    c["x"][hold] = float("nan")
    c["x"][hold & torch.as_tensor(r.random((T, rows, cols)) < 0.5).cuda()] = float("-inf")
    c["g"][0, 0], c["g"][0, 0, ::2] = -float("inf"), -big
    c["x"][0, 0] = 1.5
    c["h0"][0] = float("nan")
    if T > 4:
        c["g"][4, :, 0], c["x"][4, :, 0] = float("inf"), float("nan")
    h, last = _forward(c)
    assert bool(h.isfinite().all())
    held = hold.clone()
    held[0] = False
    prev = torch.cat([h[:1], h[:-1]])
    if rows * cols > 2000:  # unsplit: held states keep their bits
        assert torch.equal(h[held], prev[held])
    assert bool((h[0, 0] == 1.5).all())
    dg, dx, dh0 = _backward(c, h)
    assert bool(dg.isfinite().all()) and bool(dx.isfinite().all()) and bool(dh0.isfinite().all())
    assert not dg[held].any() and not dx[held].any()
    assert not dg[0, 0].any() and not dh0[0].any()
    # the finite part against float64
    z = dict(c, h0=c["h0"].nan_to_num(0.0), x=torch.where(hold, torch.zeros_like(c["x"]), c["x"]))
    if T > 4:
        z["x"][4, :, 0] = 0
    _check(z)


def test_nan_in_one_column_stays_there():
    c = _case(40, 3, 64, "fp32", False, seed=4)
    h0, _ = _forward(c)
    c["x"][17, 1, 5] = float("nan")
    h, _ = _forward(c)
    bad = torch.zeros_like(h, dtype=torch.bool)
    bad[17:, 1, 5] = True
    assert bool(h[bad].isnan().all()) and torch.equal(h[~bad], h0[~bad])


def test_running_mean():
    """g_t = log(t): h is the running mean of x (the temporal mean)."""
    T, rows, cols = 600, 50, 5
    x = torch.randn(T, rows, cols, device="cuda")
    g = torch.log(torch.arange(T, device="cuda", dtype=torch.float32))[:, None, None].expand(T, rows, cols).contiguous()
    m = GatedMemory(rows, cols)
    h = m.scan(g, x)
    want = x.double().cumsum(0) / torch.arange(1, T + 1, device="cuda", dtype=torch.float64)[:, None, None]
    assert float((h.double() - want).abs().max()) <= 1e-5
    assert torch.equal(m.state, h[-1])


def test_grad_against_differences():
    T, rows, cols, step = 6, 2, 3, 1e-6
    c = _case(T, rows, cols, "fp32", False, seed=5)
    c["starts"] = torch.zeros(T, dtype=torch.uint8, device="cuda")
    c["starts"][3] = 1
    st = c["starts"].cpu().numpy()
    v = {k: ref.f64(c[k]) for k in ("g", "x", "h0")}
    w, wl = ref.f64(c["dh"]), ref.f64(c["dh_last"])

    def loss(g, x, h0):
        h = ref.scan(g, x, h0, st)[0]
        return float(np.sum(h * w) + np.sum(h[-1] * wl))

    got = dict(zip(("g", "x", "h0"), _backward(c, _forward(c)[0])))
    for k in v:
        num = np.zeros_like(v[k])
        for i in np.ndindex(num.shape):
            p, q = dict(v), dict(v)
            d = np.zeros_like(num)
            d[i] = step
            p[k], q[k] = v[k] + d, v[k] - d
            num[i] = (loss(**p) - loss(**q)) / (2 * step)
        assert np.allclose(ref.f64(got[k]), num, rtol=1e-4, atol=1e-4 * np.abs(num).max()), k


@pytest.mark.parametrize("T,rows,cols", [(1, 200, 128), (12, 40, 64), (100, 9, 64), (40, 900, 128), (3000, 1, 64)])
def test_state_in_place_and_windows(T, rows, cols):
    """h_last on h0, dh0 on dh_last, and a trajectory cut into windows that
    hand the state (backward: its gradient) on."""
    c = _case(T, rows, cols, "fp32", False, seed=6)
    h, last = _forward(c)
    s = c["h0"].clone()
    mgn.mgn_gated_scan(c["g"], c["x"], h_last=s, h0=s)
    assert torch.equal(s, last)
    s, h2 = c["h0"].clone(), torch.empty_like(h)
    mgn.mgn_gated_scan(c["g"], c["x"], h=h2, h_last=s, h0=s)
    assert torch.equal(s, last) and torch.equal(h2, h)
    dg, dx, dh0 = _backward(c, h)
    d = c["dh_last"].clone()
    mgn.mgn_gated_scan_grad(c["g"], c["x"], h, torch.empty_like(dg), torch.empty_like(dx), dh=c["dh"], dh_last=d, dh0=d,
                            h0=c["h0"])
    assert torch.equal(d, dh0)
    m = GatedMemory(rows, cols)
    m.state.copy_(c["h0"])
    cut = T // 3
    parts, hs = [(0, cut), (cut, cut), (cut, T)], []
    for a, b in parts:  # one of them empty
        hs.append((m.scan(c["g"][a:b], c["x"][a:b]), m.h0.clone()))
    assert torch.allclose(torch.cat([p[0] for p in hs]), h, rtol=1e-5, atol=1e-5)
    carry = c["dh_last"]
    for (a, b), (hp, h0) in reversed(list(zip(parts, hs))):
        m.h0.copy_(h0)
        gp, xp, carry = m.grad(c["g"][a:b], c["x"][a:b], hp, c["dh"][a:b].contiguous(), carry)
        assert torch.allclose(gp, dg[a:b], rtol=1e-3, atol=1e-4) and torch.allclose(xp, dx[a:b], rtol=1e-3, atol=1e-4)
    assert torch.allclose(carry, dh0, rtol=1e-3, atol=1e-4)


def test_no_steps_and_no_rows():
    g = torch.empty(0, 7, 64, device="cuda")
    h0 = torch.randn(7, 64, device="cuda")
    out = torch.full((7, 64), 9.0, device="cuda")
    mgn.mgn_gated_scan(g, g, h_last=out, h0=h0)
    assert torch.equal(out, h0)
    mgn.mgn_gated_scan(g, g, h_last=out)
    assert not out.any()
    mgn.mgn_gated_scan_grad(g, g, g, g, g, dh_last=h0, dh0=out)
    assert torch.equal(out, h0)
    mgn.mgn_gated_scan_grad(g, g, g, g, g, dh0=out)
    assert not out.any()
    e = torch.empty(5, 0, 64, device="cuda")
    mgn.mgn_gated_scan(e, e, h=e, h_last=e[0])
    mgn.mgn_gated_scan_grad(e, e, e, e, e, dh=e)


@pytest.mark.parametrize("typ", ["fp32", "bf16"])
@pytest.mark.parametrize("T,rows,cols", [(5, 40, 128), (700, 1, 64)])
def test_arrays_aligned_to_their_type_only(T, rows, cols, typ):
    c = _case(T, rows, cols, typ, False, seed=7)
    h, last = _forward(c)
    want = _backward(c, h)

    def at(v, o):
        return torch.full((v.numel() + 8,), 5.0, dtype=v.dtype, device="cuda")[o:o + v.numel()].view(v.shape).copy_(v)

    for o in (1, 2, 3):
        u = dict(c, **{k: at(c[k], (o + i) % 4) for i, k in enumerate(("g", "x", "h0", "dh", "dh_last"))})
        h2, last2 = at(h * 0, o), at(last * 0, 1)
        mgn.mgn_gated_scan(u["g"], u["x"], h=h2, h_last=last2, h0=u["h0"])
        # (another dealing of columns may split the time axis elsewhere)
        assert torch.allclose(h2, h, rtol=1e-5, atol=1e-5) and torch.allclose(last2, last, rtol=1e-5, atol=1e-5)
        dg, dx, d0 = at(want[0] * 0, o), at(want[1] * 0, 1), at(want[2] * 0, 3)
        mgn.mgn_gated_scan_grad(u["g"], u["x"], at(h, 3), dg, dx, dh=u["dh"], dh_last=u["dh_last"], dh0=d0, h0=u["h0"])
        tol = 1e-2 if typ == "bf16" else 1e-4
        assert all(torch.allclose(p.float(), q.float(), rtol=tol, atol=tol) for p, q in zip((dg, dx, d0), want))


@pytest.mark.parametrize("T,rows,cols,typ,x8", [(9, 1 << 22, 128, "bf16", False), (2, 600_001, 121, "bf16", False),
                                                (700, 1000, 128, "fp32", False), (400, 2000, 128, "bf16", True),
                                                (40, 40_001, 128, "fp32", False), (40, 40_001, 128, "fp32", True),
                                                (40, 60_001, 128, "bf16", True)])
def test_large_windows(T, rows, cols, typ, x8):
    """Offsets past 2^32 elements, more columns than one launch takes (four
    and one a lane), and windows that the caches do not hold in every form and
    type: some rows against float64."""
    print(f"[scan] {T} x {rows} x {cols} {typ} x8={x8}", flush=True)
    dt = torch.float32 if typ == "fp32" else torch.bfloat16
    g = torch.empty(T, rows, cols, dtype=dt, device="cuda").normal_()
    if x8:
        c = LatentCache(T * rows, cols)
        c.store(torch.empty(T * rows, cols, device="cuda").normal_())
        x, xs = c.window(0, T, rows)
    else:
        x, xs = torch.empty_like(g).normal_(), None
    h = torch.empty(T, rows, cols, device="cuda")
    mgn.mgn_gated_scan(g, x, h=h, x_scale=xs)
    at = [0, 1, rows // 2, rows - 1]
    x64 = ref.values8(x[:, at], xs[:, at]) if x8 else ref.f64(x[:, at])
    h64, e = ref.scan(ref.f64(g[:, at]), x64, None, None)
    _near("h", h[:, at], h64, e)
    dg, dx = torch.empty_like(g), torch.empty_like(g)
    dl = torch.randn(rows, cols, device="cuda")
    dh = torch.empty_like(h).normal_() if T * rows < 1 << 24 else None
    mgn.mgn_gated_scan_grad(g, x, h, dg, dx, dh=dh, dh_last=dl, x_scale=xs)
    a, b, _, ea, eb, _ = ref.scan_grad(ref.f64(g[:, at]), x64, ref.f64(h[:, at]), None, None,
                                       None if dh is None else ref.f64(dh[:, at]), ref.f64(dl[at]))
    u = ref.half(dt) + ref.U32
    _near("dg", dg[:, at], a, ea + np.abs(a) * u)
    _near("dx", dx[:, at], b, eb + np.abs(b) * u)


@pytest.mark.parametrize("T,rows,cols", [(6, 50, 128), (5000, 1, 64)])
def test_streams_and_captured_replays(T, rows, cols):
    """A stream of its own with its own scratch; two graphs of the same call
    replayed in turn on two streams; new inputs and eager work between."""
    c = _case(T, rows, cols, "fp32", False, seed=8)
    h, last = _forward(c)
    want = _backward(c, h)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        h1, last1 = _forward(c, stream=side.cuda_stream)
        got = _backward(c, h1, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(h, h1) and all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            hg, lg = _forward(c)
            dg = _backward(c, hg)
        graphs.append((gr, hg, lg, dg))
    for k in range(3):
        d = _case(T, rows, cols, "fp32", False, seed=20 + k)
        for key in ("g", "x", "h0", "dh", "dh_last"):
            c[key].copy_(d[key])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0][0].replay()
        graphs[1][0].replay()
        torch.cuda.synchronize()
        h, last = _forward(c)
        want = _backward(c, h)
        for _, hg, lg, dg in graphs:
            assert torch.equal(hg, h) and torch.equal(lg, last)
            assert all(torch.equal(a, b) for a, b in zip(dg, want))
