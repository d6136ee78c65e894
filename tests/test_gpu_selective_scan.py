"""The selective state space scan and its backward (mgn_selective_scan,
mgn_selective_scan_grad) against float64 step by step, within the bounds of
memory_ref."""
import numpy as np
import pytest
import torch

import memory_ref as ref
import paper_2307_13592_amd as mgn

pytestmark = pytest.mark.gpu
# single steps, odd widths, one column, rows that share a wave, few columns over many
# steps (chunks of the time axis), many rows, several tiles of columns
SHAPES = [(1, 1, 1, 1), (1, 300, 128, 16), (2, 3, 5, 3), (7, 33, 64, 4), (8, 1, 77, 5), (9, 70, 12, 16), (17, 19, 130, 8),
          (20, 103, 64, 16), (33, 2, 300, 16), (64, 3, 16, 33), (70, 1, 64, 64), (25, 2, 1025, 2), (130, 3, 20, 17),
          (600, 1, 64, 16), (1030, 2, 33, 7), (2050, 1, 3, 1), (301, 1, 65, 48), (12, 2, 8191, 1)]


def _case(T, rows, cols, n, dtype, gate=True, D=True, bias=True, softplus=True, starts=None, state=True, seed=0):
    r = np.random.default_rng([seed, T, rows, cols, n])
    t = lambda *s: torch.as_tensor(r.standard_normal(s).astype(np.float32)).cuda()
    c = dict(x=t(T, rows, cols).to(dtype), B=t(T, rows, n).to(dtype), C=t(T, rows, n).to(dtype), dy=t(T, rows, cols).to(dtype),
             z=t(T, rows, cols).to(dtype) if gate else None, D=t(cols) if D else None, softplus=softplus,
             A=-torch.exp(t(cols, n)), h0=t(rows, cols, n) if state else None, dh_last=t(rows, cols, n) if state else None,
             starts=None, bias=None)
    if softplus:
        c["dt"], c["bias"] = (2 * t(T, rows, cols)).to(dtype), t(cols) - 1 if bias else None
    else:
        c["dt"], c["bias"] = (0.3 * t(T, rows, cols).abs()).to(dtype), 0.1 * t(cols).abs() if bias else None
    if starts is not None:
        c["starts"] = torch.as_tensor((r.random(T) < starts).astype(np.uint8)).cuda()
    return c


def _args(c):
    return dict(D=c["D"], dt_bias=c["bias"], z=c["z"], starts=c["starts"], softplus=c["softplus"])


def _forward(c, **kw):
    y, last = torch.empty_like(c["x"]), torch.empty(c["x"].shape[1:] + c["A"].shape[1:], device="cuda")
    marks = mgn.mgn_selective_marks(c["x"], c["A"])
    mgn.mgn_selective_scan(c["x"], c["dt"], c["A"], c["B"], c["C"], y, h0=c["h0"], h_last=last, marks=marks, **_args(c), **kw)
    return y, last, marks


def _backward(c, marks, **kw):
    e = torch.empty_like
    g = dict(dx=e(c["x"]), ddt=e(c["x"]), dA=e(c["A"]), dB=e(c["B"]), dC=e(c["C"]), d_bias=torch.empty(c["x"].shape[2], device="cuda"),
             dz=None if c["z"] is None else e(c["z"]), dD=None if c["D"] is None else e(c["D"]),
             dh0=torch.empty(c["x"].shape[1:] + c["A"].shape[1:], device="cuda"))
    mgn.mgn_selective_scan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], marks, c["dy"], dh_last=c["dh_last"], **g, **_args(c), **kw)
    return {k: v for k, v in g.items() if v is not None}


def _ref(c):
    o = lambda v: v if v is None or isinstance(v, bool) else v.cpu().numpy() if v.dtype == torch.uint8 else ref.f64(v)
    return {k: o(v) for k, v in c.items()}


def _chunked(c):
    """Steps whose deltas are summed at once: the whole axis at most where it is cut."""
    T, R, D = c["x"].shape
    n = c["A"].shape[1]
    cut = mgn.mgn_selective_scan_work(T, R, D, n) > 0 or T >= 64
    return T if cut else 0


def _check(c, again=True):
    r = _ref(c)
    k = _chunked(c)
    with np.errstate(invalid="ignore", over="ignore"):
        f = ref.ssm(r, k)
        y, last, marks = _forward(c)
        ref.near("y", y, f["y"], f["ey"], y.dtype)
        ref.near("h_last", last, f["last"], f["elast"])
        for m in range(1, marks.shape[0]):
            at = m * mgn.MGN_MARK_STEPS - 1
            ref.near(f"mark {m}", marks[m], f["h"][at], f["eh"][at])
        g = _backward(c, marks)
        want = ref.ssm_grad(r, f, r["dy"], r["dh_last"], tiles=-(-c["x"].shape[2] // 64), chunk=k)
        for name, got in g.items():
            ref.near(name, got, *want[name], got.dtype)
    if again:
        y2, last2, marks2 = _forward(c)
        assert torch.equal(y, y2) and torch.equal(last, last2) and torch.equal(marks, marks2)  # the same bits
        g2 = _backward(c, marks)
        assert all(torch.equal(g[k], g2[k]) for k in g)
    return y, last, marks, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", SHAPES)
def test_scan_and_grad(T, rows, cols, n, dtype):
    for kw in (dict(), dict(gate=False, D=False), dict(softplus=False, bias=False, state=False)):
        print(f"[ssm] {T} x {rows} x {cols}, {n} {dtype} {kw}", flush=True)
        _check(_case(T, rows, cols, n, dtype, **kw))


@pytest.mark.parametrize("n", range(1, 65))
def test_every_number_of_states(n):
    _check(_case(11, 3, 9, n, torch.bfloat16 if n % 2 else torch.float32, gate=n % 3 > 0, seed=1))


@pytest.mark.parametrize("cols", [1, 2, 3, 4, 6, 7, 13, 16, 17, 31, 63, 64, 66, 100, 255])
def test_every_kind_of_width(cols):
    _check(_case(10, 37, cols, 16, torch.float32 if cols % 2 else torch.bfloat16, starts=0.1, seed=2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", [(75, 2101, 64, 16), (130, 1100, 62, 11), (66, 2500, 60, 13), (67, 1100, 64, 3), (129, 600, 128, 8),
                                           (65, 1030, 64, 40)])
def test_long_axes_of_many_rows(T, rows, cols, n, dtype):
    """More than 64 steps at once (whose starts are looked at 64 at a time), up to more
    waves than the card holds: some rows."""
    print(f"[ssm] long {T} x {rows} x {cols}, {n} {dtype}", flush=True)
    c = _case(T, rows, cols, n, dtype, starts=0.05, seed=15)
    c["starts"][[2, 63, 64]] = 1
    assert mgn.mgn_selective_scan_work(T, rows, cols, n) == 0
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    some = [0, 15, 16, rows // 2, rows - 1]
    few = {k: v[:, some].contiguous() if k in ("x", "dt", "B", "C", "z", "dy") else v[some].contiguous() if k in ("h0", "dh_last") else v
           for k, v in c.items()}
    r = _ref(few)
    f = ref.ssm(r, T)
    ref.near("y", y[:, some], f["y"], f["ey"], dtype)
    ref.near("h_last", last[some], f["last"], f["elast"])
    want = ref.ssm_grad(r, f, r["dy"], r["dh_last"], tiles=-(-cols // 64), chunk=T)
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        ref.near(k, g[k][:, some], *want[k], dtype)
    ref.near("dh0", g["dh0"][some], *want["dh0"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", [(1, 5, 64, 16), (20, 33, 64, 16), (30, 2, 7, 3), (700, 1, 70, 16), (130, 1, 64, 40)])
@pytest.mark.parametrize("starts", [0.03, 0.3, 1.1])
def test_trajectories_in_one_window(T, rows, cols, n, dtype, starts):
    print(f"[ssm] starts {starts} {T} x {rows} x {cols}, {n} {dtype}", flush=True)
    _check(_case(T, rows, cols, n, dtype, starts=starts, seed=3))
    _check(_case(T, rows, cols, n, dtype, starts=starts, gate=False, state=False, seed=4))


@pytest.mark.parametrize("T,rows,cols,n", [(9, 30, 64, 16), (40, 3, 9, 5), (700, 1, 64, 16), (70, 1, 32, 40)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_of_size_0(T, rows, cols, n, dtype):
    """dt of -infinity or of the type's lowest value leaves the states to the bit,
    whatever x and B hold, and nothing left out has a gradient."""
    c = _case(T, rows, cols, n, dtype, gate=False, D=False, seed=5)
    r = np.random.default_rng(T)
    held = torch.as_tensor(r.random((T, rows, cols)) < 0.3).cuda()
    whole = torch.as_tensor(r.random((T, rows)) < 0.3).cuda()  # steps of a whole row: padding
    whole[-1] = True
    held |= whole[:, :, None]
    low = torch.finfo(dtype).min
    c["dt"][held] = -float("inf")
    c["dt"][held & torch.as_tensor(r.random((T, rows, cols)) < 0.5).cuda()] = low
    c["x"][held] = float("nan")
    c["B"][whole] = float("nan")
    c["B"][whole & torch.as_tensor(r.random((T, rows)) < 0.5).cuda()] = float("inf")
    y, last, marks, g = _check(c)
    assert not g["dx"][held].any() and not g["ddt"][held].any() and not g["dB"][whole].any()
    before, after = torch.empty_like(last), torch.empty_like(last)
    one = dict(c, h0=last)
    for k in ("x", "dt", "B", "C", "dy"):
        one[k] = c[k][-1:].contiguous()
    mgn.mgn_selective_scan(one["x"], one["dt"], one["A"], one["B"], one["C"], torch.empty_like(one["x"]), h0=last, h_last=after,
                           **_args(one))
    assert torch.equal(after, last)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", [(9, 30, 64, 16), (700, 1, 64, 16), (70, 1, 32, 40)])
def test_steps_that_no_gradient_reaches(T, rows, cols, n, dtype):
    """Steps of size 0 with dy = 0: the gradients are those with zeros in x and B there."""
    c = _case(T, rows, cols, n, dtype, seed=12)
    held = torch.as_tensor(np.random.default_rng(13).random((T, rows)) < 0.3).cuda()
    c["dt"][held], c["dy"][held], c["x"][held], c["B"][held] = -float("inf"), 0, 0, 0
    _, last0, marks0 = _forward(c)
    want = _backward(c, marks0)
    c["x"][held], c["B"][held] = float("nan"), float("inf")
    _, last, marks = _forward(c)
    got = _backward(c, marks)
    assert torch.equal(last, last0) and torch.equal(marks, marks0)
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("T,rows,cols", [(600, 1, 64), (1000, 1, 8), (40, 1, 8), (600, 40, 3)])
def test_zero_states_under_growing_factors(T, rows, cols):
    """exp(A sum of delta) passes the fp32 range over many steps; states (and their
    gradients) that are zero stay so."""
    n, few = 5, 3
    c = _case(T, rows, cols, n, torch.float32, gate=False, softplus=False, bias=False, state=False, seed=14)
    c["A"] = 6 + 2 * torch.rand_like(c["A"])
    c["dt"][:] = 1
    c["x"][:-few], c["dy"][few:] = 0, 0
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    assert not y[:-few].any()
    cut = lambda s: {k: v[s] if k in ("x", "dt", "B", "C", "dy") else v for k, v in _ref(c).items()}
    end, begin = cut(slice(T - few, T)), cut(slice(0, few))
    f = ref.ssm(end)
    ref.near("y", y[-few:], f["y"], f["ey"])
    ref.near("h_last", last, f["last"], f["elast"])
    want = ref.ssm_grad(begin, ref.ssm(begin), begin["dy"], None)
    for k in ("dx", "ddt", "dB", "dC"):
        assert not g[k][few:].any(), k
        ref.near(k, g[k][:few], *want[k])
    assert not g["dA"].any()
    ref.near("dh0", g["dh0"], *want["dh0"])


@pytest.mark.parametrize("T,rows,cols,n", [(30, 3, 40, 16), (900, 1, 20, 16)])
def test_a_trajectory_that_is_not_finite_ends_at_a_start(T, rows, cols, n):
    c = _case(T, rows, cols, n, torch.float32, seed=6)
    s = T // 3
    c["starts"] = torch.zeros(T, dtype=torch.uint8, device="cuda")
    c["starts"][[s, 2 * s]] = 1
    y0, last0, marks0 = _forward(c)
    g0 = _backward(c, marks0)
    c["x"][s - 1], c["h0"][:] = float("nan"), float("inf")
    c["x"][2 * s - 1, :, 0] = float("inf")
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    assert torch.equal(y[s:2 * s - 1], y0[s:2 * s - 1]) and torch.equal(y[2 * s:], y0[2 * s:]) and torch.equal(last, last0)
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        assert torch.equal(g[k][2 * s:], g0[k][2 * s:]), k
    # the last trajectory's gradient that is not finite does not reach those before it
    c = _case(T, rows, cols, n, torch.float32, seed=6)
    c["starts"] = torch.zeros(T, dtype=torch.uint8, device="cuda")
    c["starts"][s] = 1
    c["dh_last"][:] = float("nan")
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        assert bool(g[k][:s].isfinite().all()), k
    assert bool(g["dh0"].isfinite().all()) and bool(g["dx"][s:].isnan().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_windows_and_single_steps_are_the_whole(dtype):
    """Window by window, and step by step with the states updated in place; the
    windows' backward hands dh0 on, in place too."""
    T, rows, cols, n = 31, 40, 64, 16
    c = _case(T, rows, cols, n, dtype, seed=7)
    assert mgn.mgn_selective_scan_work(T, rows, cols, n) == 0  # (chunks would add in another order)
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    for cuts in (list(range(T + 1)), [0, 8, 16, 17, 31]):
        h, ys = c["h0"].clone(), []
        for a, b in zip(cuts, cuts[1:]):
            ys.append(torch.empty_like(c["x"][a:b]))
            p = {k: (c[k][a:b] if k in ("x", "dt", "B", "C", "z") else c[k]) for k in c}
            mgn.mgn_selective_scan(p["x"], p["dt"], p["A"], p["B"], p["C"], ys[-1], h0=h, h_last=h, **_args(p))
        assert torch.equal(torch.cat(ys), y) and torch.equal(h, last)
    cuts, d, dA = [0, 8, 24, 31], c["dh_last"].clone(), None
    hs = [c["h0"]]
    parts = []
    for a, b in zip(cuts, cuts[1:]):
        p = {k: (c[k][a:b].contiguous() if k in ("x", "dt", "B", "C", "z", "dy") else c[k]) for k in c}
        p["h0"] = hs[-1]
        _, l, m = _forward(p)
        hs.append(l)
        parts.append((p, m))
    dx = []
    dA, dD, db = torch.empty_like(c["A"]), torch.empty_like(c["D"]), torch.empty_like(c["bias"])
    for k in range(len(parts) - 1, -1, -1):
        p, m = parts[k]
        e = torch.empty_like
        dxk = e(p["x"])
        mgn.mgn_selective_scan_grad(p["x"], p["dt"], p["A"], p["B"], p["C"], m, p["dy"], dxk, e(p["x"]), dA, e(p["B"]), e(p["C"]),
                                    dD, db, e(p["x"]), dh_last=d, dh0=d, accumulate=k < len(parts) - 1, **_args(p))
        dx.insert(0, dxk)
    assert torch.equal(torch.cat(dx), g["dx"]) and torch.equal(d, g["dh0"])
    r = _ref(c)
    f = ref.ssm(r)
    want = ref.ssm_grad(r, f, r["dy"], r["dh_last"])
    for got, name in ((dA, "dA"), (dD, "dD"), (db, "d_bias")):
        v, e = want[name]
        ref.near(name, got, v, e + 4 * ref.U * np.abs(v))


def test_chunks_join_in_place():
    """A time axis that is cut, with the states and their gradients in place."""
    c = _case(2000, 1, 40, 16, torch.float32, seed=8)
    assert mgn.mgn_selective_scan_work(2000, 1, 40, 16) > 0
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    h, y2 = c["h0"].clone(), torch.empty_like(y)
    mgn.mgn_selective_scan(c["x"], c["dt"], c["A"], c["B"], c["C"], y2, h0=h, h_last=h, **_args(c))
    assert torch.equal(h, last) and torch.equal(y, y2)
    d, e = c["dh_last"].clone(), torch.empty_like
    mgn.mgn_selective_scan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], marks, c["dy"], e(y), e(y), None, e(c["B"]), e(c["C"]),
                                dz=e(y), dh_last=d, dh0=d, **_args(c))
    assert torch.equal(d, g["dh0"])


def test_grad_against_differences():
    T, rows, cols, n, step = 5, 2, 3, 2, 1e-6
    c = _case(T, rows, cols, n, torch.float32, seed=9)
    r = _ref(c)
    _, _, marks = _forward(c)
    g = _backward(c, marks)

    def loss(**kw):
        f = ref.ssm(dict(r, **kw))
        return float((f["y"] * r["dy"]).sum() + (f["last"] * r["dh_last"]).sum())

    for key, name in (("x", "dx"), ("dt", "ddt"), ("A", "dA"), ("B", "dB"), ("C", "dC"), ("D", "dD"), ("z", "dz"),
                      ("bias", "d_bias"), ("h0", "dh0")):
        num = np.zeros_like(r[key])
        for i in np.ndindex(num.shape):
            lo, hi = r[key].copy(), r[key].copy()
            lo[i] -= step
            hi[i] += step
            num[i] = (loss(**{key: hi}) - loss(**{key: lo})) / (2 * step)
        assert np.allclose(ref.f64(g[name]), num, rtol=2e-5, atol=2e-5 * np.abs(num).max()), name


def test_accumulated_sums():
    c = _case(20, 50, 64, 16, torch.float32, seed=10)
    _, _, marks = _forward(c)
    g = _backward(c, marks)
    e = torch.empty_like
    sums = [torch.full_like(g[k], 2.0) for k in ("dA", "dD", "d_bias")]
    mgn.mgn_selective_scan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], marks, c["dy"], e(c["x"]), e(c["x"]), sums[0], e(c["B"]),
                                e(c["C"]), sums[1], sums[2], e(c["x"]), dh_last=c["dh_last"], accumulate=True, **_args(c))
    for s, k in zip(sums, ("dA", "dD", "d_bias")):
        assert bool(((s - 2 - g[k]).abs() <= 3 * ref.U * (s.abs() + g[k].abs() + 2)).all())


def test_step_sizes_of_any_size():
    """softplus and its slope from very small to large arguments."""
    v = torch.linspace(-86, 90, 5000, device="cuda")[None, :, None].contiguous()
    c = dict(x=torch.ones_like(v), dt=v, A=torch.full((1, 1), -1.0, device="cuda"), B=torch.ones_like(v), C=torch.ones_like(v),
             D=None, bias=None, z=None, h0=None, starts=None, softplus=True, dy=torch.ones_like(v), dh_last=None)
    y, last, marks = _forward(c)
    want = torch.nn.functional.softplus(v.double(), threshold=1000.0)
    rel = ((y.double() - want) / want).abs()
    # the exponential's argument and value, the series and the products
    assert bool((rel <= ref.U * (14 + 2 * v.double().abs().clamp(max=88) * torch.exp(-v.double().clamp(min=0)))).all())
    g = _backward(c, marks)
    slope = torch.sigmoid(v.double())
    assert bool((((g["ddt"].double() - slope) / slope).abs() <= ref.U * (16 + 2 * v.double().abs().clamp(max=88))).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_unaligned_arrays(dtype):
    c = _case(20, 7, 64, 16, dtype, starts=0.1, seed=11)

    def at(v, o):
        return torch.full((v.numel() + 8,), 5.0, dtype=v.dtype, device="cuda")[o:o + v.numel()].view(v.shape).copy_(v)

    for o in (1, 2, 3):
        d = dict(c)
        for k, key in enumerate(("x", "dt", "A", "B", "C", "D", "z", "bias", "h0", "dh_last", "dy")):
            d[key] = at(c[key], (o + k) % 4)
        _check(d)


def test_nothing_to_do():
    x, A = torch.empty(0, 3, 8, device="cuda"), -torch.ones(8, 4, device="cuda")
    p, h = torch.empty(0, 3, 4, device="cuda"), torch.randn(3, 8, 4, device="cuda")
    out = torch.empty_like(h)
    mgn.mgn_selective_scan(x, x, A, p, p, x, h0=h, h_last=out)
    assert torch.equal(out, h)
    mgn.mgn_selective_scan(x, x, A, p, p, x, h_last=out)
    assert not out.any()
    dA, marks = torch.full_like(A, 2.0), mgn.mgn_selective_marks(x, A)
    mgn.mgn_selective_scan_grad(x, x, A, p, p, marks, x, x, x, dA, p, p, dh_last=h, dh0=out, accumulate=True)
    assert bool((dA == 2).all()) and torch.equal(out, h)
    mgn.mgn_selective_scan_grad(x, x, A, p, p, marks, x, x, x, dA, p, p)
    assert not dA.any()
    e, q = torch.empty(5, 0, 8, device="cuda"), torch.empty(5, 0, 4, device="cuda")
    mgn.mgn_selective_scan(e, e, A, q, q, e)
    mgn.mgn_selective_scan_grad(e, e, A, q, q, mgn.mgn_selective_marks(e, A), e, e, e, dA.fill_(1), q, q)
    assert not dA.any()


def test_streams_and_captured_replays():
    shapes = [(24, 60, 64, 16), (700, 1, 20, 8)]
    for k, shape in enumerate(shapes):
        c = _case(*shape, torch.bfloat16, starts=0.1, seed=12)

        def run(**kw):
            y, last, marks = _forward(c, **kw)
            return [y, last] + list(_backward(c, marks, **kw).values())

        want = run()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = run(stream=side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = run()
        for i in range(4):
            new = _case(*shape, torch.bfloat16, starts=0.1, seed=30 + i)
            for key in ("x", "dt", "A", "B", "C", "D", "z", "bias", "h0", "dh_last", "dy", "starts"):
                c[key].copy_(new[key])
            g.replay()
            torch.cuda.synchronize()
            kept = [v.clone() for v in got]
            assert all(torch.equal(p, q) for p, q in zip(kept, run()))


def test_offsets_past_32_bits():
    """More than 2^32 elements: the last rows against their own call, to the bit."""
    T, rows, cols, n = 9, 7_500_000, 64, 1
    big = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    c = dict(x=big(T, rows, cols), dt=big(T, rows, cols), B=big(T, rows, n), C=big(T, rows, n), z=None, D=None, bias=None, h0=None,
             starts=None, softplus=True, A=-torch.rand(cols, n, device="cuda"), dh_last=None)
    for k in ("x", "dt", "B", "C"):
        for t in range(T):
            c[k][t].normal_()
    c["dy"] = c["x"]
    tail = slice(rows - 500, rows)
    y, last, marks = _forward(c)
    e = torch.empty_like
    dx, dB = e(c["x"]), e(c["B"])
    mgn.mgn_selective_scan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], marks, c["dy"], dx, e(c["x"]), None, dB, e(c["C"]), **_args(c))
    p = {k: (v[:, tail].contiguous() if k in ("x", "dt", "B", "C", "dy") else v) for k, v in c.items()}
    assert mgn.mgn_selective_scan_work(T, 500, cols, n) == 0
    py, plast, pmarks = _forward(p)
    assert torch.equal(y[:, tail], py) and torch.equal(last[tail], plast) and torch.equal(marks[:, tail], pmarks)
    g = _backward(p, pmarks)
    assert torch.equal(dx[:, tail], g["dx"]) and torch.equal(dB[:, tail], g["dB"])
