"""The short causal convolution along time and its backward (mgn_causal_conv,
mgn_causal_conv_grad) against float64, within the bounds of memory_ref."""
import numpy as np
import pytest
import torch

import memory_ref as ref
import paper_2307_13592_amd as mgn

pytestmark = pytest.mark.gpu
# single steps, windows shorter than the taps, odd widths, wide rows, few columns
# over many steps (split time axes), many rows
SHAPES = [(1, 1, 1), (1, 1885, 128), (2, 3, 5), (3, 70, 64), (7, 33, 77), (20, 203, 64), (33, 2, 1025), (64, 17, 128),
          (65, 5, 200), (300, 1, 2049), (600, 3, 128), (1000, 1, 7), (2049, 2, 33), (4100, 1, 64), (5, 2, 8191)]


def _case(T, rows, cols, W, dtype, starts=None, state=True, silu=True, bias=True, seed=0):
    r = np.random.default_rng([seed, T, rows, cols, W])
    t = lambda *s: torch.as_tensor(r.standard_normal(s).astype(np.float32)).cuda()
    c = dict(x=t(T, rows, cols).to(dtype), weight=t(cols, W), bias=t(cols) if bias else None, silu=silu, starts=None,
             past=None, dy=t(T, rows, cols).to(dtype), d_past_out=None)
    if state:
        c["past"], c["d_past_out"] = t(W - 1, rows, cols).to(dtype), t(W - 1, rows, cols)
    if starts is not None:
        c["starts"] = torch.as_tensor((r.random(T) < starts).astype(np.uint8)).cuda()
    return c


def _run(c, **kw):
    W = c["weight"].shape[1]
    y, out = torch.empty_like(c["x"]), torch.empty((W - 1,) + c["x"].shape[1:], dtype=c["x"].dtype, device="cuda")
    mgn.mgn_causal_conv(c["x"], c["weight"], y, bias=c["bias"], past=c["past"], past_out=out, starts=c["starts"],
                        silu=c["silu"], **kw)
    return y, out


def _back(c, **kw):
    W = c["weight"].shape[1]
    dx, dw, db = torch.empty_like(c["x"]), torch.empty_like(c["weight"]), torch.empty(c["x"].shape[2], device="cuda")
    dp = torch.empty((W - 1,) + c["x"].shape[1:], device="cuda")
    mgn.mgn_causal_conv_grad(c["x"], c["weight"], c["dy"], dx, dw, db, bias=c["bias"], past=c["past"], d_past=dp,
                             d_past_out=c["d_past_out"], starts=c["starts"], silu=c["silu"], **kw)
    return dx, dw, db, dp


def _ref(c):
    o = lambda k: None if c[k] is None else ref.f64(c[k])
    return (ref.f64(c["x"]), ref.f64(c["weight"]), o("bias"), o("past"), None if c["starts"] is None else c["starts"].cpu().numpy(),
            c["silu"])


def _check(c):
    a = _ref(c)
    y64, e, out64 = ref.conv(*a)
    y, out = _run(c)
    ref.near("y", y, y64, e, y.dtype)
    assert np.array_equal(ref.f64(out), out64)  # inputs as they are
    got = _back(c)
    r = ref.conv_grad(*a, ref.f64(c["dy"]), None if c["d_past_out"] is None else ref.f64(c["d_past_out"]))
    for name, g, w, b in zip(("dx", "dw", "db", "d_past"), got, r[:4], r[4:]):
        ref.near(name, g, w, b, g.dtype)
    assert all(torch.equal(p, q) for p, q in zip(_run(c) + _back(c), (y, out) + got))  # the same bits
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols", SHAPES)
def test_conv_and_grad(T, rows, cols, dtype):
    for W in (1, 2, 3, 4, 5, 6, 7, 8) if T * rows * cols < 40000 else (4, 7):
        print(f"[conv] {T} x {rows} x {cols}, {W} {dtype}", flush=True)
        _check(_case(T, rows, cols, W, dtype, silu=W != 3, bias=W != 4))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols", [(1, 5, 64), (6, 3, 5), (20, 103, 64), (200, 1, 77), (700, 2, 128)])
@pytest.mark.parametrize("starts", [0.03, 0.4, 1.1])
def test_trajectories_in_one_window(T, rows, cols, dtype, starts):
    for W in (2, 4, 8):
        print(f"[conv] starts {starts} {T} x {rows} x {cols}, {W} {dtype}", flush=True)
        _check(_case(T, rows, cols, W, dtype, starts=starts, seed=1))
        _check(_case(T, rows, cols, W, dtype, starts=starts, state=False, silu=False, seed=2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,W,starts", [(70, 33_000, 64, 4, True), (131, 140_000, 9, 8, True), (67, 33_000, 62, 3, False)])
def test_long_segments_of_many_rows(T, rows, cols, W, starts, dtype):
    """More than 64 steps at once (whose starts are looked at 64 at a time): some rows."""
    print(f"[conv] long {T} x {rows} x {cols}, {W} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    t = lambda *s: torch.randn(s, generator=g, device="cuda")
    c = dict(x=t(T, rows, cols).to(dtype), weight=t(cols, W), bias=t(cols), silu=True, starts=None,
             past=t(W - 1, rows, cols).to(dtype), dy=t(T, rows, cols).to(dtype), d_past_out=t(W - 1, rows, cols))
    if starts:
        c["starts"] = torch.zeros(T, dtype=torch.uint8, device="cuda")
        c["starts"][[3, 4, 40, 63, 64, 66]] = 1
    got = _run(c) + _back(c)
    some = [0, 15, 16, rows // 2, rows - 1]
    few = {k: v[:, some].contiguous() if k in ("x", "past", "dy", "d_past_out") else v for k, v in c.items()}
    a = _ref(few)
    y64, e, out64 = ref.conv(*a)
    ref.near("y", got[0][:, some], y64, e, dtype)
    assert np.array_equal(ref.f64(got[1][:, some]), out64)
    r = ref.conv_grad(*a, ref.f64(few["dy"]), ref.f64(few["d_past_out"]))
    ref.near("dx", got[2][:, some], r[0], r[4], dtype)
    ref.near("d_past", got[5][:, some], r[3], r[7])


@pytest.mark.parametrize("T,rows,cols", [(9, 30, 64), (700, 1, 33)])
def test_nothing_before_a_start_is_seen(T, rows, cols):
    """NaN and infinite inputs, past and gradients before a start stay there."""
    c = _case(T, rows, cols, 4, torch.float32, seed=3)
    s = T // 2
    c["starts"] = torch.zeros(T, dtype=torch.uint8, device="cuda")
    c["starts"][s] = 1
    y0, out0 = _run(c)
    g0 = _back(dict(c))
    c["x"][:s], c["past"][:] = float("nan"), float("inf")
    y, out = _run(c)
    assert torch.equal(y[s:], y0[s:]) and torch.equal(out, out0)
    dx = _back(c)[0]
    assert torch.equal(dx[s:], g0[0][s:])
    c["starts"][T - 1] = 1
    out = _run(c)[1]
    assert not out[:-1].any() and torch.equal(out[-1], c["x"][-1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("W", [2, 4, 8])
def test_windows_and_single_steps_are_the_whole(W, dtype):
    """A trajectory window by window, down to single steps with `past` updated in
    place, and the windows' backward handing on d_past."""
    T, rows, cols = 90, 3, 40
    c = _case(T, rows, cols, W, dtype, seed=4)
    y, out = _run(c)
    for cuts in (range(0, T + 1), [0, 1, 3, 50, 50, 90], [0, 90]):
        past, ys = c["past"].clone(), []
        cuts = list(cuts)
        for a, b in zip(cuts, cuts[1:]):
            ys.append(torch.empty_like(c["x"][a:b]))
            mgn.mgn_causal_conv(c["x"][a:b], c["weight"], ys[-1], bias=c["bias"], past=past, past_out=past, silu=True)
        assert torch.equal(torch.cat(ys), y) and torch.equal(past, out)
    dx, dw, db, dp = _back(c)
    pasts, cuts = [c["past"]], [0, 1, 4, 45, 90]
    for a, b in zip(cuts, cuts[1:]):
        pasts.append(torch.empty_like(c["past"]))
        mgn.mgn_causal_conv(c["x"][a:b], c["weight"], torch.empty_like(c["x"][a:b]), bias=c["bias"], past=pasts[-2],
                            past_out=pasts[-1], silu=True)
    d, dw2, db2, dxs = c["d_past_out"], torch.empty_like(dw), torch.empty_like(db), []
    for k in range(len(cuts) - 2, -1, -1):
        w = dict(c, x=c["x"][cuts[k]:cuts[k + 1]], dy=c["dy"][cuts[k]:cuts[k + 1]], past=pasts[k], d_past_out=d)
        first = k == len(cuts) - 2
        dxk, d = torch.empty_like(w["x"]), torch.empty_like(d)
        mgn.mgn_causal_conv_grad(w["x"], w["weight"], w["dy"], dxk, dw2, db2, bias=w["bias"], past=w["past"], d_past=d,
                                 d_past_out=w["d_past_out"], silu=True, accumulate=not first)
        dxs.insert(0, dxk)
    # (at a cut one more sum is rounded to fp32, and the sums run in another order)
    r = ref.conv_grad(*_ref(c), ref.f64(c["dy"]), ref.f64(c["d_past_out"]))
    ref.near("dx", torch.cat(dxs), r[0], r[4] * 2, dtype)
    ref.near("dw", dw2, r[1], 2 * r[5] + 5 * ref.U * np.abs(r[1]))
    ref.near("d_past", d, r[3], r[7] * 2)


def test_grad_against_differences():
    T, rows, cols, W, step = 5, 2, 3, 4, 1e-6
    c = _case(T, rows, cols, W, torch.float32, seed=5)
    x, w, b, past, _, _ = _ref(c)
    dy, dpo = ref.f64(c["dy"]), ref.f64(c["d_past_out"])

    def loss(x, w, b, past):
        y, _, out = ref.conv(x, w, b, past, None, True)
        return float((y * dy).sum() + (out * dpo).sum())

    args, got = [x, w, b, past], _back(c)
    for k, g in ((0, got[0]), (1, got[1]), (2, got[2]), (3, got[3])):
        num = np.zeros_like(args[k])
        for i in np.ndindex(num.shape):
            lo, hi = [a.copy() for a in args], [a.copy() for a in args]
            lo[k][i] -= step
            hi[k][i] += step
            num[i] = (loss(*hi) - loss(*lo)) / (2 * step)
        assert np.allclose(ref.f64(g), num, rtol=1e-5, atol=1e-5 * np.abs(num).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols", [(20, 37, 64), (300, 1, 128)])
def test_unaligned_arrays(T, rows, cols, dtype):
    c = _case(T, rows, cols, 4, dtype, starts=0.1, seed=6)

    def at(v, o):
        return torch.full((v.numel() + 8,), 5.0, dtype=v.dtype, device="cuda")[o:o + v.numel()].view(v.shape).copy_(v)

    for o in (1, 2, 3):
        _check(dict(c, x=at(c["x"], o), past=at(c["past"], o), dy=at(c["dy"], (o + 1) % 4), weight=at(c["weight"], 1),
                    d_past_out=at(c["d_past_out"], o)))


def test_nothing_to_do():
    x, w = torch.empty(0, 3, 64, device="cuda"), torch.ones(64, 4, device="cuda")
    past, out = torch.randn(3, 3, 64, device="cuda"), torch.empty(3, 3, 64, device="cuda")
    mgn.mgn_causal_conv(x, w, x, past=past, past_out=out)
    assert torch.equal(past, out)
    mgn.mgn_causal_conv(x, w, x, past_out=out)
    assert not out.any()
    dw, dp = torch.full((64, 4), 2.0, device="cuda"), torch.empty(3, 3, 64, device="cuda")
    mgn.mgn_causal_conv_grad(x, w, x, x, dw, d_past=dp, d_past_out=past, accumulate=True)
    assert bool((dw == 2).all()) and torch.equal(dp, past)
    mgn.mgn_causal_conv_grad(x, w, x, x, dw, d_past=dp)
    assert not dw.any() and not dp.any()
    e = torch.empty(5, 0, 64, device="cuda")
    mgn.mgn_causal_conv(e, w, e)
    mgn.mgn_causal_conv_grad(e, w, e, e, dw)
    assert not dw.any()


def test_streams_and_captured_replays():
    c = _case(40, 100, 64, 4, torch.bfloat16, starts=0.1, seed=7)
    want = _run(c) + _back(c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _run(c, stream=side.cuda_stream) + _back(c, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = _run(c) + _back(c)
    for k in range(4):
        n = _case(40, 100, 64, 4, torch.bfloat16, starts=0.1, seed=20 + k)
        for key in ("x", "weight", "bias", "past", "dy", "d_past_out", "starts"):
            c[key].copy_(n[key])
        g.replay()
        torch.cuda.synchronize()
        kept = [v.clone() for v in got]
        assert all(torch.equal(p, q) for p, q in zip(kept, _run(c) + _back(c)))


def test_offsets_past_32_bits():
    """More than 2^32 elements: the last rows and steps against their own call."""
    T, rows, cols, W = 5, 13_500_000, 64, 4
    c = dict(x=torch.empty(T, rows, cols, dtype=torch.bfloat16, device="cuda"), weight=torch.randn(cols, W, device="cuda"),
             bias=None, silu=True, starts=None, past=None, d_past_out=None)
    for t in range(T):
        c["x"][t].normal_()
    y = torch.empty_like(c["x"])
    mgn.mgn_causal_conv(c["x"], c["weight"], y, silu=True)
    tail = slice(rows - 1000, rows)
    part = c["x"][:, tail].contiguous()
    want = torch.empty_like(part)
    mgn.mgn_causal_conv(part, c["weight"], want, silu=True)
    assert torch.equal(y[:, tail], want)
    dx, dw = torch.empty_like(y), torch.empty_like(c["weight"])
    mgn.mgn_causal_conv_grad(c["x"], c["weight"], y, dx, dw, silu=True)
    dwant = torch.empty_like(part)
    mgn.mgn_causal_conv_grad(part, c["weight"], want, dwant, None, silu=True)
    assert torch.equal(dx[:, tail], dwant)
