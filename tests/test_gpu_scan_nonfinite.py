"""NaN and infinite gates, inputs and states in the gated recurrence: they
reach what the definition says and nothing else, however the time axis is
dealt to waves and workgroups."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref

pytestmark = pytest.mark.gpu
# one column a lane: a wave alone (few steps; many odd columns), four waves,
# eight, chunks of one tile and of several; four columns a lane: a wave alone, four
DEALS = [(8, 30, 64), (40, 2101, 63), (30, 3, 64), (400, 160, 128), (1000, 3, 64), (2050, 50, 128), (40, 1700, 128),
         (40, 600, 128)]


def _inputs(T, rows, cols, seed, gate=0.0):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=r, device="cuda")
    return dict(g=2 * rand(T, rows, cols) + gate, x=rand(T, rows, cols), h0=rand(rows, cols), dh=rand(T, rows, cols),
                dh_last=rand(rows, cols), starts=torch.zeros(T, dtype=torch.uint8, device="cuda"))


def _run(c):
    h, last = torch.empty_like(c["g"]), torch.empty_like(c["h0"])
    mgn.mgn_gated_scan(c["g"], c["x"], h=h, h_last=last, h0=c["h0"], starts=c["starts"])
    dg, dx, dh0 = torch.empty_like(c["g"]), torch.empty_like(c["x"]), torch.empty_like(c["h0"])
    mgn.mgn_gated_scan_grad(c["g"], c["x"], h, dg, dx, dh=c["dh"], dh_last=c["dh_last"], dh0=dh0, h0=c["h0"],
                            starts=c["starts"])
    return dict(h=h, last=last, dg=dg, dx=dx, dh0=dh0)


def _like(what, got, want, bound):
    """NaN and infinities where the definition has them, the rest within the bound."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), what
    assert np.all(np.abs(got[fin] - want[fin]) <= bound[fin]), what


def _against_definition(c, out, cols):
    """`out` against float64, in the columns (of the flattened rows) given."""
    T = c["g"].shape[0]
    at = lambda t: ref.f64(t.view(t.shape[0], -1)[:, cols])[:, None] if t.dim() == 3 else ref.f64(t.view(-1)[cols])[None]
    st = c["starts"].cpu().numpy()
    with np.errstate(all="ignore"):
        h, e = ref.scan(at(c["g"]), at(c["x"]), at(c["h0"]), st)
        _like("h", at(out["h"]), h, e)
        dg, dx, d0, eg, ex, e0 = ref.scan_grad(at(c["g"]), at(c["x"]), at(out["h"]), at(c["h0"]), st, at(c["dh"]),
                                               at(c["dh_last"]))
    # (the results' own half-step; E carries the rest)
    _like("dg", at(out["dg"]), dg, eg + np.abs(dg) * 2 * ref.U32)
    _like("dx", at(out["dx"]), dx, ex + np.abs(dx) * 2 * ref.U32)
    _like("dh0", at(out["dh0"]), d0, e0)


@pytest.mark.parametrize("reset", ["start", "replaced"])
@pytest.mark.parametrize("T,rows,cols", DEALS)
def test_nan_gate_ends_with_its_trajectory(T, rows, cols, reset):
    """A NaN gate is gone (forward) behind the next start or gate of -inf, and
    (backward) before the one that precedes it."""
    print(f"[scan] NaN gate, then {reset}: T={T} {rows} x {cols}", flush=True)
    C = rows * cols
    for k, (a, bad, b) in enumerate([(1, 2, 3), (max(0, T // 3 - 9), T // 3, T // 3 + 2),
                                     (T // 2 - 1, T // 2, T // 2 + 1), (max(2, T - 12), T - 3, T - 2)]):
        if not a < bad < b < T:
            continue
        c = _inputs(T, rows, cols, seed=k)
        col = [0, C // 2, C - 1]
        if reset == "start":
            c["starts"][[a, b]] = 1
        else:
            c["g"].view(T, C)[a, col] = c["g"].view(T, C)[b, col] = -float("inf")
        clean = _run(c)
        c["g"].view(T, C)[bad, col] = float("nan")
        out = _run(c)
        hit = torch.zeros(T, C, dtype=torch.bool, device="cuda")
        hit[bad:b, col] = True  # the states that the NaN reaches
        assert torch.equal(out["h"].view(T, C).isnan(), hit)
        assert torch.equal(out["h"].view(T, C)[~hit], clean["h"].view(T, C)[~hit])
        assert bool(out["last"].isfinite().all()) and bool(out["dh0"].isfinite().all())
        _against_definition(c, out, col + [C // 3])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,rows,cols", DEALS + [(8192, 3, 64), (8192, 1, 1)])
def test_nonfinite_states_last(T, rows, cols, value):
    """A state (backward: a gradient) that is NaN or infinite stays so, however
    far its finite part would have decayed, to the next start or gate of -inf."""
    print(f"[scan] a state of {value} lasts: T={T} {rows} x {cols}", flush=True)
    C = rows * cols
    col = [0, C // 2, C - 1]
    for where in ("x", "h0"):
        c = _inputs(T, rows, cols, seed=4)
        clean = _run(c)
        if where == "x":
            c["x"].view(T, C)[1, col] = value
            c["dh"].view(T, C)[T - 2, col] = value
        else:
            c["h0"].view(C)[col] = value
            c["dh_last"].view(C)[col] = value
        out = _run(c)
        first = 1 if where == "x" else 0
        bad = out["h"].view(T, C)[first:, col]
        assert bool(bad.isnan().all()) if value != value else bool((bad == value).all())
        assert not bool(out["dh0"].view(C)[col].isfinite().any())
        keep = torch.ones(C, dtype=torch.bool, device="cuda")
        keep[col] = False
        for k in ("h", "dg", "dx"):
            assert torch.equal(out[k].view(T, C)[:, keep], clean[k].view(T, C)[:, keep]), k
        _against_definition(c, out, col)
        # and with a start and a replaced state far behind
        a, b = T // 3, T - T // 3
        c["starts"][a] = 1
        c["g"].view(T, C)[b, col] = -float("inf")
        out = _run(c)
        assert bool(out["h"].view(T, C)[a:].isfinite().all()) and bool(out["dh0"].isfinite().all())
        _against_definition(c, out, col)


def test_nan_gate_leaves_neighbours_alone():
    c = _inputs(1000, 3, 64, seed=9)
    clean = _run(c)
    c["g"][17, 1, 5] = float("nan")
    out = _run(c)
    for k in ("h", "dg", "dx"):
        keep = torch.ones_like(out[k], dtype=torch.bool)
        keep[:, 1, 5] = False
        assert torch.equal(out[k][keep], clean[k][keep]), k
    _against_definition(c, out, [69, 0])


@pytest.mark.parametrize("T,rows,cols", [(1000, 3, 64), (2050, 50, 128), (40, 600, 128)])
def test_large_states_decay(T, rows, cols):
    """A finite state of 1e30 leaves no more than the smallest number's share
    behind (2^-149 of it, below half a step of states near 1e-6)."""
    c = _inputs(T, rows, cols, seed=5, gate=-1.0)
    c["h0"].mul_(1e30)
    c["dh_last"].mul_(1e30)
    _against_definition(c, _run(c), [0, 1, rows * cols // 2, rows * cols - 1])


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,rows,cols", DEALS)
def test_gradients_that_are_not_finite_where_state_and_input_agree(T, rows, cols, value):
    """h_{t-1} = x: dg is 0 times the gradient D, 0 for a finite D and NaN for
    others, unless the step holds or replaces its state."""
    C = rows * cols
    c = _inputs(T, rows, cols, seed=6)
    col = [0, C // 2, C - 1]
    c["x"].view(T, C)[:, col] = 0
    c["h0"].view(C)[col] = 0
    c["dh"].view(T, C)[T - 1, col] = value
    c["g"].view(T, C)[T - 1, 0] = float("inf")  # held
    c["g"].view(T, C)[T // 2, C // 2] = -float("inf")  # replaced
    out = _run(c)
    dg = out["dg"].view(T, C)
    assert float(dg[T - 1, 0]) == 0 and bool(dg[T - 1, col[1:]].isnan().all())
    assert not dg[:T // 2 + 1, C // 2].any()
    _against_definition(c, out, col + [C // 3])
