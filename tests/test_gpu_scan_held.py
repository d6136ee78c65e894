"""Held and replaced states of the gated recurrence in every dealing of the time
axis: a gate of +inf (or the type's largest value) holds a state through steps
whose x is NaN or infinite, -inf (or the lowest value) replaces one that is NaN,
and what is left out has no gradient."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref
from paper_2307_13592_amd.runner import LatentCache

pytestmark = pytest.mark.gpu
# (steps, rows, cols, one wave goes through all steps): one column a lane, four
SHAPES = [(8, 30, 64, True), (40, 2101, 63, True), (30, 3, 64, False), (400, 160, 128, False), (1000, 3, 64, False),
          (2050, 50, 128, False), (4, 600, 128, True), (9, 1700, 128, True), (9, 600, 128, False), (40, 600, 128, False)]


@pytest.mark.parametrize("typ,x8", [("fp32", False), ("bf16", False), ("fp32", True), ("bf16", True)])
@pytest.mark.parametrize("T,rows,cols,alone", SHAPES)
def test_held_and_replaced(T, rows, cols, alone, typ, x8):
    print(f"[scan] held and replaced T={T} {rows} x {cols} {typ} x8={x8}", flush=True)
    dt = torch.float32 if typ == "fp32" else torch.bfloat16
    big = torch.finfo(dt).max
    r = torch.Generator(device="cuda")
    r.manual_seed(T + rows)
    rand = lambda *s: torch.randn(s, generator=r, device="cuda")
    where = lambda p: torch.rand(T, rows, cols, generator=r, device="cuda") < p
    g, x = (1 + 2 * rand(T, rows, cols)).to(dt), rand(T, rows, cols)
    hold = where(0.3)
    hold[0, 0] = False
    g[hold] = float("inf")
    g[hold & where(0.5)] = big
    g[0, 0], g[0, 0, ::2] = -float("inf"), -big
    x[0, 0] = 1.5
    xs = None
    if x8:
        cache = LatentCache(T * rows, cols)
        cache.store(x.view(T * rows, cols))
        x, xs = cache.window(0, T, rows)
        x[hold] = 0x7f  # NaN
    else:
        x = x.to(dt)
        x[hold] = float("nan")
        x[hold & where(0.5)] = -float("inf")
    h0, dh, dl = rand(rows, cols), rand(T, rows, cols), rand(rows, cols)
    h0[0] = float("nan")
    h, last = torch.empty(T, rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    mgn.mgn_gated_scan(g, x, h=h, h_last=last, h0=h0, x_scale=xs)
    assert bool(h.isfinite().all()) and torch.equal(last, h[-1])
    assert bool((h[0, 0] == 1.5).all())  # (1.5 is exact in 8 bits)
    prev = torch.cat([h0[None], h[:-1]])
    if alone:
        assert torch.equal(h[hold], prev[hold])  # the same bits
    dg, dx, d0 = torch.empty_like(g), torch.empty_like(g), torch.empty_like(h0)
    mgn.mgn_gated_scan_grad(g, x, h, dg, dx, dh=dh, dh_last=dl, dh0=d0, h0=h0, x_scale=xs)
    assert all(bool(v.isfinite().all()) for v in (dg, dx, d0))
    assert not dg[hold].any() and not dx[hold].any() and not dg[0, 0].any() and not d0[0].any()
    # rows 0, 1 and the last against float64 (the definition leaves the same terms out)
    at = [0, 1, rows - 1]
    f = lambda v: ref.f64(v[..., at, :])
    x64 = ref.values8(x[:, at], xs[:, at]) if x8 else f(x)
    h64, e = ref.scan(f(g), x64, f(h0), None)
    assert np.all(np.abs(f(h) - h64) <= e)
    held = hold[:, at].cpu().numpy()
    before = np.concatenate([f(h0)[None], f(h)[:-1]])
    eb = np.concatenate([np.zeros_like(e[:1]), e[:-1]])
    assert np.all(np.abs(f(h) - before)[held] <= (e + eb)[held])
    a, b, c, ea, ebx, ec = ref.scan_grad(f(g), x64, f(h), f(h0), None, f(dh), f(dl))
    u = ref.half(dt) + ref.U32
    assert np.all(np.abs(f(dg) - a) <= ea + np.abs(a) * u)
    assert np.all(np.abs(f(dx) - b) <= ebx + np.abs(b) * u)
    assert np.all(np.abs(f(d0) - c) <= ec)
