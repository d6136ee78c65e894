"""Rows of the root-mean-square norm at the ends of the fp32 range: a finite row
whose squares pass it gives zeros and takes no gradient (but d_total), whatever
dy and the weight are; its neighbours and dweight do not notice it."""
import pytest
import torch

import paper_2307_13592_amd as mgn
from paper_2307_13592_amd.runner import LatentCache

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [1, 5, 16, 64, 77, 128, 300, 1000, 1500, 4100, 8191])
def test_rows_past_the_range(cols, dtype):
    print(f"[rms] rows past the fp32 range, {cols} columns {dtype}", flush=True)
    n = 24
    r = torch.Generator(device="cuda")
    r.manual_seed(cols)
    t = torch.randn(n, cols, generator=r, device="cuda")
    dy = torch.randn(n, cols, generator=r, device="cuda").to(dtype)
    ds = torch.randn(n, cols, generator=r, device="cuda").to(dtype)
    w = torch.full((cols,), 2.0, device="cuda")
    big = [2, 3, 9, 11, 23]
    keep = [i for i in range(n) if i not in big]
    t[2] = 1e20 * t[2].sign()
    t[3] = 3e38
    t[9] = 1e37
    t[11] = 3e38 * t[11].sign()
    t[23, 0] = -3e38
    t = t.to(dtype)
    dy[3], dy[9], dy[23] = 1, 1, 2  # their sum of t w dy passes the range too
    small = t.clone()
    small[big] = 0
    y0, y = torch.empty_like(t), torch.empty_like(t)
    mgn.mgn_rms_norm(small, w, y0, eps=EPS)
    mgn.mgn_rms_norm(t, w, y, eps=EPS)
    assert torch.equal(y, y0) and not y[big].any()
    c = LatentCache(n, cols)
    mgn.mgn_rms_norm(t, w, c.q, y_scale=c.scale, eps=EPS)
    assert not (c.q[big] & 0x7f).any() and bool((c.scale[big] == 1).all())  # zeros of either sign
    for d_total in (None, ds):
        dx0, dx = torch.empty_like(t), torch.empty_like(t)
        dw0, dw = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        mgn.mgn_rms_norm_grad(small, w, dy, dx0, dw0, d_total=d_total, eps=EPS)
        mgn.mgn_rms_norm_grad(t, w, dy, dx, dw, d_total=d_total, eps=EPS)
        assert torch.equal(dx[keep], dx0[keep])
        assert torch.equal(dx[big], torch.zeros_like(dx[big]) if d_total is None else ds[big])
        assert torch.equal(dw, dw0)


@pytest.mark.parametrize("cols", [64, 77, 1500])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite_have_nan_gradients(cols, value):
    t = torch.randn(9, cols, device="cuda")
    dy = torch.randn(9, cols, device="cuda")
    t[4, cols - 1] = value
    clean = t.clone()
    clean[4] = 0
    dx0, dx = torch.empty_like(t), torch.empty_like(t)
    mgn.mgn_rms_norm_grad(clean, None, dy, dx0, eps=EPS)
    mgn.mgn_rms_norm_grad(t, None, dy, dx, eps=EPS)
    assert bool(dx[4].isnan().all())
    keep = [0, 1, 2, 3, 5, 6, 7, 8]
    assert torch.equal(dx[keep], dx0[keep])
