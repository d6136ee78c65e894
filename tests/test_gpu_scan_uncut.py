"""The selective scan over long time axes that are not cut, within the bounds of steps
that are taken one after another (no sum of step sizes over a chunk enters a factor)."""
import pytest
import torch

import memory_ref as ref
import paper_2307_13592_amd as mgn
from test_gpu_selective_scan import _backward, _case, _forward, _ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", [(75, 2101, 64, 16), (130, 1100, 62, 11), (67, 1100, 64, 3), (129, 600, 128, 8), (65, 1030, 64, 40)])
def test_long_axes(T, rows, cols, n, dtype):
    c = _case(T, rows, cols, n, dtype, starts=0.02, seed=16)
    assert mgn.mgn_selective_scan_work(T, rows, cols, n) == 0
    y, last, marks = _forward(c)
    g = _backward(c, marks)
    some = [0, 15, 16, rows // 2, rows - 1]
    few = {k: v[:, some].contiguous() if k in ("x", "dt", "B", "C", "z", "dy") else v[some].contiguous() if k in ("h0", "dh_last") else v
           for k, v in c.items()}
    r = _ref(few)
    f = ref.ssm(r)
    ref.near("y", y[:, some], f["y"], f["ey"], dtype)
    ref.near("h_last", last[some], f["last"], f["elast"])
    for m in range(1, marks.shape[0]):
        at = m * mgn.MGN_MARK_STEPS - 1
        ref.near(f"mark {m}", marks[m][some], f["h"][at], f["eh"][at])
    want = ref.ssm_grad(r, f, r["dy"], r["dh_last"], tiles=-(-cols // 64))
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        ref.near(k, g[k][:, some], *want[k], dtype)
    ref.near("dh0", g["dh0"][some], *want["dh0"])
