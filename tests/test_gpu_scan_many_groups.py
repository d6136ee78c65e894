"""A selective scan of more groups of columns than one launch takes (2^28): rows at both
sides of the border and the last ones against their own call, to the bit."""
import pytest
import torch

import paper_2307_13592_amd as mgn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 2])
def test_several_launches(T):
    rows, cols, n = (1 << 28) // 16 + 70_001, 64, 1
    assert rows * (cols // 4) > 1 << 28
    big = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    x, dt, B, C, y = big(T, rows, cols), big(T, rows, cols), big(T, rows, n), big(T, rows, n), big(T, rows, cols)
    for v in (x, dt, B, C):
        for t in range(T):
            v[t].normal_()
    A, h = -torch.rand(cols, n, device="cuda"), torch.empty(rows, cols, n, device="cuda")
    assert mgn.mgn_selective_scan_work(T, rows, cols, n) == 0
    mgn.mgn_selective_scan(x, dt, A, B, C, y, h_last=h, softplus=True)
    border = (1 << 28) // 16
    for a, b in ((0, 40), (border - 40, border + 40), (rows - 3000, rows)):
        p = [v[:, a:b].contiguous() for v in (x, dt, B, C)]
        py, ph = torch.empty_like(p[0]), torch.empty(b - a, cols, n, device="cuda")
        mgn.mgn_selective_scan(p[0], p[1], A, p[2], p[3], py, h_last=ph, softplus=True)
        assert torch.equal(y[:, a:b], py) and torch.equal(h[a:b], ph), (a, b)
