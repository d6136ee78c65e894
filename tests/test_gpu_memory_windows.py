"""A trajectory in windows: every scan() of a GatedMemory first, then every
grad(), as a training step over a long trajectory does."""
import pytest
import torch

import paper_2307_13592_amd as mgn
from paper_2307_13592_amd.runner import GatedMemory

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,rows,cols", [(6, 40, 64), (30, 7, 5), (600, 2, 64)])
def test_gradients_of_earlier_windows(T, rows, cols):
    r = torch.Generator(device="cuda")
    r.manual_seed(T)
    rand = lambda *s: torch.randn(s, generator=r, device="cuda")
    m = GatedMemory(rows, cols)
    m.state.copy_(rand(rows, cols))
    cuts = [(0, T // 3), (T // 3, T // 2), (T // 2, T)]
    g, x, dh = rand(T, rows, cols), rand(T, rows, cols), rand(T, rows, cols)
    starts, hs = [], []
    for a, b in cuts:
        starts.append(m.state.clone())
        hs.append(m.scan(g[a:b], x[a:b]))
    assert torch.equal(m.h0, starts[-1])
    carry = None
    for (a, b), h, h0 in reversed(list(zip(cuts, hs, starts))):
        want = torch.empty_like(g[a:b]), torch.empty_like(g[a:b]), torch.empty_like(h0)
        mgn.mgn_gated_scan_grad(g[a:b], x[a:b], h, want[0], want[1], dh=dh[a:b], dh_last=carry, dh0=want[2], h0=h0)
        got = m.grad(g[a:b], x[a:b], h, dh[a:b], carry)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), (a, b)
        carry = want[2]
    # from a copy of the first window's states, with its start given
    a, b = cuts[0]
    one = m.grad(g[a:b], x[a:b], hs[0].clone(), dh[a:b], h0=starts[0])
    two = m.grad(g[a:b], x[a:b], hs[0], dh[a:b])
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    # a copy of the last window's states: that of the last scan()
    a, b = cuts[-1]
    one = m.grad(g[a:b], x[a:b], hs[-1].clone(), dh[a:b])
    two = m.grad(g[a:b], x[a:b], hs[-1], dh[a:b])
    assert all(torch.equal(p, q) for p, q in zip(one, two))
